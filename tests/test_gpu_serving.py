"""The serving operators against plain implementations in 64 bits (or plain integers), at the sizes where they can go wrong.

Tolerances.  u = unit roundoff of the result's type (2^-8 bfloat16, 2^-11 fp16), e = 2^-24.  A result is rounded once:
|out - exact| <= u |exact| + (error of the fp32 value) + the type's smallest subnormal.  The fp32 errors are derived at each test.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def mmv():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2506_23906_b200 as m
    m.debug_configure(0, -1)
    return m


def inside(got, want, bound):
    """|got - want| <= bound everywhere (the same NaN and infinities in both)."""
    got, want, bound = got.double(), want.double(), bound.double() if torch.is_tensor(bound) else torch.full_like(want, bound)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    over = ((got - want).abs() - bound)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0.0, f"outside the bound by {float(over.max())}"


def ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


# ---------------------------------------------------------------------------------------------------------------------
# block tables
# ---------------------------------------------------------------------------------------------------------------------
def tables_plain(past, added, free, table, nslots, block):
    """Token by token; what does not fit gets slot -1 and no table entry."""
    table, slots, off, at = [list(r) for r in table], [], [0], 0
    width = len(table[0]) if table else 0
    for r in range(len(past)):
        had, need = -(-past[r] // block), -(-(past[r] + added[r]) // block)
        for p in range(past[r], past[r] + added[r]):
            b = p // block
            t = len(slots)
            if b >= width:
                slots.append(-1)
                continue
            if b >= had:
                k = at + b - had
                if k >= len(free):
                    slots.append(-1)
                    continue
                if p % block == 0 and t < nslots:
                    table[r][b] = free[k]
                entry = free[k]
            else:
                entry = table[r][b]
            slots.append(entry * block + p % block if entry >= 0 else -1)
        at += need - had
        off.append(len(slots))
    return table, (slots + [-1] * nslots)[:nslots], off, [a + b for a, b in zip(past, added)], [min(at, len(free))]


def run_tables(mmv, past, added, free, table, nslots, block, stride=None):
    n, width = len(past), len(table[0]) if table else 0
    wide = torch.full((max(n, 1), (stride or width) + 1), 777, dtype=torch.int32, device="cuda")
    td = wide[:n, :width]
    if n and width:
        td.copy_(ints(table))
    guard = torch.full((nslots + 7,), -99, dtype=torch.int64, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    off, total, used = mmv.block_tables(ints(past), ints(added), ints(free), td, guard[:nslots], block, workspace=ws)
    status = mmv.last_async_status(ws)
    assert (guard[nslots:] == -99).all() and (wide[:, width:] == 777).all()
    return (td.tolist(), guard[:nslots].tolist(), off.tolist(), total.tolist(), used.tolist()), status


@pytest.mark.parametrize("n", [1, 2, 31, 255, 1024, 1025, 3000])
@pytest.mark.parametrize("block", [1, 7, 16, 64])
def test_block_tables(mmv, n, block):
    rng = np.random.default_rng(n * 100 + block)
    top = max(2, 30000 // n)
    past = rng.integers(0, top, n) * (rng.random(n) < 0.6)
    added = rng.integers(0, top, n) * (rng.random(n) < 0.7)
    if n == 255:
        added[:] = 1                                              # a decoding step
    past, added = past.tolist(), added.tolist()
    had = [-(-p // block) for p in past]
    fresh = sum(-(-(p + a) // block) - h for p, a, h in zip(past, added, had))
    width = max(-(-(p + a) // block) for p, a in zip(past, added)) + 2
    ids = rng.permutation(sum(had) + fresh + 5).tolist()
    table, at = [], 0
    for h in had:
        table.append(ids[at:at + h] + [-5] * (width - h))
        at += h
    want = tables_plain(past, added, ids[at:], table, sum(added) + 3, block)
    got, status = run_tables(mmv, past, added, ids[at:], table, sum(added) + 3, block, stride=width + 4)
    assert status == 0
    for g, w in zip(got, want):
        assert g == list(w)


@pytest.mark.parametrize("past,added", [([0], [0]), ([5], [0]), ([0], [1]), ([15], [1]), ([16], [1]), ([16], [17]),
                                        ([0, 0, 0], [0, 0, 0]), ([3, 0, 9], [0, 4, 0]), ([0] * 40, [0] * 39 + [33])])
def test_block_tables_by_hand(mmv, past, added):
    table = [[100 * r + b for b in range(6)] for r in range(len(past))]
    want = tables_plain(past, added, list(range(1000, 1040)), table, sum(added), 16)
    got, status = run_tables(mmv, past, added, list(range(1000, 1040)), table, sum(added), 16)
    assert status == 0
    for g, w in zip(got, want):
        assert g == list(w)


def test_block_tables_without_requests(mmv):
    got, status = run_tables(mmv, [], [], [3, 4], [], 9, 16)
    assert status == 0 and got[1] == [-1] * 9 and got[2] == [0] and got[4] == [0]


@pytest.mark.parametrize("short", ["free", "table", "slots", "no free", "no table"])
def test_block_tables_that_do_not_fit(mmv, short):
    past, added, block = [0, 20, 7, 0], [50, 30, 40, 21], 8
    ids = list(range(500, 540))
    width = {"table": 5, "no table": 0}.get(short, 12)
    free = {"free": ids[:6], "no free": []}.get(short, ids)
    table = [[40 + 20 * r + b for b in range(width)] for r in range(4)]
    nslots = 100 if short == "slots" else 150
    want = tables_plain(past, added, free, table, nslots, block)
    got, status = run_tables(mmv, past, added, free, table, nslots, block)
    assert status == 7
    for g, w in zip(got, want):
        assert g == list(w)


@pytest.mark.parametrize("many", [0, 9000])
@pytest.mark.parametrize("past,added,status", [(40, 3, 7), (33, 15, 7), (31, 2, 7), (30, 2, 0), (40, 0, 0)])
def test_block_tables_held_block_past_the_row(mmv, past, added, status, many):
    """New tokens in a block that the request holds and its row does not reach: no slot, and reported (with requests enough for two kernels too)."""
    past, added = [5] * many + [past, 8], [0] * many + [added, 2]
    table = [[10 * r, 10 * r + 1] for r in range(many + 2)]
    want = tables_plain(past, added, [900, 901, 902], table, 20, 16)
    got, code = run_tables(mmv, past, added, [900, 901, 902], table, 20, 16)
    assert code == status
    for g, w in zip(got, want):
        assert g == list(w)


@pytest.mark.parametrize("n,tokens", [(1, 3), (300, 2), (700, 40), (5000, 3), (8192, 150), (8193, 0), (20000, 2)])
@pytest.mark.parametrize("over", ["past", "added"])
def test_block_tables_totals_over_the_lengths(mmv, n, tokens, over):
    """total handed in as past, or as added: every result is that of a buffer of its own (one CTA, several, two kernels; no slots at all)."""
    gen = torch.Generator("cuda").manual_seed(n)
    past, added = (torch.randint(0, top + 1, (n,), device="cuda", generator=gen, dtype=torch.int32) for top in (100, tokens))
    table = torch.randint(0, 1 << 20, (n, 40), device="cuda", generator=gen, dtype=torch.int32)
    free = torch.randperm(1 << 20, device="cuda", generator=gen).to(torch.int32)
    slots = torch.empty(int(added.sum()), dtype=torch.int64, device="cuda")
    want_table, want_slots = table.clone(), slots.clone()
    want = mmv.block_tables(past, added, free, want_table, want_slots, 8)
    for _ in range(3):
        p, a, t = past.clone(), added.clone(), table.clone()
        slots.fill_(-7)
        got = mmv.block_tables(p, a, free, t, slots, 8, total=p if over == "past" else a)
        assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(t, want_table) and torch.equal(slots, want_slots)
        assert got[1].data_ptr() == (p if over == "past" else a).data_ptr() and torch.equal(*((a, added) if over == "past" else (p, past)))


def test_block_tables_bad_lengths_are_reported(mmv):
    table = [[7, 8], [9, 10]]
    got, status = run_tables(mmv, [-4, 3], [5, -1], [1, 2], table, 5, 16)
    assert status == 4
    assert got[2] == [0, 5, 5] and got[3] == [5, 3] and got[1] == [16, 17, 18, 19, 20]
    got, status = run_tables(mmv, [2 ** 31 - 3, 0], [9, 4], [1, 2], table, 8, 16)
    assert status == 4 and got[3][0] == 2 ** 31 - 1


def test_block_tables_more_requests_than_shared_memory_holds(mmv):
    """Closed form: request r holds r % 5 tokens and adds r % 3, block size 4 (a held block each where r % 5 > 0)."""
    for n in (8192, 8193, 70001):
        r = np.arange(n)
        past, added = r % 5, r % 3
        had, need = -(-past // 4), -(-(past + added) // 4)
        fresh = need - had
        table = np.full((n, 2), -1, dtype=np.int32)
        table[:, 0] = np.where(had > 0, r, -1)
        free = (10 ** 6 + np.arange(fresh.sum())).astype(np.int32)
        base = np.cumsum(fresh) - fresh
        want = table.copy()
        for b in range(2):
            sel = (b >= had) & (b < need)
            want[sel, b] = free[base[sel] + b - had[sel]]
        tok = np.repeat(r, added)
        off = np.concatenate([[0], np.cumsum(added)])
        p = past[tok] + np.arange(tok.size) - off[tok]
        slots = want[tok, p // 4].astype(np.int64) * 4 + p % 4
        td = torch.from_numpy(table).cuda()
        sd = torch.empty(tok.size + 2, dtype=torch.int64, device="cuda")
        o, t, u = mmv.block_tables(ints(past), ints(added), torch.from_numpy(free).cuda(), td, sd, 4)
        assert np.array_equal(td.cpu().numpy(), want)
        assert np.array_equal(sd.cpu().numpy(), np.concatenate([slots, [-1, -1]]))
        assert np.array_equal(o.cpu().numpy(), off) and np.array_equal(t.cpu().numpy(), past + added) and u.item() == fresh.sum()


# ---------------------------------------------------------------------------------------------------------------------
# the write into the cache
# ---------------------------------------------------------------------------------------------------------------------
def paged(blocks, block, heads, dim, dtype, order="bthd", pad=0):
    """Two caches in the given order of their axes in memory, with `pad` unused columns of 8 behind each head's row."""
    size = {"b": blocks, "t": block, "h": heads}
    shape = [size[c] for c in order[:3]] + [dim + pad]
    perm = [order.index(c) for c in "bth"] + [3]
    return [torch.randn(shape, device="cuda").to(dtype).permute(perm)[..., :dim] for _ in range(2)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,heads,dim,block,order,pad", [
    (1, 1, 8, 1, "bthd", 0), (3, 2, 64, 16, "bthd", 0), (77, 5, 80, 7, "bhtd", 8), (513, 8, 128, 16, "bthd", 0), (1000, 3, 256, 32, "hbtd", 16),
    (20000, 8, 128, 64, "bthd", 0)])
def test_kv_append(mmv, dtype, tokens, heads, dim, block, order, pad):
    rng = np.random.default_rng(tokens)
    blocks = -(-tokens // block) + 2
    kc, vc = paged(blocks, block, heads, dim, dtype, order, pad)
    kc0, vc0 = kc.clone(), vc.clone()
    qkv = torch.randn(tokens, 2 * heads + 1, dim, device="cuda").to(dtype)
    k, v = qkv[:, :heads], qkv[:, heads:2 * heads]
    slots = rng.permutation(blocks * block)[:tokens].astype(np.int64)
    slots[rng.random(tokens) < 0.1] = -1
    if tokens > 2:
        slots[-1] = blocks * block                               # past the end: skipped
        slots[-2] = 2 ** 40
    mmv.kv_append(k, v, torch.from_numpy(slots).cuda(), kc, vc)
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < blocks * block:
            kc0[s // block, s % block] = k[t]
            vc0[s // block, s % block] = v[t]
    assert torch.equal(kc, kc0) and torch.equal(vc, vc0)


def test_kv_append_slots_past_32_bits_of_bytes(mmv):
    """A cache of more than 2^32 elements, written at its far end."""
    blocks, block, heads, dim = (1 << 32) // (64 * 2 * 64) + 3, 64, 2, 64
    kc = torch.zeros(blocks, block, heads, dim, dtype=torch.float16, device="cuda")
    vc = torch.zeros(blocks, block, heads, dim, dtype=torch.float16, device="cuda")
    k = torch.randn(70, heads, dim, device="cuda").half()
    v = torch.randn(70, heads, dim, device="cuda").half()
    slots = blocks * block - 1 - torch.arange(70, device="cuda")
    mmv.kv_append(k, v, slots, kc, vc)
    assert torch.equal(kc.view(-1, heads, dim)[-70:].flip(0), k) and torch.equal(vc.view(-1, heads, dim)[-70:].flip(0), v)
    assert int((kc.view(-1, heads, dim)[:1 << 20] != 0).sum()) == 0


def test_kv_append_nothing(mmv):
    kc, vc = paged(2, 4, 1, 8, torch.float16)
    k0 = kc.clone()
    e = torch.empty(0, 1, 8, dtype=torch.float16, device="cuda")
    mmv.kv_append(e, e, torch.empty(0, dtype=torch.int64, device="cuda"), kc, vc)
    assert torch.equal(kc, k0)


# ---------------------------------------------------------------------------------------------------------------------
# linear attention, one token
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,heads,kv,dk,dv", [(1, 1, 1, 8, 8), (2, 4, 2, 64, 64), (3, 6, 1, 40, 72), (1, 16, 16, 128, 128), (64, 16, 4, 128, 128),
                                              (130, 5, 5, 128, 96), (7, 3, 3, 16, 128)])
@pytest.mark.parametrize("in_place", [False, True])
def test_linear_step(mmv, dtype, n, heads, kv, dk, dv, in_place):
    """State: one rounding of exp(g) (2 units in the last place: 4 e), of exp(g) S and of the fused sum: <= 8 e (|exp(g) S| + |k v|).
    Result: a sum of dk products of q with such states, in any order: (dk + 8) e on the sum of magnitudes."""
    gen = torch.Generator("cuda").manual_seed(n * 7 + dk)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=gen)                                        # noqa: E731
    q, kk, v = rand(n, heads, dk).to(dtype), rand(n, kv, dk + 8).to(dtype)[..., :dk], rand(n, kv, dv).to(dtype)
    g = -torch.rand(heads, device="cuda", generator=gen) * 2
    g[0] = 0.0
    if heads > 2:
        g[1], g[2] = -float("inf"), -200.0
    pool = n + 3
    state = rand(pool, heads, dk, dv)
    slots = torch.randperm(pool, device="cuda", generator=gen)[:n].to(torch.int32)
    if n > 2:
        slots[1] = -1
        slots[2] = pool
    before = state.clone()
    target = state if in_place else torch.full_like(state, 7.0)
    untouched = target.clone()
    out = mmv.linear_attention_step(q, kk, v, g, state, scale=0.3, slots=slots, state_out=target)
    on = [r for r in range(n) if 0 <= slots[r] < pool]
    at = slots[on].long()
    rep = heads // kv
    kd, vd = kk.double().repeat_interleave(rep, 1)[on], v.double().repeat_interleave(rep, 1)[on]
    old = torch.exp(g.double())[:, None, None] * before[at].double()
    new = kd[..., :, None] * vd[..., None, :]
    inside(target[at], old + new, 8 * E * (old.abs() + new.abs()))
    rest = torch.ones(pool, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert torch.equal(target[rest], untouched[rest])
    want = 0.3 * torch.einsum("nhk,nhkv->nhv", q[on].double(), old + new)
    size = 0.3 * torch.einsum("nhk,nhkv->nhv", q[on].double().abs(), old.abs() + new.abs())
    inside(out[on], want, U[dtype] * want.abs() + (dk + 16) * E * size + TINY[dtype])
    off = [r for r in range(n) if r not in on]
    assert (out[off] == 0).all()


def test_linear_step_own_index_and_nothing(mmv):
    q = torch.randn(4, 2, 16, device="cuda").half()
    state = torch.randn(5, 2, 16, 16, device="cuda")
    g = torch.tensor([-0.5, -1.0], device="cuda")
    a, s1, s2 = torch.arange(4, dtype=torch.int32, device="cuda"), torch.zeros_like(state), torch.zeros_like(state)
    assert torch.equal(mmv.linear_attention_step(q, q, q, g, state, state_out=s1), mmv.linear_attention_step(q, q, q, g, state, slots=a, state_out=s2))
    assert torch.equal(s1, s2)
    assert mmv.linear_attention_step(q[:0], q[:0], q[:0], g, state).shape == (0, 2, 16)


# ---------------------------------------------------------------------------------------------------------------------
# attention of one token over the paged cache
# ---------------------------------------------------------------------------------------------------------------------
def paged_case(seed, lens, heads, kv, dim, block, dtype, order="bthd", pad=0, spare=3, garbage=float("nan"), far=0):
    """Caches filled with `garbage` except at the requests' own tokens, pages in random order, the rest of the table out of range."""
    gen = torch.Generator("cuda").manual_seed(seed)
    pages = [-(-n // block) for n in lens]
    blocks = sum(pages) + spare + far
    kc, vc = paged(blocks, block, kv, dim, dtype, order, pad)
    ids = (far + torch.randperm(sum(pages) + spare, device="cuda", generator=gen)).tolist()
    table = torch.full((len(lens), max(pages + [1]) + 1), -7, dtype=torch.int32, device="cuda")
    wide = torch.full((len(lens), table.size(1) + 3), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    keep = torch.zeros(blocks, block, dtype=torch.bool, device="cuda")
    at = 0
    for r, n in enumerate(lens):
        mine = torch.tensor(ids[at:at + pages[r]], dtype=torch.int64, device="cuda")
        at += pages[r]
        table[r, :pages[r]] = mine.to(torch.int32)
        j = torch.arange(n, device="cuda")
        keep[mine[j // block], j % block] = True
    wide[:, :table.size(1)] = table
    for c in (kc, vc):
        c.masked_fill_(~keep[:, :, None, None], garbage)
    q = torch.randn(len(lens), heads, dim + 16, device="cuda", generator=gen).to(dtype)[..., :dim]
    return q, kc, vc, wide[:, :table.size(1)], torch.tensor(lens, dtype=torch.int32, device="cuda")


def paged_plain(q, kc, vc, table, lens, scale, window):
    """Definition in 64 bits, with the magnitudes that the bound needs."""
    n, heads, dim = q.shape
    kv, block = kc.size(2), kc.size(1)
    group = heads // kv
    out = torch.zeros(n, heads, dim, dtype=torch.float64, device="cuda")
    mag, lse, big = torch.zeros_like(out), torch.full((n, heads), -float("inf"), dtype=torch.float64, device="cuda"), torch.zeros(n, heads, device="cuda").double()
    for r, length in enumerate(lens.tolist()):
        if length <= 0:
            continue
        lo = max(0, length - window) if window else 0
        pages = table[r, :-(-length // block)].long()
        for h in range(kv):
            k, v = (c[pages, :, h].reshape(-1, dim)[lo:length].double() for c in (kc, vc))
            rows = slice(h * group, (h + 1) * group)
            x = scale * q[r, rows].double() @ k.T
            w = torch.softmax(x, 1)
            out[r, rows], mag[r, rows], lse[r, rows] = w @ v, w @ v.abs(), torch.logsumexp(x, 1)
            # (a token whose score is -infinity has weight 0 whatever its rounding: it has no part in the bound)
            big[r, rows] = scale * torch.where(torch.isfinite(x), q[r, rows].double().abs() @ k.abs().T, 0.0).amax(1)
    return out, mag, lse, big


def check_paged(mmv, case, dtype, scale, window=0):
    """Scores: a sum of dim products in fp32, (dim + 8) e S with S the largest scale sum |q k|, the base-2 exponent's rounding among it;
    weights: that relative error twice (weight and sum), 2^-16 for the pair of 16-bit values, and the running sums' roundings, one per 16
    tokens of a warp and one per partial result."""
    q, kc, vc, table, lens = case
    n, heads, dim = q.shape
    ws = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    guard = torch.full((n * heads * dim + 64,), 3.0, dtype=dtype, device="cuda")
    out, lse = mmv.paged_attention(q, kc, vc, table, lens, scale=scale, window=window, out=guard[:n * heads * dim].view(n, heads, dim), workspace=ws)
    assert mmv.last_async_status(ws) == 0 and (guard[n * heads * dim:] == 3.0).all()
    want, mag, wlse, big = paged_plain(q, kc, vc, table, lens, scale, window)
    chain = (lens.double() / 16 + 700)[:, None]
    score = (dim + 16) * E * big
    inside(out, want, U[dtype] * want.abs() + mag * (2.0 ** -16 + 3 * score + chain * E)[..., None] + TINY[dtype])
    inside(lse, wlse, torch.nan_to_num(2 * score + chain * E + 8 * E * wlse.abs(), posinf=0.0))
    again, _ = mmv.paged_attention(q, kc, vc, table, lens, scale=scale, window=window)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,kv,dim,block,order,pad", [
    (1, 1, 8, 16, "bthd", 0), (4, 4, 64, 16, "bthd", 0), (8, 1, 40, 7, "bthd", 8), (32, 8, 128, 16, "bthd", 0), (12, 2, 80, 1, "bhtd", 0),
    (71, 1, 64, 64, "hbtd", 0), (48, 2, 128, 48, "bhtd", 16), (16, 2, 256, 16, "bthd", 0), (5, 5, 136, 24, "bthd", 0)])
@pytest.mark.parametrize("lens", [[1], [0, 1, 2, 15, 16, 17, 0], [63, 64, 65, 127, 128, 129], [1000, 3, 0, 517, 2048, 1]])
def test_paged_attention(mmv, dtype, heads, kv, dim, block, order, pad, lens):
    check_paged(mmv, paged_case(dim + len(lens), lens, heads, kv, dim, block, dtype, order, pad), dtype, dim ** -0.5)


@pytest.mark.parametrize("window", [1, 15, 16, 17, 64, 100, 1000, 10 ** 6])
def test_paged_attention_window(mmv, window):
    lens = [1, 16, 17, 100, 101, 640, 999, 0, 1500]
    check_paged(mmv, paged_case(window, lens, 8, 2, 64, 16, torch.float16), torch.float16, 0.125, window)
    check_paged(mmv, paged_case(window + 1, lens, 2, 2, 128, 9, torch.bfloat16), torch.bfloat16, 0.1, window)


@pytest.mark.parametrize("dtype,lens,heads,kv,dim,block", [
    (torch.bfloat16, [70001], 8, 1, 128, 16), (torch.float16, [50000, 1, 0, 2], 4, 2, 64, 64), (torch.bfloat16, [30011], 1, 1, 256, 16),
    (torch.float16, [5] * 700 + [20000] + [0] * 50 + [64] * 300, 16, 4, 64, 16)])
def test_paged_attention_split(mmv, dtype, lens, heads, kv, dim, block):
    """Few long requests over many ranges, and many short ones in each."""
    check_paged(mmv, paged_case(sum(lens), lens, heads, kv, dim, block, dtype), dtype, 1.5 * dim ** -0.5)


def test_paged_attention_large_scores(mmv):
    """Scores of hundreds: the running maximum carries the sum; and equal ones (q = 0): the mean."""
    q, kc, vc, table, lens = paged_case(3, [300, 5000], 8, 2, 64, 16, torch.float16)
    check_paged(mmv, (q * 8, kc, vc, table, lens), torch.float16, 2.0)
    check_paged(mmv, (q * 0, kc, vc, table, lens), torch.float16, 2.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,kv", [(8, 2), (32, 2)])
@pytest.mark.parametrize("gap", [10.0, 14.0, 16.0, 17.5, 20.0])
def test_paged_attention_dominant_tokens_without_a_value(mmv, dtype, heads, kv, gap):
    """Tokens that take almost all of the weight and whose value is zero (four in 256, one for each warp of a tile): the result is made of weights of
    e^-gap.  All of them have the same score and positive values, so the bound is one on the result itself."""
    q, kc, vc, table, lens = paged_case(int(gap), [6000] * 24 + [700, 65], heads, kv, 64, 16, dtype, garbage=0.0)
    q[:] = 0.0
    q[..., 0] = 1.0
    vc.abs_()
    kc[..., 0] = 0.0
    for r, n in enumerate(lens.tolist()):
        j = torch.arange(n, device="cuda")
        j = j[(j % 256 < 64) & (j % 16 == 0)]
        page = table[r, j // 16].long()
        kc[page, j % 16, :, 0] = gap
        vc[page, j % 16] = 0.0
    check_paged(mmv, (q, kc, vc, table, lens), dtype, 1.0)


def test_paged_attention_not_finite_inside(mmv):
    """A NaN among a request's own values stays in that request and head group; scores of -infinity weigh nothing."""
    q, kc, vc, table, lens = paged_case(5, [300, 200, 9000], 4, 2, 64, 16, torch.float16, garbage=0.0)
    vc[table[1, 3], 2, 1, 7] = float("nan")
    kc[table[2, 100], 1, 0, 3] = float("nan")
    out, lse = mmv.paged_attention(q, kc, vc, table, lens)
    bad = torch.isnan(out)
    assert bad[1, 2:, 7].all() and bad[2, :2].all() and int(bad.sum()) == 2 + 2 * 64
    q, kc, vc, table, lens = paged_case(6, [90, 5000], 2, 1, 64, 16, torch.float16, garbage=0.0)
    q[:] = 1.0
    for j in (0, 1, 17, 63, 64, 80):
        for r in range(2):
            kc[table[r, j // 16], j % 16] = -float("inf")
    check_paged(mmv, (q, kc, vc, table, lens), torch.float16, 0.125)
    kc[:] = -float("inf")
    out, lse = mmv.paged_attention(q, kc, vc, table, lens)
    assert (out == 0).all() and (lse == -float("inf")).all()


def test_paged_attention_far_pages(mmv):
    """Pages whose offsets pass 32 bits."""
    far = (1 << 32) // (16 * 2 * 128) + 10
    check_paged(mmv, paged_case(9, [100, 33], 8, 2, 128, 16, torch.float16, garbage=0.0, far=far), torch.float16, 0.1)


def test_paged_attention_bad_metadata_is_reported(mmv):
    q, kc, vc, table, lens = paged_case(11, [100, 50, 70], 4, 2, 64, 16, torch.float16)
    ws = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    good, _ = mmv.paged_attention(q, kc, vc, table, lens)
    for change in ("page", "negative page", "length", "negative length"):
        t, n = table.clone(), lens.clone()
        if change == "page":
            t[1, 2] = kc.size(0)
        elif change == "negative page":
            t[1, 0] = -1
        else:
            n[1] = 10 ** 6 if change == "length" else -5
        out, _ = mmv.paged_attention(q, kc, vc, t, n, workspace=ws)
        assert mmv.last_async_status(ws) == 1
        assert torch.equal(out[[0, 2]], good[[0, 2]])
    mmv.paged_attention(q, kc, vc, table, lens, workspace=ws)
    assert mmv.last_async_status(ws) == 0


def test_paged_attention_without_requests(mmv):
    q, kc, vc, table, lens = paged_case(12, [4], 2, 1, 64, 16, torch.float16)
    ws = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    out, lse = mmv.paged_attention(q[:0], kc, vc, table[:0], lens[:0], workspace=ws)
    assert out.shape == (0, 2, 64) and mmv.last_async_status(ws) == 0
    out, lse = mmv.paged_attention(q, kc, vc, table[:, :0], lens * 0, workspace=ws)      # a table without columns
    assert (out == 0).all() and (lse == -float("inf")).all() and mmv.last_async_status(ws) == 0


# ---------------------------------------------------------------------------------------------------------------------
# linear attention over packed prompts
# ---------------------------------------------------------------------------------------------------------------------
def linear_plain(q, k, v, off, g, scale, state):
    """The recurrence in 64 bits, token by token, and the same recurrence on magnitudes."""
    t, heads, dk = q.shape
    dv, rep, n = v.size(2), heads // k.size(1), len(off) - 1
    q, k, v = q.double(), k.double().repeat_interleave(rep, 1), v.double().repeat_interleave(rep, 1)
    fall = torch.exp(g.double())[:, None, None]
    out, mag = torch.zeros(t, heads, dv, dtype=torch.float64, device="cuda"), torch.zeros(t, heads, dv, dtype=torch.float64, device="cuda")
    last, size = [torch.zeros(n, heads, dk, dv, dtype=torch.float64, device="cuda") for _ in range(2)]
    for s in range(n):
        x = torch.zeros(heads, dk, dv, dtype=torch.float64, device="cuda") if state is None else state[s].double()
        y = x.abs()
        for i in range(off[s], off[s + 1]):
            new = k[i][:, :, None] * v[i][:, None, :]
            x = fall * x + new
            y = fall * y + new.abs()
            out[i] = scale * torch.einsum("hk,hkv->hv", q[i], x)
            mag[i] = scale * torch.einsum("hk,hkv->hv", q[i].abs(), y)
        last[s], size[s] = x, y
    return out, mag, last, size


def linear_case(seed, lens, heads, kv, dk, dv, state=True, first=0, behind=0):
    gen = torch.Generator("cuda").manual_seed(seed)
    off = [first]
    for n in lens:
        off.append(off[-1] + n)
    t = off[-1] + behind
    rand = lambda *s: torch.randn(*s, device="cuda", generator=gen)                                        # noqa: E731
    qkv = rand(t, heads * dk + kv * (dk + dv)).bfloat16()
    q = qkv[:, :heads * dk].view(t, heads, dk)
    k = qkv[:, heads * dk:(heads + kv) * dk].view(t, kv, dk)
    v = qkv[:, (heads + kv) * dk:].view(t, kv, dv)
    g = torch.log1p(-torch.exp2(-torch.linspace(1, 11, heads, device="cuda")))
    if heads > 2:
        g[0], g[1] = 0.0, -float("inf")
    if heads > 3:
        g[2] = -60.0
    return q, k, v, off, g, rand(len(lens), heads, dk, dv) if state else None


def check_linear(mmv, case, scale=0.1, **more):
    """Operands that are formed (scores, the state's copy, decayed keys) are held as sums of at least two bfloat16 values: 2^-16 relative for scores
    and states, less for keys.  States: chains of fp32 sums over the tokens a decay reaches, each rounded or cut (<= 2 e), and decays whose
    exponent and value are rounded (8 e): 2^-20 on the magnitudes covers 2^4 chunks' roundings of a unit each; results: 2^-14."""
    q, k, v, off, g, state = case
    t, heads, dk = q.shape
    dv, n = v.size(2), len(off) - 1
    guard = torch.full((t * heads * dv + 64,), 3.0, dtype=q.dtype, device="cuda")
    out = guard[:t * heads * dv].view(t, heads, dv)
    ws = torch.empty(max(256, mmv.linear_attention_workspace_bytes(q, k, v, n)), dtype=torch.uint8, device="cuda")
    _, last = mmv.linear_attention(q, k, v, ints(off), g, scale=scale, state=state, out=out, workspace=ws, **more)
    assert mmv.last_async_status(ws) == 0
    assert (guard[t * heads * dv:] == 3.0).all() and (out[:off[0]] == 3.0).all() and (out[off[-1]:] == 3.0).all()
    want, mag, wlast, size = linear_plain(q, k, v, off, g, scale, state)
    rows = slice(off[0], off[-1])
    inside(out[rows], want[rows], U[q.dtype] * want[rows].abs() + 2.0 ** -14 * mag[rows] + TINY[q.dtype])
    inside(last, wlast, 2.0 ** -20 * size + 1e-37)
    return out, last


@pytest.mark.parametrize("heads,kv,dk,dv", [(1, 1, 8, 8), (4, 4, 64, 64), (6, 2, 128, 128), (5, 5, 40, 72), (3, 1, 128, 64), (4, 4, 96, 128), (2, 2, 16, 120)])
@pytest.mark.parametrize("lens", [[1], [0, 1, 2, 0], [63, 64, 65], [127, 0, 128, 129, 1], [300, 5, 700]])
@pytest.mark.parametrize("state", [False, True])
def test_linear_attention(mmv, heads, kv, dk, dv, lens, state):
    check_linear(mmv, linear_case(dk + dv + len(lens), lens, heads, kv, dk, dv, state))


def test_linear_attention_rows_outside_the_sequences(mmv):
    check_linear(mmv, linear_case(1, [70, 64, 3], 3, 3, 64, 64, first=37, behind=50))


@pytest.mark.parametrize("lens,heads,dim", [([5000], 1, 128), ([3000, 1, 2500], 2, 64), ([1] * 150 + [900], 3, 128), ([4100, 64, 128, 3000], 4, 128)])
def test_linear_attention_split(mmv, lens, heads, dim):
    """Long sequences of few heads are cut over the CTAs; many short ones share one."""
    check_linear(mmv, linear_case(sum(lens), lens, heads, heads, dim, dim))


def test_linear_attention_neighbours_that_are_not_finite(mmv):
    """Sequences share chunks of memory, not values: NaN and infinities of one stay out of the next and out of the rows in front."""
    q, k, v, off, g, state = linear_case(2, [40, 70, 200], 4, 4, 64, 64)
    want, last = mmv.linear_attention(q, k, v, ints(off), g, state=state)
    q2, k2, v2 = q.clone(), k.clone(), v.clone()
    for x in (q2, k2, v2):
        x[40:110] = float("nan")
    v2[60] = float("inf")
    out, last2 = mmv.linear_attention(q2, k2, v2, ints(off), g, state=state)
    assert torch.equal(out[:40], want[:40]) and torch.equal(out[110:], want[110:]) and torch.equal(last2[[0, 2]], last[[0, 2]])
    assert torch.isnan(out[40:110]).all() and torch.isnan(last2[1]).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tail", [1, 31, 32, 33, 63])
def test_linear_attention_neighbours_that_are_not_finite_in_long_ranges(mmv, dim, tail):
    """Ranges of many chunks, so that a sequence's short last chunk runs between others: its rows behind the end hold the next sequence's NaN and
    infinities, or those of rows that no sequence has.  Every other sequence keeps its results bit by bit, however often it runs."""
    heads, lens = 16, [64 * (1 + 3 * s % 6) + tail for s in range(200)]
    q, k, v, off, g, state = linear_case(dim + tail, lens, heads, heads, dim, dim, first=37, behind=50)
    offsets = ints(off)
    want, last = mmv.linear_attention(q, k, v, offsets, g, scale=0.1, state=state)
    clean = torch.zeros(q.size(0), dtype=torch.bool, device="cuda")
    for s in range(0, 200, 2):
        clean[off[s]:off[s + 1]] = True
    bad = [x.clone() for x in (q, k, v)]
    for i, value in enumerate((float("nan"), float("inf"), -float("inf"))):
        mask = ~clean
        mask[::3] &= i == 0
        mask[1::3] &= i == 1
        mask[2::3] &= i == 2
        for x in bad:
            x[mask] = value
    for _ in range(5):
        out, last2 = mmv.linear_attention(*bad, offsets, g, scale=0.1, state=state)
        assert torch.equal(out[clean], want[clean]) and torch.equal(last2[::2], last[::2])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_linear_attention_later_tokens_do_not_reach_earlier_ones(mmv, dim, bad):
    """A value of v, k or q that is not finite reaches no result in front of its token, and no other column, row or sequence: those stay
    the same bit by bit, but for the tokens of v's column in front of it in its chunk of 64, which are summed up another way and stay
    inside the bound."""
    q, k, v, off, g, state = linear_case(12, [700, 90], 4, 4, dim, dim)
    g[:] = -0.01
    want, last = mmv.linear_attention(q, k, v, ints(off), g, state=state)
    exact, mag, _, _ = linear_plain(q, k, v, off, g, 1.0, state)
    for at in (0, 1, 37, 63, 64, 100, 447, 699):
        x = v.clone()
        x[at, 2, 11] = bad
        x[min(at + 70, 699), 2, 12] = bad
        out, s = mmv.linear_attention(q, k, x, ints(off), g, state=state)
        hit = torch.zeros_like(out, dtype=torch.bool)
        again = torch.zeros_like(hit)
        for col, first in ((11, at), (12, min(at + 70, 699))):
            hit[first:700, 2, col] = True
            again[first // 64 * 64:first, 2, col] = True
        same = ~hit & ~again
        assert torch.equal(out[same], want[same]) and not torch.isfinite(out[hit]).any()
        inside(out[again], exact[again], U[q.dtype] * exact[again].abs() + 2.0 ** -14 * mag[again] + TINY[q.dtype])
        hit = torch.zeros_like(s, dtype=torch.bool)
        hit[0, 2, :, 11:13] = True
        assert torch.equal(s[~hit], last[~hit]) and not torch.isfinite(s[hit]).any()
        x = k.clone()
        x[at, 1, 5] = bad
        out, s = mmv.linear_attention(q, x, v, ints(off), g, state=state)
        hit = torch.zeros_like(out, dtype=torch.bool)
        hit[at:700, 1] = True
        assert torch.equal(out[~hit], want[~hit]) and not torch.isfinite(out[hit]).any()
        assert not torch.isfinite(s[0, 1, 5]).any() and torch.equal(s[1], last[1]) and torch.equal(s[0, [0, 2, 3]], last[0, [0, 2, 3]])
        x = q.clone()
        x[at, 3, 6] = bad
        out, s = mmv.linear_attention(x, k, v, ints(off), g, state=state)
        hit = torch.zeros_like(out, dtype=torch.bool)
        hit[at, 3] = True
        assert torch.equal(out[~hit], want[~hit]) and not torch.isfinite(out[hit]).any() and torch.equal(s, last)


def test_linear_attention_step_continues_a_prompt(mmv):
    """The prompt form's state, taken on by single tokens, is the longer prompt's."""
    q, k, v, off, g, state = linear_case(4, [65, 66], 4, 2, 64, 128)
    want, mag, wlast, size = linear_plain(q, k, v, off, g, 0.2, state)
    pick = torch.cat([torch.arange(0, 64), torch.arange(65, 129)])
    out, s = mmv.linear_attention(q[pick].contiguous(), k[pick].contiguous(), v[pick].contiguous(), ints([0, 64, 128]), g, scale=0.2, state=state)
    at = torch.tensor([64, 129], device="cuda")
    o = mmv.linear_attention_step(q[at].contiguous(), k[at].contiguous(), v[at].contiguous(), g, s, scale=0.2)
    inside(o, want[at], U[torch.bfloat16] * want[at].abs() + 2.0 ** -14 * mag[at])
    o2 = mmv.linear_attention_step(q[130:131], k[130:131], v[130:131], g, s, scale=0.2, slots=ints([1]))
    inside(o2, want[130:131], U[torch.bfloat16] * want[130:131].abs() + 2.0 ** -14 * mag[130:131])
    inside(s[1], wlast[1], 2.0 ** -20 * size[1])


def test_linear_attention_bad_offsets_are_reported(mmv):
    q, k, v, off, g, state = linear_case(7, [64, 64, 64], 2, 2, 64, 64)
    ws = torch.empty(max(256, mmv.linear_attention_workspace_bytes(q, k, v, 3)), dtype=torch.uint8, device="cuda")
    for bad in ([0, 100, 64, 192], [-3, 64, 128, 192], [0, 64, 128, 193], [0, 2 ** 31 - 1, 128, 192]):
        mmv.linear_attention(q, k, v, ints(bad), g, state=state, workspace=ws)
        assert mmv.last_async_status(ws) == 4
    mmv.linear_attention(q, k, v, ints(off), g, state=state, workspace=ws)
    assert mmv.last_async_status(ws) == 0


def test_linear_attention_states_that_overlap_are_refused(mmv):
    q, k, v, off, g, state = linear_case(9, [70, 5], 2, 2, 64, 64)
    both = torch.zeros(3, *state.shape[1:], device="cuda")
    both[:2] = state
    for to in (both[:2], both[1:]):
        with pytest.raises(mmv.MmvError):
            mmv.linear_attention(q, k, v, ints(off), g, state=both[:2], state_out=to)
    _, last = mmv.linear_attention(q, k, v, ints(off), g, state=both[:1].expand(2, -1, -1, -1).contiguous(), state_out=both[1:])
    assert last.data_ptr() == both[1:].data_ptr()


def test_linear_attention_nothing(mmv):
    q, k, v, off, g, state = linear_case(8, [4], 2, 2, 64, 64)
    out, last = mmv.linear_attention(q[:0], k[:0], v[:0], ints([0, 0]), g, state=state)
    assert out.shape == (0, 2, 64) and torch.equal(last, state)
    out, last = mmv.linear_attention(q[:0], k[:0], v[:0], ints([0, 0, 0]), g)
    assert (last == 0).all()
    out, last = mmv.linear_attention(q[:0], k[:0], v[:0], ints([0]), g)
    assert last.shape == (0, 2, 64, 64)


# ---------------------------------------------------------------------------------------------------------------------
# the binding's checks, streams, graphs, the example
# ---------------------------------------------------------------------------------------------------------------------
def test_binding_refusals(mmv):
    q, kc, vc, table, lens = paged_case(1, [5, 7], 4, 2, 64, 16, torch.float16)
    for error, change in [(TypeError, dict(lens=lens.long())), (ValueError, dict(lens=lens[:1])), (TypeError, dict(table=table.long())), (TypeError, dict(q=q.bfloat16())),
                          (ValueError, dict(q=q[:, :3])), (ValueError, dict(q=q[..., :32])), (ValueError, dict(q=q.cpu())), (TypeError, dict(q=3)),
                          (ValueError, dict(q=q.transpose(1, 2))), (ValueError, dict(v_cache=vc[:, :8])), (ValueError, dict(out=torch.empty(2, 4, 32, dtype=q.dtype, device="cuda"))),
                          (TypeError, dict(lse=torch.empty(2, 4, dtype=torch.float64, device="cuda"))), (TypeError, dict(scale="x")), (mmv.MmvError, dict(window=-1)),
                          (mmv.MmvError, dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda")))]:
        args = dict(q=q, k_cache=kc, v_cache=vc, table=table, lens=lens)
        args.update(change)
        with pytest.raises(error):
            mmv.paged_attention(**args)
    x = torch.zeros(3, 2, 64, dtype=torch.float16, device="cuda")
    s, g = torch.zeros(3, 2, 64, 64, device="cuda"), torch.zeros(2, device="cuda")
    with pytest.raises(mmv.MmvError):
        mmv.linear_attention(x, x, x, ints([0, 3]), g)                   # the prompt form takes bfloat16
    with pytest.raises(ValueError):
        mmv.linear_attention_step(x, x, x, g, s[:, :1].contiguous())
    with pytest.raises(ValueError):
        mmv.linear_attention_step(x, x[:, :, :32], x, g, s)
    with pytest.raises(mmv.MmvError):
        mmv.linear_attention_step(x, x, x, g, s[:2])                     # fewer states than requests
    with pytest.raises(TypeError):
        mmv.kv_append(x, x, torch.zeros(3, dtype=torch.int32, device="cuda"), kc, vc)
    with pytest.raises(mmv.MmvError):
        mmv.block_tables(ints([1]), ints([1]), ints([0]), torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), 0)


def test_tensors_that_require_a_gradient(mmv):
    """Refused in grad mode, each of them; the same call under no_grad gives the results of plain tensors."""
    q, kc, vc, table, lens = paged_case(2, [5, 40], 4, 2, 64, 16, torch.bfloat16, garbage=0.0)
    lq, lk, lv, off, g, state = linear_case(3, [3, 70], 4, 2, 64, 64)
    slots = torch.arange(3, device="cuda")
    calls = [(mmv.paged_attention, dict(q=q, k_cache=kc, v_cache=vc, table=table, lens=lens), ("q", "k_cache", "v_cache")),
             (mmv.kv_append, dict(k=lk[:3], v=lv[:3], slots=slots, k_cache=kc.clone(), v_cache=vc.clone()), ("k", "v", "k_cache", "v_cache")),
             (mmv.linear_attention, dict(q=lq, k=lk, v=lv, offsets=ints(off), log_decay=g, state=state), ("q", "k", "v", "log_decay", "state")),
             (mmv.linear_attention_step, dict(q=lq[:2], k=lk[:2], v=lv[:2], log_decay=g, state=state, state_out=torch.empty_like(state)),
              ("q", "k", "v", "log_decay", "state"))]
    first = lambda r: r[0] if isinstance(r, tuple) else r                                                  # noqa: E731
    for call, args, names in calls:
        want = first(call(**args))
        for name in names:
            wanting = dict(args, **{name: args[name].detach().requires_grad_()})
            with pytest.raises(RuntimeError, match="no_grad"):
                call(**wanting)
            with torch.no_grad():
                got = first(call(**wanting))
            assert got is None and want is None or torch.equal(got, want)


def test_calls_on_another_stream_and_in_a_graph(mmv):
    """The same results on a side stream, and from a captured step replayed with new contents."""
    q, kc, vc, table, lens = paged_case(21, [300, 77, 4000], 8, 2, 64, 16, torch.bfloat16, garbage=0.0)
    lq, lk, lv, off, g, st = linear_case(22, [300, 77, 500], 4, 4, 64, 64)
    offsets = ints(off)
    want, _ = mmv.paged_attention(q, kc, vc, table, lens)
    lwant, swant = mmv.linear_attention(lq, lk, lv, offsets, g, state=st)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, _ = mmv.paged_attention(q, kc, vc, table, lens, stream=side)
    lout, sout = mmv.linear_attention(lq, lk, lv, offsets, g, state=st, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want) and torch.equal(lout, lwant) and torch.equal(sout, swant)
    graph = torch.cuda.CUDAGraph()
    q1, lq1 = torch.zeros_like(q), torch.zeros_like(lq)
    with torch.cuda.graph(graph):
        out, _ = mmv.paged_attention(q1, kc, vc, table, lens)
        lout, sout = mmv.linear_attention(lq1, lk, lv, offsets, g, state=st)
    q1.copy_(q)
    lq1.copy_(lq)
    for _ in range(2):
        graph.replay()
    assert torch.equal(out, want) and torch.equal(lout, lwant) and torch.equal(sout, swant)


@pytest.mark.parametrize("order", ["head first", "padded"])
def test_linear_attention_layouts(mmv, order):
    """[head, token, column] in memory, and rows with other data between them."""
    q, k, v, off, g, state = linear_case(31, [100, 3, 129], 4, 2, 64, 96)
    want, last = mmv.linear_attention(q, k, v, ints(off), g, state=state)
    if order == "head first":
        q, k, v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v))
    else:
        q, k, v = (torch.cat([x, torch.full_like(x[..., :8], float("nan"))], -1)[..., :x.size(2)] for x in (q, k, v))
    out, last2 = mmv.linear_attention(q, k, v, ints(off), g, state=state)
    assert torch.equal(out, want) and torch.equal(last, last2)


def test_example_serves_a_ragged_batch(mmv):
    """The example's last logits against the dense fp32 model on the whole sequences: no further off than twice what the dense model itself
    makes of rounding its activations to bfloat16 at the same places (the server's roundings are others, and as many)."""
    import importlib.util
    from pathlib import Path
    spec = importlib.util.spec_from_file_location("serve_ragged_batch", Path(__file__).resolve().parent.parent / "examples" / "serve_ragged_batch.py")
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    off, own = ex.difference(*ex.serve(5, 6, seed=3))
    assert off < 2 * own


@pytest.mark.parametrize("schedule", [[[2, 0]], [[5, 30], [2, 0]], [[3, 1, 2], [1, 0, 2]], None])
def test_example_serves_pieces(mmv, schedule):
    """Steps in which some requests add no token and others several, as many in all as there are requests among them; the bound as above."""
    import importlib.util
    from pathlib import Path
    spec = importlib.util.spec_from_file_location("serve_ragged_batch", Path(__file__).resolve().parent.parent / "examples" / "serve_ragged_batch.py")
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    server, texts, last = ex.serve_in_pieces(schedule or ex.PIECES, seed=5)
    there = [r for r, t in enumerate(texts) if t.numel()]
    off, own = ex.difference(server, [texts[r] for r in there], last[there])
    assert off < 2 * own
