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
