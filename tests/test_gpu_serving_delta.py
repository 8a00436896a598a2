"""The gated delta rule against its recurrence in 64 bits, token by token.

Tolerances.  u = unit roundoff of the result's type (2^-8 bfloat16, 2^-11 fp16), e = 2^-24.  A result is rounded once:
|out - exact| <= u |exact| + (error of the fp32 value) + the type's smallest subnormal.  The fp32 errors are derived at each check.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TYPES = [torch.bfloat16, torch.float16]
INF = float("inf")


@pytest.fixture(scope="module")
def mmv():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2506_23906_b200 as m
    m.debug_configure(0, -1)
    return m


def ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def inside(got, want, bound):
    over = (got.double() - want).abs() - bound
    assert torch.isfinite(got).all() and (over.numel() == 0 or float(over.max()) <= 0.0), f"outside the bound by {float(over.max())}"


def unit(x):
    return x / x.norm(dim=-1, keepdim=True).clamp(min=1e-6)


# ---------------------------------------------------------------------------------------------------------------------
# one token
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,hk,rep,dk,dv", [(1, 1, 1, 8, 8), (2, 2, 2, 64, 64), (3, 3, 2, 40, 72), (1, 16, 1, 128, 128), (64, 4, 4, 128, 128), (130, 5, 1, 128, 96), (7, 3, 1, 16, 128)])
@pytest.mark.parametrize("in_place", [False, True])
def test_step(mmv, dtype, n, hk, rep, dk, dv, in_place):
    """k S and q S: sums of dk products, (dk + 2) e of their magnitudes, the decay's two parts and the products' roundings a few e more:
    |u - exact| <= (dk + 16) e b (|v| + a |k| |S|); the state adds |k| times that and 8 e of its own terms, the result |q k| times it and (dk + 16) e of its own."""
    gen = torch.Generator("cuda").manual_seed(n * 7 + dk)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=gen)                                        # noqa: E731
    h = hk * rep
    q, k, v = rand(n, hk, dk).to(dtype), unit(rand(n, hk, dk + 8)).to(dtype)[..., :dk], rand(n, h, dv).to(dtype)
    g, beta = (-torch.rand(n, h + 3, device="cuda", generator=gen) * 2)[:, :h], torch.rand(n, 2 * h, device="cuda", generator=gen)[:, h:]
    g[0, 0], beta[-1, 0] = 0.0, 0.0
    if h > 2:
        g[0, 1], g[-1, 2], beta[0, 2] = -INF, -200.0, 1.0
    pool = n + 3
    state = rand(pool, h, dk, dv)
    slots = torch.randperm(pool, device="cuda", generator=gen)[:n].to(torch.int32)
    if n > 2:
        slots[1] = -1
        slots[2] = pool
    before = state.clone()
    target = state if in_place else torch.full_like(state, 7.0)
    untouched = target.clone()
    out = mmv.gated_delta_step(q, k, v, g, beta, state, scale=0.3, slots=slots, state_out=target)
    on = [r for r in range(n) if 0 <= slots[r] < pool]
    at = slots[on].long()
    kd, qd = (x.double().repeat_interleave(rep, 1)[on] for x in (k, q))
    vd, bd = v.double()[on], beta.double()[on][..., None]
    old = torch.exp(g.double()[on])[..., None, None] * before[at].double()
    u = bd * (vd - torch.einsum("nhk,nhkv->nhv", kd, old))
    eu = (dk + 16) * E * bd * (vd.abs() + torch.einsum("nhk,nhkv->nhv", kd.abs(), old.abs()))
    new = kd[..., :, None] * u[..., None, :]
    inside(target[at], old + new, 8 * E * (old.abs() + new.abs()) + kd.abs()[..., :, None] * eu[..., None, :] + 1e-37)
    rest = torch.ones(pool, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert torch.equal(target[rest], untouched[rest])
    want = 0.3 * torch.einsum("nhk,nhkv->nhv", qd, old + new)
    qk = (qd.abs() * kd.abs()).sum(-1, keepdim=True)
    size = 0.3 * (torch.einsum("nhk,nhkv->nhv", qd.abs(), old.abs()) + qk * u.abs())
    inside(out[on], want, U[dtype] * want.abs() + (dk + 16) * E * size + 0.3 * qk * eu + TINY[dtype])
    off = [r for r in range(n) if r not in on]
    assert (out[off] == 0).all()


def test_step_own_index_and_nothing(mmv):
    q = torch.randn(4, 2, 16, device="cuda").half()
    state = torch.randn(5, 2, 16, 16, device="cuda")
    g = -torch.rand(4, 2, device="cuda")
    a, s1, s2 = torch.arange(4, dtype=torch.int32, device="cuda"), torch.zeros_like(state), torch.zeros_like(state)
    assert torch.equal(mmv.gated_delta_step(q, q, q, g, -g, state, state_out=s1), mmv.gated_delta_step(q, q, q, g, -g, state, slots=a, state_out=s2))
    assert torch.equal(s1, s2)
    assert mmv.gated_delta_step(q[:0], q[:0], q[:0], g[:0], g[:0], state).shape == (0, 2, 16)


# ---------------------------------------------------------------------------------------------------------------------
# packed prompts
# ---------------------------------------------------------------------------------------------------------------------
def delta_case(seed, lens, hk, rep, dk, dv, state=True, first=0, behind=0, odd=True):
    """Normalised keys; decays from none to forgetting at once, betas from 0 to 1, by token."""
    gen = torch.Generator("cuda").manual_seed(seed)
    off = [first]
    for n in lens:
        off.append(off[-1] + n)
    t, h = off[-1] + behind, hk * rep
    rand = lambda *s: torch.randn(*s, device="cuda", generator=gen)                                        # noqa: E731
    qkv = torch.cat([unit(rand(t, 2 * hk, dk)).flatten(1), rand(t, h * dv)], 1).bfloat16()
    q, k, v = qkv[:, :hk * dk].view(t, hk, dk), qkv[:, hk * dk:2 * hk * dk].view(t, hk, dk), qkv[:, 2 * hk * dk:].view(t, h, dv)
    g = -torch.exp2(-torch.linspace(0, 9, h, device="cuda")) * torch.rand(t, h, device="cuda", generator=gen)
    beta = torch.rand(t, h, device="cuda", generator=gen)
    if odd and t > 2:
        pick = torch.rand(t, h, device="cuda", generator=gen)
        g[pick < 0.02] = -INF
        g[(pick > 0.02) & (pick < 0.04)] = -90.0
        g[(pick > 0.04) & (pick < 0.05)] = -3000.0
        g[(pick > 0.05) & (pick < 0.2)] = 0.0
        beta[(pick > 0.5) & (pick < 0.6)] = 0.0
        beta[(pick > 0.6) & (pick < 0.8)] = 1.0
        g[:, 0] = 0.0
    return q, k, v, off, g, beta, rand(len(lens), h, dk, dv) if state else None


def delta_plain(q, k, v, off, g, beta, scale, state):
    """The recurrence in 64 bits and bounds of what the chunked form may lose.

    An operand that is formed is held as two bfloat16 values, 2^-17 of it, and a product of two such leaves 2^-18 out.  With M = b (|v| + exp(G) |k| |S|)
    the sizes of R's terms, R's and S's copies and the product cost U = T R at most 2.5 x 2^-17 |T| M, T's own parts 2^-17 |T| M and the roundings of L
    and of the blocks' products in T = (1 + L)^-1 at most 4 x 2^-17 |T| |L| |T| M; the copies of U 2^-17 more: 2^-14 (|T| M + |T| |L| |T| M) covers all, fp32
    roundings among it.  The state of the next chunk takes |k|^T (exp(G_n - G) of that), and 2^-21 of its own size for the decay and the sums.  A token's
    step a (1 - b k k^T) makes no column of an error longer (b |k|^2 <= 2), so a column's errors add up in the 2-norm; a result sees them through |q|."""
    t, h = v.shape[:2]
    dk, dv, rep, n = q.size(2), v.size(2), h // q.size(1), len(off) - 1
    q, k, v = (x.double().repeat_interleave(h // x.size(1), 1).transpose(0, 1) for x in (q, k, v))
    g, beta = g.double().t(), beta.double().t()[..., None]
    out, bound = torch.zeros(h, t, dv, dtype=torch.float64, device="cuda"), torch.zeros(h, t, dv, dtype=torch.float64, device="cuda")
    last, room = [torch.zeros(n, h, dk, dv, dtype=torch.float64, device="cuda") for _ in range(2)]
    for s in range(n):
        x = torch.zeros(h, dk, dv, dtype=torch.float64, device="cuda") if state is None else state[s].double()
        err = torch.zeros(h, 1, dv, dtype=torch.float64, device="cuda")
        for lo in range(off[s], off[s + 1], 64):
            hi = min(lo + 64, off[s + 1])
            kc, qc, bc = k[:, lo:hi], q[:, lo:hi], beta[:, lo:hi]
            G = g[:, lo:hi].clamp(min=-200).cumsum(1)
            D = torch.exp((G[:, :, None] - G[:, None, :]).clamp(max=0)).tril()
            low = (bc * (kc @ kc.transpose(1, 2)) * D).tril(-1)
            T = torch.linalg.inv(torch.eye(hi - lo, dtype=torch.float64, device="cuda") + low).abs()
            past = torch.exp(G)[..., None]
            m = T @ (bc * (v[:, lo:hi].abs() + past * (kc.abs() @ x.abs())))
            m = m + T @ (low.abs() @ m)
            bound[:, lo:hi] = scale * (2.0 ** -14 * (past * (qc.abs() @ x.abs()) + ((qc @ kc.transpose(1, 2)) * D).abs() @ m) + qc.norm(dim=-1, keepdim=True) * err)
            grown = kc.abs().transpose(1, 2) @ (torch.exp(G[:, -1:] - G)[..., None] * m)
            err = err + (2.0 ** -14 * grown + 2.0 ** -21 * x.abs()).norm(dim=1, keepdim=True)
            for i in range(lo, hi):
                x = torch.exp(g[:, i])[:, None, None] * x
                u = beta[:, i] * (v[:, i] - torch.einsum("hk,hkv->hv", k[:, i], x))
                x = x + k[:, i, :, None] * u[:, None, :]
                out[:, i] = scale * torch.einsum("hk,hkv->hv", q[:, i], x)
        last[s], room[s] = x, err
    return out.transpose(0, 1), bound.transpose(0, 1), last, room


def check_delta(mmv, case, scale=0.1, **more):
    q, k, v, off, g, beta, state = case
    t, h, dv = v.shape
    n = len(off) - 1
    guard = torch.full((t * h * dv + 64,), 3.0, dtype=q.dtype, device="cuda")
    out = guard[:t * h * dv].view(t, h, dv)
    ws = torch.empty(max(256, mmv.gated_delta_workspace_bytes(q, k, v, g, beta, n)), dtype=torch.uint8, device="cuda")
    _, last = mmv.gated_delta(q, k, v, ints(off), g, beta, scale=scale, state=state, out=out, workspace=ws, **more)
    assert mmv.last_async_status(ws) == 0
    assert (guard[t * h * dv:] == 3.0).all() and (out[:off[0]] == 3.0).all() and (out[off[-1]:] == 3.0).all()
    want, bound, wlast, room = delta_plain(q, k, v, off, g, beta, scale, state)
    rows = slice(off[0], off[-1])
    inside(out[rows], want[rows], U[q.dtype] * want[rows].abs() + bound[rows] + TINY[q.dtype])
    inside(last, wlast, room + 1e-37)
    return out, last


@pytest.mark.parametrize("hk,rep,dk,dv", [(1, 1, 8, 8), (4, 1, 64, 64), (2, 3, 128, 128), (5, 1, 40, 72), (3, 1, 128, 64), (2, 2, 96, 128), (1, 2, 16, 120)])
@pytest.mark.parametrize("lens", [[1], [0, 1, 2, 0], [63, 64, 65], [127, 0, 128, 129, 1], [300, 5, 700]])
@pytest.mark.parametrize("state", [False, True])
def test_delta(mmv, hk, rep, dk, dv, lens, state):
    check_delta(mmv, delta_case(dk + dv + len(lens), lens, hk, rep, dk, dv, state))


@pytest.mark.parametrize("lens,hk,rep,dk,dv", [([5000], 1, 1, 128, 128), ([3000, 1, 2500], 1, 2, 64, 64), ([1] * 150 + [900], 3, 1, 128, 80), ([1000, 64, 128, 3000], 2, 2, 128, 128)])
def test_delta_long(mmv, lens, hk, rep, dk, dv):
    check_delta(mmv, delta_case(sum(lens), lens, hk, rep, dk, dv, odd=False))


@pytest.mark.parametrize("hk,rep,lens", [(256, 4, [1200, 5, 900, 0, 700]), (128, 4, [130, 64, 1, 5000])])
def test_delta_in_parts(mmv, hk, rep, lens):
    """More chunks times heads than one pair of launches takes: sequences go on in the next, the state through state_out."""
    check_delta(mmv, delta_case(1, lens, hk, rep, 16, 8))


@pytest.mark.parametrize("hk,rep,count,most,first,behind", [(64, 1, 300, 200, 0, 0), (128, 4, 100, 100, 37, 3000), (256, 4, 9, 150, 0, 2000), (256, 2, 200, 3, 5, 64)])
def test_delta_many_sequences_in_parts(mmv, hk, rep, count, most, first, behind):
    """A part's launches have CTAs for the sequences that may lie in it alone; empty sequences, parts without one, rows around them.  The bits are those of
    the sequences a few at a time."""
    lens = torch.randint(0, most + 1, (count,), generator=torch.Generator().manual_seed(count)).tolist()
    q, k, v, off, g, beta, state = delta_case(count, lens, hk, rep, 16, 8, first=first, behind=behind)
    out = torch.full((v.shape[0], hk * rep, 8), 7.0, dtype=q.dtype, device="cuda")
    last = mmv.gated_delta(q, k, v, ints(off), g, beta, state=state, out=out)[1]
    assert (out[:off[0]] == 7).all() and (out[off[-1]:] == 7).all()
    group = 40 if hk * rep < 512 else 4 if hk * rep < 1024 else 1
    for i in range(0, count, group):
        j = min(count, i + group)
        a, b = off[i], off[j]
        o, s = mmv.gated_delta(q[a:b], k[a:b], v[a:b], ints([x - a for x in off[i:j + 1]]), g[a:b], beta[a:b], state=state[i:j])
        assert torch.equal(o, out[a:b]) and torch.equal(s, last[i:j])


def test_delta_in_parts_back_to_back(mmv):
    """Parts whose first kernels run beside the second ones in front of them, call after call in one workspace: always the same bits."""
    q, k, v, off, g, beta, state = delta_case(2, [9000], 36, 1, 64, 64, odd=False)
    q2, k2, v2, off2, g2, beta2, state2 = delta_case(3, [150] * 20, 256, 4, 16, 24)
    need = max(mmv.gated_delta_workspace_bytes(q, k, v, g, beta, 1), mmv.gated_delta_workspace_bytes(q2, k2, v2, g2, beta2, 20))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    want = mmv.gated_delta(q, k, v, ints(off), g, beta, state=state), mmv.gated_delta(q2, k2, v2, ints(off2), g2, beta2, state=state2)
    torch.cuda.synchronize()
    for _ in range(3):
        got = (mmv.gated_delta(q, k, v, ints(off), g, beta, state=state, workspace=ws), mmv.gated_delta(q2, k2, v2, ints(off2), g2, beta2, state=state2, workspace=ws))
        for a, b in zip(got, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    exact, bound, last, room = delta_plain(q, k, v, off, g, beta, 1.0, state)
    inside(want[0][0], exact, U[q.dtype] * exact.abs() + bound)


def test_delta_rows_outside_the_sequences(mmv):
    check_delta(mmv, delta_case(1, [70, 64, 3], 3, 1, 64, 64, first=37, behind=50))


def test_delta_equal_keys(mmv):
    """One key for all tokens, betas of 1 and 2, no decay: T's entries do not fall off with the distance."""
    q, k, v, off, g, beta, state = delta_case(3, [200, 64], 2, 1, 64, 64, odd=False)
    k[:] = k[:1]
    g[:] = 0.0
    for b in (1.0, 1.9):
        beta[:] = b
        check_delta(mmv, (q, k, v, off, g, beta, state))


@pytest.mark.parametrize("order", ["head first", "padded"])
def test_delta_layouts(mmv, order):
    q, k, v, off, g, beta, state = delta_case(31, [100, 3, 129], 2, 2, 64, 96)
    want, last = mmv.gated_delta(q, k, v, ints(off), g, beta, state=state)
    if order == "head first":
        q, k, v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v))
    else:
        q, k, v = (torch.cat([x, torch.full_like(x[..., :8], float("nan"))], -1)[..., :x.size(2)] for x in (q, k, v))
        g, beta = (torch.cat([x, torch.full_like(x, float("nan"))], -1)[:, :x.size(1)] for x in (g, beta))
    out, last2 = mmv.gated_delta(q, k, v, ints(off), g, beta, state=state)
    assert torch.equal(out, want) and torch.equal(last, last2)


def test_delta_state_in_place(mmv):
    q, k, v, off, g, beta, state = delta_case(5, [70, 0, 300], 2, 1, 64, 64)
    want, last = mmv.gated_delta(q, k, v, ints(off), g, beta, state=state)
    out, same = mmv.gated_delta(q, k, v, ints(off), g, beta, state=state, state_out=state)
    assert same.data_ptr() == state.data_ptr() and torch.equal(out, want) and torch.equal(state, last)
    both = torch.zeros(4, *state.shape[1:], device="cuda")
    for to in (both[1:], ):
        with pytest.raises(mmv.MmvError):
            mmv.gated_delta(q, k, v, ints(off), g, beta, state=both[:3], state_out=to)


def test_delta_neighbours_that_are_not_finite(mmv):
    """Sequences share chunks of memory, not values."""
    q, k, v, off, g, beta, state = delta_case(2, [40, 70, 200], 2, 2, 64, 64)
    want, last = mmv.gated_delta(q, k, v, ints(off), g, beta, state=state)
    bad = [x.clone() for x in (q, k, v, g, beta)]
    for x in bad:
        x[40:110] = float("nan")
    out, last2 = mmv.gated_delta(*bad[:3], ints(off), *bad[3:], state=state)
    assert torch.equal(out[:40], want[:40]) and torch.equal(out[110:], want[110:]) and torch.equal(last2[[0, 2]], last[[0, 2]])
    assert torch.isnan(out[40:110]).all() and torch.isnan(last2[1]).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("value", [float("nan"), INF, -INF])
def test_delta_later_tokens_do_not_reach_earlier_ones(mmv, dim, value):
    """A value that is not finite reaches no result in front of its token and no other column (of v), head or sequence.  Where its chunk is taken token by
    token the others stay inside the bound; what has no part in such a chunk stays the same bit by bit."""
    q, k, v, off, g, beta, state = delta_case(12, [300, 90], 2, 2, dim, dim, odd=False)
    want, last = mmv.gated_delta(q, k, v, ints(off), g, beta, scale=0.1, state=state)
    exact, bound, elast, room = delta_plain(q, k, v, off, g, beta, 0.1, state)
    for at in (0, 37, 63, 64, 150, 299):
        for name in ("v", "k", "q", "g", "beta"):
            if name == "g" and value == -INF:                        # (a decay of zero: finite)
                continue
            x = {n: t.clone() for n, t in zip(("q", "k", "v", "g", "beta"), (q, k, v, g, beta))}
            hit = torch.zeros_like(want, dtype=torch.bool)
            lost = torch.zeros_like(last, dtype=torch.bool)
            if name == "v":
                x["v"][at, 2, 11] = value
                hit[at:300, 2, 11] = True
                lost[0, 2, :, 11] = True
                heads = [2]
            elif name == "q":
                x["q"][at, 1, 6] = value
                hit[at, 2:] = True
                heads = [2, 3]
            elif name == "k":
                x["k"][at, 0, 5] = value
                hit[at:300, :2] = True
                lost[0, :2] = True
                heads = [0, 1]
            else:
                x[name][at, 1] = value
                hit[at:300, 1] = True
                lost[0, 1] = True
                heads = [1]
            out, s = mmv.gated_delta(x["q"], x["k"], x["v"], ints(off), x["g"], x["beta"], scale=0.1, state=state)
            other = [h for h in range(4) if h not in heads]
            assert torch.equal(out[:, other], want[:, other]) and torch.equal(s[:, other], last[:, other])
            assert torch.equal(out[:at // 64 * 64], want[:at // 64 * 64]) and torch.equal(out[300:], want[300:]) and torch.equal(s[1], last[1])
            if name == "v":                                          # (k times an infinity: a row that k has a zero in is NaN, others infinite)
                assert not torch.isfinite(out[hit]).any() and not torch.isfinite(s[lost]).any()
            else:
                assert not torch.isfinite(out[hit]).any() and not torch.isfinite(s[lost]).any()
            inside(out[~hit], exact[~hit], 2 * (U[q.dtype] * exact.abs() + bound)[~hit])
            inside(s[~lost], elast[~lost], 2 * room.expand_as(elast)[~lost])


def test_delta_states_that_are_not_finite(mmv):
    """They stay in their column."""
    q, k, v, off, g, beta, state = delta_case(14, [200, 90], 2, 1, 64, 64, odd=False)
    want, last = mmv.gated_delta(q, k, v, ints(off), g, beta, state=state)
    for value in (float("nan"), INF):
        x = state.clone()
        x[0, 1, 3, 40] = value
        out, s = mmv.gated_delta(q, k, v, ints(off), g, beta, state=x)
        hit = torch.zeros_like(out, dtype=torch.bool)
        hit[:200, 1, 40] = True
        assert torch.equal(out[~hit], want[~hit]) and not torch.isfinite(out[hit]).any()
        lost = torch.zeros_like(s, dtype=torch.bool)
        lost[0, 1, :, 40] = True
        assert torch.equal(s[~lost], last[~lost]) and not torch.isfinite(s[lost]).any()


def test_step_continues_a_prompt(mmv):
    """The prompt form's state, taken on by single tokens, is the longer prompt's."""
    q, k, v, off, g, beta, state = delta_case(4, [65, 66], 2, 2, 64, 128, odd=False)
    want, bound, wlast, room = delta_plain(q, k, v, off, g, beta, 0.2, state)
    pick = torch.cat([torch.arange(0, 64), torch.arange(65, 129)])
    out, s = mmv.gated_delta(q[pick].contiguous(), k[pick].contiguous(), v[pick].contiguous(), ints([0, 64, 128]), g[pick], beta[pick], scale=0.2, state=state)
    at = torch.tensor([64, 129], device="cuda")
    o = mmv.gated_delta_step(q[at], k[at], v[at], g[at], beta[at], s, scale=0.2)
    inside(o, want[at], U[torch.bfloat16] * want[at].abs() + 2 * bound[at])
    at = at[1:] + 1
    o = mmv.gated_delta_step(q[at], k[at], v[at], g[at], beta[at], s, scale=0.2, slots=ints([1]))
    inside(o, want[at], U[torch.bfloat16] * want[at].abs() + 2 * bound[at])
    inside(s, wlast, 2 * room)


def test_delta_bad_offsets_are_reported(mmv):
    q, k, v, off, g, beta, state = delta_case(7, [64, 64, 64], 2, 1, 64, 64)
    ws = torch.zeros(max(256, mmv.gated_delta_workspace_bytes(q, k, v, g, beta, 3)), dtype=torch.uint8, device="cuda")
    for bad in ([0, 100, 64, 192], [-3, 64, 128, 192], [0, 64, 128, 193], [0, 2 ** 31 - 1, 128, 192]):
        mmv.gated_delta(q, k, v, ints(bad), g, beta, state=state, workspace=ws)
        assert mmv.last_async_status(ws) == 4
    mmv.gated_delta(q, k, v, ints(off), g, beta, state=state, workspace=ws)
    assert mmv.last_async_status(ws) == 0


def test_delta_nothing(mmv):
    q, k, v, off, g, beta, state = delta_case(8, [4], 2, 1, 64, 64)
    e = (q[:0], k[:0], v[:0]), (g[:0], beta[:0])
    out, last = mmv.gated_delta(*e[0], ints([0, 0]), *e[1], state=state)
    assert out.shape == (0, 2, 64) and torch.equal(last, state)
    out, last = mmv.gated_delta(*e[0], ints([0, 0, 0]), *e[1])
    assert (last == 0).all()
    out, last = mmv.gated_delta(*e[0], ints([0]), *e[1])
    assert last.shape == (0, 2, 64, 64)


def test_binding_refusals(mmv):
    q, k, v, off, g, beta, state = delta_case(9, [3, 5], 2, 2, 64, 64)
    args = dict(q=q, k=k, v=v, offsets=ints(off), log_decay=g, beta=beta, state=state)
    mmv.gated_delta(**args)
    half = dict(q=q.half(), k=k.half(), v=v.half())
    for error, change in [(mmv.MmvError, half), (TypeError, dict(q=q.half())), (ValueError, dict(k=k[:, :1])), (ValueError, dict(v=v[:, :3])), (ValueError, dict(v=v[:4])),
                          (TypeError, dict(beta=beta.double())), (ValueError, dict(beta=beta[:, :2])), (ValueError, dict(log_decay=g[0])), (ValueError, dict(log_decay=g.t().contiguous().t())),
                          (TypeError, dict(offsets=ints(off).long())), (ValueError, dict(state=state[:1])), (TypeError, dict(state=state.double())), (ValueError, dict(q=q.cpu())),
                          (TypeError, dict(scale="x")), (mmv.MmvError, dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))),
                          (ValueError, dict(out=torch.empty(8, 4, 32, dtype=q.dtype, device="cuda")))]:
        with pytest.raises(error):
            mmv.gated_delta(**dict(args, **change))
    step = dict(q=q[:2], k=k[:2], v=v[:2], log_decay=g[:2], beta=beta[:2], state=state, state_out=torch.empty_like(state))
    mmv.gated_delta_step(**step)
    with pytest.raises(mmv.MmvError):
        mmv.gated_delta_step(**dict(step, state=state[:1], state_out=None))                            # fewer states than requests
    with pytest.raises(ValueError):
        mmv.gated_delta_step(**dict(step, state=state[:, :1].contiguous(), state_out=None))
    for call, kw, names in ((mmv.gated_delta, args, ("q", "k", "v", "log_decay", "beta", "state")), (mmv.gated_delta_step, step, ("q", "k", "v", "log_decay", "beta", "state"))):
        for name in names:
            wanting = dict(kw, **{name: kw[name].detach().clone().requires_grad_()})
            with pytest.raises(RuntimeError, match="no_grad"):
                call(**wanting)
            with torch.no_grad():
                call(**wanting)


def test_calls_on_another_stream_and_in_a_graph(mmv):
    q, k, v, off, g, beta, state = delta_case(22, [300, 77, 500], 2, 2, 64, 64)
    offsets = ints(off)
    want, swant = mmv.gated_delta(q, k, v, offsets, g, beta, state=state)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, s = mmv.gated_delta(q, k, v, offsets, g, beta, state=state, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want) and torch.equal(s, swant)
    graph, q1 = torch.cuda.CUDAGraph(), torch.zeros_like(q)
    with torch.cuda.graph(graph):
        out, s = mmv.gated_delta(q1, k, v, offsets, g, beta, state=state)
        o2 = mmv.gated_delta_step(q1[:3], k[:3], v[:3], g[:3], beta[:3], s)
    q1.copy_(q)
    for _ in range(2):
        graph.replay()
    assert torch.equal(out, want)
    assert torch.equal(mmv.gated_delta_step(q[:3], k[:3], v[:3], g[:3], beta[:3], swant), o2) and torch.equal(s, swant)


def test_parts_in_a_graph_and_two_calls_at_once(mmv):
    """A batch that is taken in parts, captured and replayed over other inputs; calls on two streams, each with a workspace of its own."""
    lens = [300, 0, 1500, 64, 700]
    q, k, v, off, g, beta, state = delta_case(31, lens, 256, 4, 16, 16)
    q2, k2, v2, off2, g2, beta2, state2 = delta_case(32, lens, 256, 4, 16, 16)
    offsets = ints(off)
    wants = [mmv.gated_delta(q, k, v, offsets, g, beta, state=state), mmv.gated_delta(q2, k2, v2, offsets, g2, beta2, state=state2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [mmv.gated_delta(q, k, v, offsets, g, beta, state=state, stream=streams[0]), mmv.gated_delta(q2, k2, v2, offsets, g2, beta2, state=state2, stream=streams[1])]
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    for (out, last), want in zip(got, wants):
        assert torch.equal(out, want[0]) and torch.equal(last, want[1])
    held = [x.clone() for x in (q, k, v, g, beta, state)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, last = mmv.gated_delta(held[0], held[1], held[2], offsets, held[3], held[4], state=held[5])
    for inputs, want in (((q2, k2, v2, g2, beta2, state2), wants[1]), ((q, k, v, g, beta, state), wants[0])):
        for x, y in zip(held, inputs):
            x.copy_(y)
        graph.replay()
        graph.replay()
        assert torch.equal(out, want[0]) and torch.equal(last, want[1])
