"""The operators on a key-value cache in 8 bits against plain implementations in 64 bits.

Codes and scales are compared exactly: both are defined by one rounding each, which the plain implementation makes in 64 bits (a quotient of numbers
of 11 bits is 2^-19 of itself away from every half that it is not, far more than 64 bits lose).  Attention's tolerance is derived at its check;
u = unit roundoff of the result's type (2^-8 bfloat16, 2^-11 fp16), e = 2^-24.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TYPES = [torch.bfloat16, torch.float16]
CODES = [torch.int8, torch.float8_e4m3fn]
TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


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
    got, want, bound = got.double(), want.double(), bound.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    over = ((got - want).abs() - bound)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0.0, f"outside the bound by {float(over.max())}"


# ---------------------------------------------------------------------------------------------------------------------
# the plain cache: numbers that codes are, in 64 bits on the host
# ---------------------------------------------------------------------------------------------------------------------
def scale_of(amax, top):
    if amax < 2.0 ** -100:
        return 0.0
    m, e = np.frexp(amax / top)
    return float(np.ldexp(np.ceil(m * 2048) / 2048 if top == 127.0 else (1.0 if m > 0.5 else 0.5), e))


def codes_of(x, scale, top):
    if not scale > 0:
        return np.zeros_like(x)
    y = x / scale
    if top == 127.0:
        return np.sign(y) * np.floor(np.abs(y) + 0.5)
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
    return np.rint(y / step) * step


def append_plain(codes, scale, x, off, total, table, block, top):
    """codes [blocks, block, heads, dim] (numbers), scale [blocks, heads], x [tokens, heads, dim]; numpy, 64 bits; in place."""
    for r, end in enumerate(total):
        p, t = end - (off[r + 1] - off[r]), off[r]
        while p < end:
            b, place = p // block, p % block
            n = min(block - place, end - p)
            page = table[r][b] if b < len(table[r]) else -1
            if 0 <= page < codes.shape[0]:
                for h in range(scale.shape[1]):
                    new, old = x[t:t + n, h], scale[page, h] if place else 0.0
                    amax = np.abs(new).max()
                    if not np.isfinite(new).all() or not (0 <= old < np.inf):
                        scale[page, h] = np.nan
                        codes[page, place:place + n, h] = 0
                        continue
                    now = old if amax <= old * top else scale_of(amax, top)
                    if place and now > old:
                        codes[page, :place, h] = codes_of(codes[page, :place, h] * old, now, top)
                    scale[page, h] = now
                    codes[page, place:place + n, h] = codes_of(new, now, top)
            p, t = p + n, t + n


def numbers(cache):
    return cache.float().double().cpu().numpy()


def empty_cache(blocks, block, heads, dim, code, order="bthd", pad=0, scale_order="bh"):
    """Two caches of random codes in the given order of their axes, `pad` unused columns behind each head's row, and their scales."""
    size = {"b": blocks, "t": block, "h": heads}
    shape = [size[c] for c in order[:3]] + [dim + pad]
    perm = [order.index(c) for c in "bth"] + [3]
    caches, scales = [], []
    for _ in range(2):
        x = torch.randint(-127, 128, shape, device="cuda")
        x = x.to(torch.int8) if code == torch.int8 else (x.float() * 3).to(code)
        caches.append(x.permute(perm)[..., :dim])
        s = torch.tensor([scale_of(v, TOP[code]) for v in np.exp2(np.random.default_rng(blocks + dim).uniform(-3, 3, blocks * heads))], dtype=torch.float32, device="cuda")
        s = s.view(blocks, heads)
        scales.append(s if scale_order == "bh" else s.t().contiguous().t())
    return caches, scales


def batch(rng, counts, pasts, block, spare=3):
    """offsets, total, table (numpy) of requests that add counts[r] to pasts[r], pages in random order."""
    off = np.concatenate([[0], np.cumsum(counts)]).astype(int).tolist()
    total = [a + b for a, b in zip(pasts, counts)]
    pages = [-(-t // block) for t in total]
    ids = rng.permutation(sum(pages) + spare)
    width = max(pages + [1]) + 1
    table, at = np.full((len(counts), width), -5, dtype=np.int32), 0
    for r, n in enumerate(pages):
        table[r, :n] = ids[at:at + n]
        at += n
    return off, total, table, sum(pages) + spare


def check_append(mmv, dtype, code, counts, pasts, heads, dim, block, order="bthd", pad=0, behind=0, scale_order="bh", seed=0, grow=1.0):
    rng = np.random.default_rng(seed + dim)
    off, total, table, blocks = batch(rng, counts, pasts, block)
    caches, scales = empty_cache(blocks, block, heads, dim, code, order, pad, scale_order)
    n = off[-1] + behind
    gen = torch.Generator("cuda").manual_seed(seed)
    qkv = torch.randn(n, 2 * heads + 1, dim, device="cuda", generator=gen) * torch.exp2(grow * torch.randn(n, 2 * heads + 1, 1, device="cuda", generator=gen))
    qkv[::5, 0] = 0.0
    if n > 3:
        qkv[2] *= 2.0 ** -60
    qkv = qkv.to(dtype)
    new = [qkv[:, :heads], qkv[:, heads:2 * heads]]
    want = [(numbers(c), s.double().cpu().numpy()) for c, s in zip(caches, scales)]
    mmv.kv_append_q8(*new, ints(off), ints(total), torch.from_numpy(table).cuda(), *caches, *scales)
    for (codes, scale), x, c, s in zip(want, new, caches, scales):
        append_plain(codes, scale, x.double().cpu().numpy(), off, total, table.tolist(), block, TOP[code])
        assert np.array_equal(s.double().cpu().numpy(), scale, equal_nan=True)
        assert np.array_equal(numbers(c), codes)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("heads,dim,block,order,pad,scale_order", [
    (1, 16, 1, "bthd", 0, "bh"), (2, 64, 16, "bthd", 0, "bh"), (5, 80, 7, "bhtd", 16, "hb"), (3, 256, 32, "hbtd", 0, "hb"), (4, 128, 130, "bthd", 32, "bh")])
@pytest.mark.parametrize("counts,pasts", [
    ([1], [0]), ([1, 1, 1, 1], [0, 15, 16, 33]), ([3, 0, 70, 1], [2, 5, 0, 31]), ([0, 0], [4, 0]), ([200, 1, 129], [0, 127, 61])])
def test_append(mmv, dtype, code, heads, dim, block, order, pad, scale_order, counts, pasts):
    check_append(mmv, dtype, code, counts, pasts, heads, dim, block, order, pad, behind=len(counts) % 3, scale_order=scale_order)


@pytest.mark.parametrize("code", CODES)
def test_append_many_requests(mmv, code):
    """More requests than one trip of the search takes, empty ones among them; and long prompts of whole blocks."""
    rng = np.random.default_rng(1)
    counts = rng.integers(0, 4, 1500).tolist()
    check_append(mmv, torch.bfloat16, code, counts, rng.integers(0, 40, 1500).tolist(), 2, 32, 16, seed=4)
    check_append(mmv, torch.float16, code, [0] * 40 + [700, 0, 513] + [0] * 30, [0] * 40 + [5, 9, 0] + [0] * 30, 2, 128, 64, seed=5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("code", CODES)
def test_append_token_by_token(mmv, dtype, code):
    """A request that grows by a token 50 times: the scale grows now and then, and the codes are converted as often."""
    heads, dim, block, steps = 3, 48, 16, 50
    caches, scales = empty_cache(6, block, heads, dim, code)
    want = [(numbers(c), s.double().cpu().numpy()) for c, s in zip(caches, scales)]
    table = np.array([[4, 1, 0, 5]], dtype=np.int32)
    gen = torch.Generator("cuda").manual_seed(9)
    for i in range(steps):
        kv = (torch.randn(2, 1, heads, dim, device="cuda", generator=gen) * 2.0 ** float(i % 16 / 5)).to(dtype)
        mmv.kv_append_q8(kv[0], kv[1], ints([0, 1]), ints([i + 1]), torch.from_numpy(table).cuda(), *caches, *scales)
        for (codes, scale), x in zip(want, kv):
            append_plain(codes, scale, x.double().cpu().numpy(), [0, 1], [i + 1], table.tolist(), block, TOP[code])
    for (codes, scale), c, s in zip(want, caches, scales):
        assert np.array_equal(s.double().cpu().numpy(), scale) and np.array_equal(numbers(c), codes)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("code", CODES)
def test_append_halves(mmv, dtype, code):
    """Quotients that are halves exactly, and their neighbours in the inputs' type."""
    heads, dim, block = 1, 256, 4
    for top in (127.0, 254.0, 31.75, 3.984375, 126.0, 101.5):
        base = torch.arange(dim, device="cuda").double() / 2 * top / 127
        x = torch.stack([base, base * (1 + 2.0 ** -8), -base, -base * (1 - 2.0 ** -9)]).to(dtype)
        x = torch.where(x.abs() <= top, x, 0.0)
        x[:, -1] = top
        caches, scales = empty_cache(2, block, heads, dim, code)
        want = [(numbers(c), s.double().cpu().numpy()) for c, s in zip(caches, scales)]
        new = x.to(dtype).view(4, 1, dim).contiguous()
        mmv.kv_append_q8(new, new, ints([0, 4]), ints([4]), ints([[1]]), *caches, *scales)
        for (codes, scale), c, s in zip(want, caches, scales):
            append_plain(codes, scale, new.double().cpu().numpy(), [0, 4], [4], [[1]], block, TOP[code])
            assert np.array_equal(s.double().cpu().numpy(), scale) and np.array_equal(numbers(c), codes)


@pytest.mark.parametrize("code", CODES)
def test_append_values_that_are_not_finite(mmv, code):
    """They make one scale NaN, until the block is begun anew; very small and very large ones do not."""
    heads, dim, block = 3, 32, 8
    caches, scales = empty_cache(4, block, heads, dim, code)
    table = ints([[2, 0]])
    k, v = (torch.randn(10, heads, dim, device="cuda").bfloat16() for _ in range(2))
    k[3, 1, 7] = float("nan")
    v[9, 2, 0] = -float("inf")
    k[0, 2] = 3e38
    v[0, 0] *= 1e-38
    mmv.kv_append_q8(k, v, ints([0, 10]), ints([10]), table, *caches, *scales)
    bad = [torch.isnan(s) for s in scales]
    assert bad[0].nonzero().tolist() == [[2, 1]] and bad[1].nonzero().tolist() == [[0, 2]]
    rk, rv = mmv.kv_read_q8(*caches, *scales, table, ints([0, 10]), 10)
    assert torch.isnan(rk[:8, 1]).all() and torch.isnan(rv[8:, 2]).all() and int(torch.isnan(rk).sum()) == 8 * dim and int(torch.isnan(rv).sum()) == 2 * dim
    one = torch.ones(1, heads, dim, device="cuda").bfloat16()
    mmv.kv_append_q8(one, one, ints([0, 1]), ints([11]), table, *caches, *scales)
    assert torch.isnan(scales[1][0, 2]) and scales[0][0, 2] > 0                                       # (goes on: stays NaN)
    mmv.kv_append_q8(one, one, ints([0, 1]), ints([9]), table, *caches, *scales)
    assert torch.isfinite(scales[1][0]).all()
    tiny = torch.full((4, heads, dim), 2.0 ** -110, device="cuda").bfloat16()
    mmv.kv_append_q8(tiny, tiny, ints([0, 4]), ints([4]), table, *caches, *scales)
    assert (scales[0][2] == 0).all() and (caches[0][2, :4].float() == 0).all()
    mmv.kv_append_q8(one, one, ints([0, 1]), ints([5]), table, *caches, *scales)                      # zeros go on
    rk, _ = mmv.kv_read_q8(*caches, *scales, table, ints([0, 5]), 5)
    assert (rk[:4] == 0).all() and (rk[4] == 1).all()


def test_append_tokens_without_a_place(mmv):
    """Pages out of range, rows too short, totals and offsets that make no sense: nothing is written for them, and the others are."""
    heads, dim, block = 2, 64, 16
    for code in CODES:
        caches, scales = empty_cache(5, block, heads, dim, code)
        keep = [x.clone() for x in (*caches, *scales)]
        x = torch.randn(40, heads, dim, device="cuda").half()
        for off, total, table in [([0, 40], [40], [[-1, 5, 2 ** 31 - 1]]), ([0, 40], [40 + 48], [[1, 2, 3]]), ([0, 40], [39], [[1, 2, 3]]),
                                  ([0, 41], [41], [[1, 2, 3]]), ([-1, 40], [41], [[1, 2, 3]]), ([40, 0], [40], [[1, 2, 3]]), ([40, 40], [40], [[1, 2, 3]]),
                                  ([0, 40], [-2 ** 31], [[1, 2, 3]])]:
            mmv.kv_append_q8(x, x, ints(off), ints(total), ints(table), *caches, *scales)
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(keep, (*caches, *scales)))
        mmv.kv_append_q8(x, x, ints([0, 20, 40]), ints([20, 20]), ints([[-1, 7], [3, -9]]), *caches, *scales)
        changed = [(a.float() != b.float()).flatten(1).any(1).nonzero().flatten().tolist() for a, b in zip(keep[:2], caches)]
        assert changed == [[3], [3]]
        assert torch.equal(scales[0][[0, 1, 2, 4]], keep[2][[0, 1, 2, 4]]) and not torch.equal(scales[0][3], keep[2][3])


def test_append_and_read_far_blocks(mmv):
    """Blocks whose bytes lie past 2^32."""
    block, heads, dim = 64, 2, 64
    blocks = (1 << 32) // (block * heads * dim) + 3
    caches = [torch.zeros(blocks, block, heads, dim, dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(blocks, heads, device="cuda") for _ in range(2)]
    x = torch.randn(70, heads, dim, device="cuda").half()
    table = ints([[blocks - 1, blocks - 2]])
    mmv.kv_append_q8(x, -x, ints([0, 70]), ints([70]), table, *caches, *scales)
    k, v = mmv.kv_read_q8(*caches, *scales, table, ints([0, 70]), 70, dtype=torch.float16)
    assert torch.equal(k, -v) and float((k - x).abs().max()) <= float(scales[0].max()) * 0.5 + 2.0 ** -11 * 4
    assert int((caches[0][:blocks - 2] != 0).sum(dtype=torch.int64)) == 0


# ---------------------------------------------------------------------------------------------------------------------
# the read
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("heads,dim,block,order,pad,scale_order", [
    (1, 16, 1, "bthd", 0, "bh"), (2, 64, 16, "bthd", 0, "bh"), (5, 80, 7, "bhtd", 16, "hb"), (3, 256, 32, "hbtd", 0, "hb"), (8, 128, 64, "bthd", 0, "bh"),
    (300, 256, 3, "bthd", 0, "bh")])
@pytest.mark.parametrize("lens", [[1], [0, 5, 0, 0, 33, 1], [300, 64, 0]])
def test_read(mmv, dtype, code, heads, dim, block, order, pad, scale_order, lens):
    """One rounding of the fp32 product, exactly; rows around the batch stay as they are."""
    rng = np.random.default_rng(dim)
    off, _, table, blocks = batch(rng, lens, [0] * len(lens), block)
    off = [o + 3 for o in off]
    caches, scales = empty_cache(blocks, block, heads, dim, code, order, pad, scale_order)
    scales = [s * 1.2345 for s in scales]                            # (any fp32 scale)
    tokens = off[-1] + 2
    out = [torch.full((tokens, heads, dim), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    k, v = mmv.kv_read_q8(*caches, *scales, torch.from_numpy(table).cuda(), ints(off), tokens, dtype=dtype, k=out[0], v=out[1])
    assert k is out[0] or k.data_ptr() == out[0].data_ptr()
    for got, c, s in zip((k, v), caches, scales):
        assert (got[:3] == 7.0).all() and (got[off[-1]:] == 7.0).all()
        for r, n in enumerate(lens):
            pages = torch.from_numpy(table[r, :-(-n // block)].astype(np.int64)).cuda()
            want = (c.float()[pages] * s[pages][:, None, :, None]).flatten(0, 1)[:n].to(dtype)
            assert torch.equal(got[off[r]:off[r + 1]], want)


def test_read_many_requests_and_missing_pages(mmv):
    heads, dim, block = 2, 32, 8
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 20, 2500).tolist()
    off, _, table, blocks = batch(rng, lens, [0] * len(lens), block)
    caches, scales = empty_cache(blocks, block, heads, dim, torch.int8)
    table[7, 0], table[100, 0] = -1, blocks
    k, _ = mmv.kv_read_q8(*caches, *scales, torch.from_numpy(table).cuda(), ints(off), off[-1])
    t = np.arange(off[-1])
    r = np.searchsorted(np.array(off[1:]), t, side="right")
    p = t - np.array(off)[r]
    page = torch.from_numpy(table[r, p // block].astype(np.int64)).cuda()
    there = (page >= 0) & (page < blocks)
    page = torch.where(there, page, 0)
    want = torch.where(there[:, None, None], (caches[0][page, torch.from_numpy(p % block).cuda()].float() * scales[0][page][:, :, None]), 0.0).bfloat16()
    assert torch.equal(k, want)
    k2, _ = mmv.kv_read_q8(*caches, *scales, torch.from_numpy(table[:, :1].copy()).cuda(), ints(off), off[-1])      # rows that are too short
    assert torch.equal(k2, torch.where(torch.from_numpy(p < block).cuda()[:, None, None], want, 0.0))
    for bad in ([0, 50, 20, 90], [-5, 10, 20, 90], [0, 2 ** 31 - 1, 3, 90]):                             # no offsets: nothing outside is touched
        mmv.kv_read_q8(*caches, *scales, torch.from_numpy(table[:3].copy()).cuda(), ints(bad), 90)
    torch.cuda.synchronize()


def test_nothing(mmv):
    caches, scales = empty_cache(2, 4, 1, 16, torch.int8)
    e = torch.empty(0, 1, 16, dtype=torch.float16, device="cuda")
    none = torch.empty(0, 3, dtype=torch.int32, device="cuda")
    keep = caches[0].clone()
    mmv.kv_append_q8(e, e, ints([0]), ints([]), none, *caches, *scales)
    mmv.kv_append_q8(e, e, ints([0, 0]), ints([4]), ints([[0]]), *caches, *scales)
    assert torch.equal(keep, caches[0])
    assert mmv.kv_read_q8(*caches, *scales, none, ints([0]), 0)[0].shape == (0, 1, 16)


# ---------------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------------
def paged_case(seed, lens, heads, kv, dim, block, dtype, code, order="bthd", pad=0, spare=3, far=0, spread=3.0):
    """Random codes; scales of a block and head between 2^-spread and 2^spread, NaN in blocks that no request has; the rest of the table out of range."""
    gen = torch.Generator("cuda").manual_seed(seed)
    pages = [-(-n // block) for n in lens]
    blocks = sum(pages) + spare + far
    caches, _ = empty_cache(blocks, block, kv, dim, code, order, pad)
    ids = (far + torch.randperm(sum(pages) + spare, device="cuda", generator=gen)).tolist()
    wide = torch.full((len(lens), max(pages + [1]) + 4), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    scales = [torch.full((kv, blocks), float("nan"), device="cuda").t() for _ in range(2)]
    at = 0
    for r, n in enumerate(lens):
        mine = torch.tensor(ids[at:at + pages[r]], dtype=torch.int64, device="cuda")
        at += pages[r]
        wide[r, :pages[r]] = mine.to(torch.int32)
        for s in scales:
            s[mine] = torch.exp2((torch.rand(pages[r], kv, device="cuda", generator=gen) * 2 - 1) * spread) / 100
    q = torch.randn(len(lens), heads, dim + 16, device="cuda", generator=gen).to(dtype)[..., :dim]
    return q, caches, scales, wide[:, :max(pages + [1]) + 1], torch.tensor(lens, dtype=torch.int32, device="cuda")


def paged_plain(q, caches, scales, table, lens, scale, window):
    n, heads, dim = q.shape
    kv, block = caches[0].size(2), caches[0].size(1)
    group = heads // kv
    out = torch.zeros(n, heads, dim, dtype=torch.float64, device="cuda")
    mag, lse = torch.zeros_like(out), torch.full((n, heads), -float("inf"), dtype=torch.float64, device="cuda")
    big, heavy, lift = torch.zeros_like(lse), torch.zeros_like(lse), torch.zeros_like(lse)
    for r, length in enumerate(lens.tolist()):
        if length <= 0:
            continue
        lo = max(0, length - window) if window else 0
        pages = table[r, :-(-length // block)].long()
        for h in range(kv):
            k, v = ((c[pages, :, h].float().double() * s[pages, h].double()[:, None, None]).reshape(-1, dim)[lo:length] for c, s in zip(caches, scales))
            vs = scales[1][pages, h].double().repeat_interleave(block)[lo:length]
            rows = slice(h * group, (h + 1) * group)
            x = scale * q[r, rows].double() @ k.T
            w = torch.softmax(x, 1)
            out[r, rows], mag[r, rows], lse[r, rows] = w @ v, w @ v.abs(), torch.logsumexp(x, 1)
            big[r, rows] = abs(scale) * (q[r, rows].double().abs() @ k.abs().T).amax(1)
            heavy[r, rows] = (w * vs).amax(1)
            lift[r, rows] = torch.log2(vs[vs > 0]).abs().amax() if (vs > 0).any() else 0.0
    return out, mag, lse, big, heavy, lift


def check_paged(mmv, case, dtype, scale, window=0):
    """Scores: a sum of dim products and their factors in fp32, (dim + 16) e S with S the largest scale sum |q k|, the base-2 exponent's rounding among
    it.  A value's weight: that twice (weight and sum), the logarithm of its scale (2^-22 of max(1, itself), and one rounding of the sum of exponents,
    e (S / ln 2 + itself)), 2^-22 for the pair of fp16 values and 2^-40 of the largest weight for what is too small for it, times a code of 448 at most;
    and the running sums' roundings, one per 16 tokens of a warp and one per partial result."""
    q, caches, scales, table, lens = case
    n, heads, dim = q.shape
    ws = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    guard = torch.full((n * heads * dim + 64,), 3.0, dtype=dtype, device="cuda")
    out, lse = mmv.paged_attention_q8(q, *caches, *scales, table, lens, scale=scale, window=window, out=guard[:n * heads * dim].view(n, heads, dim), workspace=ws)
    assert mmv.last_async_status(ws) == 0 and (guard[n * heads * dim:] == 3.0).all()
    want, mag, wlse, big, heavy, lift = paged_plain(q, caches, scales, table, lens, scale, window)
    chain = (lens.double() / 16 + 700)[:, None]
    score = (dim + 16) * E * big
    weight = 3 * score + 2.0 ** -21 * (2 + lift) + 2 * E * (1.5 * big + lift) + chain * E
    least = lens.double()[:, None] * 2.0 ** -40 * 448 * heavy
    inside(out, want, U[dtype] * want.abs() + mag * weight[..., None] + least[..., None] + TINY[dtype])
    inside(lse, wlse, torch.nan_to_num(2 * score + chain * E + 8 * E * wlse.abs(), posinf=0.0))
    again, _ = mmv.paged_attention_q8(q, *caches, *scales, table, lens, scale=scale, window=window)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("heads,kv,dim,block,order,pad", [
    (1, 1, 16, 16, "bthd", 0), (4, 4, 64, 16, "bthd", 0), (8, 1, 48, 7, "bthd", 16), (32, 8, 128, 16, "bthd", 0), (12, 2, 80, 1, "bhtd", 0),
    (71, 1, 64, 64, "hbtd", 0), (48, 2, 128, 48, "bhtd", 16), (16, 2, 256, 16, "bthd", 0), (20, 2, 256, 16, "bthd", 0), (5, 5, 144, 24, "bthd", 0)])
@pytest.mark.parametrize("lens", [[1], [0, 1, 2, 15, 16, 17, 0], [63, 64, 65, 127, 128, 129], [1000, 3, 0, 517, 2048, 1]])
def test_paged_attention(mmv, dtype, code, heads, kv, dim, block, order, pad, lens):
    check_paged(mmv, paged_case(dim + len(lens), lens, heads, kv, dim, block, dtype, code, order, pad), dtype, dim ** -0.5)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("window", [1, 15, 16, 17, 64, 100, 1000, 10 ** 6])
def test_paged_attention_window(mmv, code, window):
    lens = [1, 16, 17, 100, 101, 640, 999, 0, 1500]
    check_paged(mmv, paged_case(window, lens, 8, 2, 64, 16, torch.float16, code), torch.float16, 0.125, window)
    check_paged(mmv, paged_case(window + 1, lens, 2, 2, 128, 9, torch.bfloat16, code), torch.bfloat16, 0.1, window)


@pytest.mark.parametrize("dtype,code,lens,heads,kv,dim,block", [
    (torch.bfloat16, torch.int8, [70001], 8, 1, 128, 16), (torch.float16, torch.float8_e4m3fn, [50000, 1, 0, 2], 4, 2, 64, 64),
    (torch.bfloat16, torch.float8_e4m3fn, [30011], 1, 1, 256, 16), (torch.float16, torch.int8, [5] * 700 + [20000] + [0] * 50 + [64] * 300, 16, 4, 64, 16),
    (torch.bfloat16, torch.int8, [40000, 100], 32, 2, 128, 32)])
def test_paged_attention_split(mmv, dtype, code, lens, heads, kv, dim, block):
    """Few long requests over many ranges, and many short ones in each."""
    check_paged(mmv, paged_case(sum(lens), lens, heads, kv, dim, block, dtype, code), dtype, 1.5 * dim ** -0.5)


@pytest.mark.parametrize("code", CODES)
def test_paged_attention_queries_of_any_magnitude(mmv, code):
    """Queries of 2^-100 to 2^100 (bfloat16) with scores of a few, scores of hundreds, and q = 0."""
    q, caches, scales, table, lens = paged_case(3, [300, 5000], 8, 2, 64, 16, torch.bfloat16, code)
    for f in (2.0 ** -100, 2.0 ** -30, 1.0, 2.0 ** 40, 2.0 ** 100):
        check_paged(mmv, ((q.float() * f).bfloat16(), caches, scales, table, lens), torch.bfloat16, 0.1 / f)
    check_paged(mmv, (q * 8, caches, scales, table, lens), torch.bfloat16, 2.0)
    check_paged(mmv, (q * 0, caches, scales, table, lens), torch.bfloat16, 2.0)
    check_paged(mmv, (q, caches, scales, table, lens), torch.bfloat16, -0.3)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("spread", [10.0, 40.0])
def test_paged_attention_scales_of_any_magnitude(mmv, code, spread):
    """Values' scales of 2^-spread to 2^spread beside one another, some zero: no scale takes another's accuracy away."""
    q, caches, scales, table, lens = paged_case(13, [300, 5000, 17], 8, 2, 64, 16, torch.bfloat16, code, spread=spread)
    scales[0][:] = torch.where(torch.isnan(scales[0]), float("nan"), 0.01)
    scales[1][::7] *= 0
    check_paged(mmv, (q, caches, scales, table, lens), torch.bfloat16, 0.1)
    scales[1][:] *= 0
    out, lse = mmv.paged_attention_q8(q, *caches, *[torch.nan_to_num(s) for s in scales], table, lens)
    assert (out == 0).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("heads,kv", [(8, 2), (32, 2)])
@pytest.mark.parametrize("gap", [10.0, 16.0, 20.0])
def test_paged_attention_dominant_tokens_without_a_value(mmv, code, heads, kv, gap):
    """Tokens that take almost all of the weight and whose codes are zero: the result is made of weights of e^-gap."""
    q, caches, scales, table, lens = paged_case(int(gap), [6000] * 24 + [700, 65], heads, kv, 64, 16, torch.bfloat16, code)
    q[:] = 0.0
    q[..., 0] = 1.0
    one = lambda x: torch.tensor(x, device="cuda").to(code)                                                  # noqa: E731
    caches[0][..., 0] = one(0)
    caches[1].copy_(caches[1].float().abs().to(code))
    scales[0][:] = gap / 100
    for r, n in enumerate(lens.tolist()):
        j = torch.arange(n, device="cuda")
        j = j[(j % 256 < 64) & (j % 16 == 0)]
        page = table[r, j // 16].long()
        view = caches[0].view(torch.uint8)
        view[page, j % 16, :, 0] = one(100 if code == torch.int8 else 96).view(torch.uint8)
        caches[1].view(torch.uint8)[page, j % 16] = 0
    check_paged(mmv, (q, caches, scales, table, lens), torch.bfloat16, 1.0)


def test_paged_attention_not_finite_inside(mmv):
    """A NaN scale or query stays in its request and head group."""
    for code in CODES:
        q, caches, scales, table, lens = paged_case(5, [300, 200, 9000], 4, 2, 64, 16, torch.float16, code)
        scales[1][table[1, 3], 1] = float("nan")
        scales[0][table[2, 100], 0] = float("nan")
        q[0, 3, 5] = float("inf")
        out, lse = mmv.paged_attention_q8(q, *caches, *scales, table, lens)
        bad = torch.isnan(out)
        assert bad[1, 2:].all() and bad[2, :2].all() and not torch.isfinite(out[0, 3]).any() and int(bad.sum()) == 5 * 64
        assert torch.isfinite(out[0, :3]).all() and torch.isfinite(lse[1]).all() and torch.isnan(lse[2, :2]).all()


def test_paged_attention_far_pages(mmv):
    far = (1 << 32) // (16 * 2 * 128) + 10
    check_paged(mmv, paged_case(9, [100, 33], 8, 2, 128, 16, torch.float16, torch.int8, far=far), torch.float16, 0.1)


def test_paged_attention_bad_metadata_is_reported(mmv):
    q, caches, scales, table, lens = paged_case(11, [100, 50, 70], 4, 2, 64, 16, torch.float16, torch.int8)
    ws = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    good, _ = mmv.paged_attention_q8(q, *caches, *scales, table, lens)
    for change in ("page", "negative page", "length", "negative length"):
        t, n = table.clone(), lens.clone()
        if change == "page":
            t[1, 2] = caches[0].size(0)
        elif change == "negative page":
            t[1, 0] = -1
        else:
            n[1] = 10 ** 6 if change == "length" else -5
        out, _ = mmv.paged_attention_q8(q, *caches, *scales, t, n, workspace=ws)
        assert mmv.last_async_status(ws) == 1
        assert torch.equal(out[[0, 2]], good[[0, 2]])
    mmv.paged_attention_q8(q, *caches, *scales, table, lens, workspace=ws)
    assert mmv.last_async_status(ws) == 0


def test_paged_attention_without_requests(mmv):
    q, caches, scales, table, lens = paged_case(12, [4], 2, 1, 64, 16, torch.float16, torch.int8)
    ws = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    out, lse = mmv.paged_attention_q8(q[:0], *caches, *scales, table[:0], lens[:0], workspace=ws)
    assert out.shape == (0, 2, 64) and mmv.last_async_status(ws) == 0
    out, lse = mmv.paged_attention_q8(q, *caches, *scales, table[:, :0], lens * 0, workspace=ws)      # a table without columns
    assert (out == 0).all() and (lse == -float("inf")).all() and mmv.last_async_status(ws) == 0


def test_written_then_attended(mmv):
    """block_tables, the quantising write and attention together: a decoding loop against the plain cache."""
    heads, kv, dim, block, n = 8, 2, 64, 16, 5
    for code in CODES:
        caches, scales = empty_cache(40, block, kv, dim, code)
        want = [(numbers(c), s.double().cpu().numpy()) for c, s in zip(caches, scales)]
        free = torch.randperm(40, device="cuda").to(torch.int32)
        table, past = torch.zeros(n, 8, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
        gen = torch.Generator("cuda").manual_seed(1)
        for counts in ([40, 3, 0, 17, 60], [1] * n, [1] * n, [0, 30, 1, 0, 2], [1] * n):
            t = sum(counts)
            slots = torch.empty(t, dtype=torch.int64, device="cuda")
            offsets, past, used = mmv.block_tables(past, ints(counts), free, table, slots, block)
            free = free[int(used):]
            qkv = torch.randn(t, heads + 2 * kv, dim, device="cuda", generator=gen).bfloat16()
            new = qkv[:, heads:heads + kv], qkv[:, heads + kv:]
            mmv.kv_append_q8(*new, offsets, past, table, *caches, *scales)
            for (codes, scale), x in zip(want, new):
                append_plain(codes, scale, x.double().cpu().numpy(), offsets.tolist(), past.tolist(), table.tolist(), block, TOP[code])
            last = (offsets[1:] - 1).clamp(min=0).long()
            check_paged(mmv, (qkv[last, :heads], caches, scales, table, past), torch.bfloat16, dim ** -0.5)
        for (codes, scale), c, s in zip(want, caches, scales):
            assert np.array_equal(s.double().cpu().numpy(), scale, equal_nan=True) and np.array_equal(numbers(c), codes)


# ---------------------------------------------------------------------------------------------------------------------
# the binding's checks, streams, graphs
# ---------------------------------------------------------------------------------------------------------------------
def test_binding_refusals(mmv):
    q, caches, scales, table, lens = paged_case(1, [5, 7], 4, 2, 64, 16, torch.float16, torch.int8)
    x = torch.zeros(3, 2, 64, dtype=torch.float16, device="cuda")
    calls = [(mmv.paged_attention_q8, dict(q=q, k_cache=caches[0], v_cache=caches[1], k_scale=scales[0], v_scale=scales[1], table=table, lens=lens),
              [(TypeError, dict(lens=lens.long())), (ValueError, dict(lens=lens[:1])), (TypeError, dict(table=table.long())), (TypeError, dict(q=q.float())),
               (ValueError, dict(q=q[:, :3])), (ValueError, dict(q=q[..., :32])), (ValueError, dict(q=q.cpu())), (TypeError, dict(k_cache=caches[0].half(), v_cache=caches[1].half())),
               (ValueError, dict(v_cache=caches[1][:, :8])), (TypeError, dict(k_scale=scales[0].double())), (ValueError, dict(v_scale=scales[1][:, :1])),
               (ValueError, dict(out=torch.empty(2, 4, 32, dtype=q.dtype, device="cuda"))), (TypeError, dict(scale="x")), (mmv.MmvError, dict(window=-1)),
               (mmv.MmvError, dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda")))]),
             (mmv.kv_append_q8, dict(k=x, v=x, offsets=ints([0, 2, 3]), total=ints([2, 1]), table=table, k_cache=caches[0], v_cache=caches[1], k_scale=scales[0], v_scale=scales[1]),
              [(TypeError, dict(offsets=ints([0, 2, 3]).long())), (ValueError, dict(offsets=ints([0, 3]))), (ValueError, dict(k=x[:, :1])), (TypeError, dict(k=x.bfloat16())),
               (TypeError, dict(k=x.float(), v=x.float())), (TypeError, dict(k_cache=caches[0].half(), v_cache=caches[1].half())), (ValueError, dict(k_cache=caches[0].cpu()))]),
             (mmv.kv_read_q8, dict(k_cache=caches[0], v_cache=caches[1], k_scale=scales[0], v_scale=scales[1], table=table, offsets=ints([0, 2, 3]), tokens=3),
              [(TypeError, dict(dtype=torch.float32)), (TypeError, dict(dtype=3)), (ValueError, dict(tokens=-1)), (TypeError, dict(offsets=ints([0, 2, 3]).long())),
               (TypeError, dict(k=x)), (ValueError, dict(k=x[:2].bfloat16())), (TypeError, dict(tokens="x"))])]
    for call, args, changes in calls:
        call(**args)
        for error, change in changes:
            with pytest.raises(error):
                call(**dict(args, **change))
        for name in ("k_scale", "v_scale"):
            wanting = dict(args, **{name: args[name].detach().requires_grad_()})
            with pytest.raises(RuntimeError, match="no_grad"):
                call(**wanting)
            with torch.no_grad():
                call(**wanting)


def test_calls_on_another_stream_and_in_a_graph(mmv):
    q, caches, scales, table, lens = paged_case(21, [300, 77, 4000], 8, 2, 64, 16, torch.bfloat16, torch.float8_e4m3fn)
    x = torch.randn(3, 2, 64, device="cuda").bfloat16()
    off, ends, keep = ints([0, 1, 2, 3]), ints([0, 300, 377, 4377]), [t.clone() for t in (*caches, *scales)]

    def step(q, x, stream=None):
        mmv.kv_append_q8(x, x, off, lens, table, *caches, *scales, stream=stream)
        out, lse = mmv.paged_attention_q8(q, *caches, *scales, table, lens, stream=stream)
        return (out, lse, *mmv.kv_read_q8(*caches, *scales, table, ends, 4377, stream=stream))

    want = [t.clone() for t in step(q, x)]
    for t, k in zip((*caches, *scales), keep):
        t.copy_(k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(q, x, side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    q1, x1 = torch.zeros_like(q), torch.zeros_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(q1, x1)
    q1.copy_(q)
    x1.copy_(x)
    for _ in range(2):
        for t, k in zip((*caches, *scales), keep):
            t.copy_(k)
        graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
