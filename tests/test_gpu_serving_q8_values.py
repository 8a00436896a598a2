"""The operators on a key-value cache in 8 bits at the ends of what scores and scales can be: value scales of zero, scores of millions, scales
that the write did not make itself, lengths at the end of 32 bits.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_serving_q8 import CODES, E, TINY, TOP, TYPES, U, append_plain, check_paged, empty_cache, inside, ints, numbers, paged_case, paged_plain  # noqa: E402


@pytest.fixture(scope="module")
def mmv():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2506_23906_b200 as m
    m.debug_configure(0, -1)
    return m


def one(x, code):
    return torch.tensor(x, device="cuda").to(code)


# ---------------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("heads,kv,block", [(8, 2, 16), (24, 2, 16), (3, 3, 7)])
@pytest.mark.parametrize("lens", [[40, 1, 0, 130], [60000, 3], [300] * 40])
@pytest.mark.parametrize("nats", [-100.0, -1000.0, 200.0])
def test_attention_to_values_of_scale_zero(mmv, code, heads, kv, block, lens, nats):
    """All values of one key head have scale 0, of another those of some blocks: its results are 0 whatever the scores are, in requests that one
    range of work holds and in those that several share."""
    q, caches, scales, table, lens = paged_case(len(lens) + kv, lens, heads, kv, 64, block, torch.bfloat16, code)
    q[:] = 1.0
    caches[0].copy_(one(1, code).expand(caches[0].shape))
    scales[0][:] = torch.where(torch.isnan(scales[0]), scales[0], 1.0)
    scales[1][:, 0] = torch.where(torch.isnan(scales[1][:, 0]), scales[1][:, 0], 0.0)
    scales[1][::3, 1] *= 0.0
    check_paged(mmv, (q, caches, scales, table, lens), torch.bfloat16, nats / 64)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("heads,kv,block,window", [(32, 2, 16, 0), (12, 3, 16, 0), (32, 2, 9, 0), (64, 2, 16, 150)])
@pytest.mark.parametrize("bits", [10.0, 17.0, 23.9, 24.0, 24.5, 27.0, 31.0])
@pytest.mark.parametrize("sign", [1, -1])
def test_attention_with_large_scores(mmv, dtype, code, heads, kv, block, window, bits, sign):
    """Scores of 2^bits, one token of each request ahead of the others by hundreds at least, so that all the others' weights are 0 in any arithmetic of
    32 bits: the result is that token's value.  Its weight is 1 = 2^0, exactly; the split into two fp16 values costs 2^-22, the factor that its scale is split into
    2^-23 (a power of two for the largest weight), the sums and products a few e: 2^-20 of it in all.  The logarithm of the sum is the score, products of a few
    factors in fp32: 8 e of it."""
    lens = [1, 2, 33, 300, 17, 9000, 0, 200]
    q, caches, scales, table, lens = paged_case(int(bits * 10) + heads, lens, heads, kv, 64, block, dtype, code)
    q[:] = 0.0
    q[..., 0] = 1.0 + torch.arange(heads, device="cuda") / 64                      # (every head another score)
    far, near = (48, 96) if sign > 0 else (-96, -48)
    caches[0][..., 0] = one(far, code)
    caches[1].copy_(torch.where(caches[1].float().abs() < 2, one(3, code).float(), caches[1].float()).to(code))
    scales[0][:] = torch.where(torch.isnan(scales[0]), scales[0], 0.01)
    rng = np.random.default_rng(3)
    for r, n in enumerate(lens.tolist()):
        if n:
            j = int(rng.integers(max(0, n - window) if window else 0, n))
            caches[0].view(torch.uint8)[table[r, j // block].long(), j % block, :, 0] = one(near, code).view(torch.uint8)
    scale = 2.0 ** bits * float(np.log(2.0)) / (0.01 * abs(near))
    case = q, caches, scales, table, lens
    out, lse = mmv.paged_attention_q8(q, *caches, *scales, table, lens, scale=scale, window=window)
    want, _, wlse, *_ = paged_plain(*case, float(np.float32(scale)), window)
    inside(out, want, (U[dtype] + 2.0 ** -20) * want.abs() + TINY[dtype])
    inside(lse, wlse, torch.nan_to_num(8 * E * wlse.abs(), posinf=0.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dim", [16, 48, 80, 112, 144, 208, 240])
@pytest.mark.parametrize("block,window", [(16, 0), (48, 70), (80, 0)])
def test_attention_odd_dims_and_unused_places(mmv, dtype, code, dim, block, window):
    """Dims between the sizes of a load, in blocks that loads take whole; places behind a request's end and in front of its window hold what is no number (e4m3),
    as do the columns behind dim."""
    lens = [1, 17, 300, 0, 95, 1000]
    q, caches, scales, table, lens = paged_case(dim + block, lens, 6, 2, dim, block, dtype, code, pad=16)
    worst = 0x7f if code == torch.float8_e4m3fn else 0x80
    for c in caches:
        whole = c.view(torch.uint8)
        keep = torch.zeros(whole.shape[:2], dtype=torch.bool, device="cuda")
        for r, n in enumerate(lens.tolist()):
            j = torch.arange(max(0, n - window) if window else 0, n, device="cuda")
            keep[table[r, j // block].long(), j % block] = True
        whole[~keep] = worst
        wide = whole.as_strided((*whole.shape[:3], dim + 16), whole.stride())
        wide[..., dim:] = worst
    check_paged(mmv, (q, caches, scales, table, lens), dtype, dim ** -0.5, window)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("block", [16, 9])
def test_attention_negative_scales(mmv, code, block):
    """A negative scale of keys or of values makes the results that read its block NaN, and no others; zero of either sign is 0."""
    q, caches, scales, table, lens = paged_case(5, [300, 200, 9000], 4, 2, 64, block, torch.float16, code)
    good, glse = mmv.paged_attention_q8(q, *caches, *scales, table, lens)
    for which in (0, 1):
        changed = [s.clone() for s in scales]
        changed[which][table[1, 3], 1] *= -1
        changed[which][table[2, 300], 0] *= -1
        out, lse = mmv.paged_attention_q8(q, *caches, *changed, table, lens)
        hit = torch.zeros(3, 4, dtype=torch.bool, device="cuda")
        hit[1, 2:] = True
        hit[2, :2] = True
        assert torch.isnan(out[hit]).all() and torch.equal(out[~hit], good[~hit]) and torch.equal(lse[~hit], glse[~hit])
        zero = [s.clone() for s in scales]
        zero[which][table[0, 2], 0] = 0.0
        zeros = [s.clone() for s in zero]
        zeros[which][table[0, 2], 0] = -0.0
        assert torch.equal(mmv.paged_attention_q8(q, *caches, *zero, table, lens)[0], mmv.paged_attention_q8(q, *caches, *zeros, table, lens)[0])


# ---------------------------------------------------------------------------------------------------------------------
# the write
# ---------------------------------------------------------------------------------------------------------------------
def arbitrary_scales(gen, n, low, high):
    """fp32 scales with all of their 24 bits, of 2^low to 2^high; ones that a write makes and their neighbours among them."""
    s = np.exp2(gen.uniform(low, high, n)).astype(np.float32)
    s[::5] = np.exp2(np.floor(np.log2(s[::5]))).astype(np.float32)
    s[1::5] = np.nextafter(np.exp2(np.floor(np.log2(s[1::5]))).astype(np.float32), np.float32(0))
    s[2::10] = ((s[2::10].view(np.uint32) & 0xffffe000).view(np.float32))
    return s


@pytest.mark.parametrize("dtype,low,high", [(torch.float16, -12, 4), (torch.bfloat16, -12, 6), (torch.bfloat16, -148.5, -90), (torch.bfloat16, 90, 115)])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("count", [1, 5, 200])
@pytest.mark.parametrize("grows", [False, True])
def test_append_goes_on_in_blocks_of_any_scale(mmv, dtype, low, high, code, count, grows):
    """Blocks whose scales another program made: new codes are x / scale to the nearest (quotients next to halves, and halves, among them), and codes that are
    converted code * old / scale to the nearest."""
    heads, dim, block, past = 6, 64, 256, 7
    top, gen = TOP[code], np.random.default_rng(1000 + count + int(high))
    caches, scales = empty_cache(3, block, heads, dim, code)
    page = 1
    new = []
    for s in scales:
        mine = arbitrary_scales(gen, heads, low, high)
        s[page] = torch.from_numpy(mine).cuda()
        steps = gen.integers(0, int(top), (count, heads, dim)) + gen.choice([0.5, 0.0, 0.25, 0.4999, 0.5001, 0.0625], (count, heads, dim))
        if code != torch.int8:                                         # between two neighbours of e4m3: 2^e (8 + i + 1/2) / 8
            steps = np.exp2(gen.integers(-9, 9, steps.shape)) * (8 + gen.integers(0, 8, steps.shape) + gen.choice([0.5, 0.499, 0.501, 0.0], steps.shape)) / 8
        x = np.minimum(steps, top) * gen.choice([-1.0, 1.0], steps.shape) * mine.astype(np.float64)[None, :, None]
        if grows:
            x[-1, ::2, 3] = mine.astype(np.float64)[::2] * top * 3.7
        x = torch.from_numpy(x).to(dtype)
        if not grows:                                                  # (what a rounding brought above the largest value that fits)
            x = torch.where(x.double().abs() <= torch.from_numpy(mine.astype(np.float64) * top)[None, :, None], x, 0.0)
        new.append(x.cuda())
    want = [(numbers(c), s.double().cpu().numpy()) for c, s in zip(caches, scales)]
    table = [[page]]
    mmv.kv_append_q8(*new, ints([0, count]), ints([past + count]), ints(table), *caches, *scales)
    for (codes, scale), x, c, s in zip(want, new, caches, scales):
        append_plain(codes, scale, x.double().cpu().numpy(), [0, count], [past + count], table, block, top)
        assert np.array_equal(s.double().cpu().numpy(), scale)
        assert np.array_equal(numbers(c), codes)


def test_append_one_quotient_below_a_half(mmv):
    """0.174560546875 / 0.049874447 = 3.49999963: 3."""
    caches, scales = empty_cache(1, 16, 1, 16, torch.int8)
    x = torch.full((1, 1, 16), 0.174560546875, dtype=torch.float16, device="cuda")
    for s in scales:
        s[:] = 0.049874447
    mmv.kv_append_q8(x, -x, ints([0, 1]), ints([2]), ints([[0]]), *caches, *scales)
    assert (caches[0][0, 1] == 3).all() and (caches[1][0, 1] == -3).all()


@pytest.mark.parametrize("block", [8, 1 << 16])
def test_append_at_the_end_of_32_bits(mmv, block):
    """The last tokens of 2^31 - 1 (one row, seen through a stride of zero)."""
    heads, dim, n = 1, 16, 2 ** 31 - 1
    x = torch.randn(1, heads, dim, device="cuda").half()
    k = x.expand(n, heads, dim)
    caches, scales = empty_cache(2, block, heads, dim, torch.int8)
    want = [c.clone() for c in caches], [s.clone() for s in scales]
    mmv.kv_append_q8(x.expand(3, heads, dim), x.expand(3, heads, dim), ints([0, 3]), ints([3]), ints([[1]]), *want[0], *want[1])
    mmv.kv_append_q8(k, k, ints([n - 3, n]), ints([3]), ints([[1]]), *caches, *scales)
    for a, b in zip((*caches, *scales), (*want[0], *want[1])):
        assert torch.equal(a, b)
