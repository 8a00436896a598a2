"""The operators on a key-value cache in 8 bits at the ends of what scores and scales can be.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_serving_q8 import CODES, E, TINY, TYPES, U, check_paged, inside, paged_case, paged_plain  # noqa: E402


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
