"""The operators on a key-value cache in 8 bits at the ends of what scales can be.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_serving_q8 import CODES, check_paged, paged_case  # noqa: E402


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
