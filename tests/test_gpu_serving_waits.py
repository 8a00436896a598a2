"""Waits for bulk loads that do not come end with a status: the call returns, other results stand, and the next call works."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_serving_delta import delta_case  # noqa: E402
from test_gpu_serving_q8 import CODES, ints, paged_case  # noqa: E402

TIMEOUT = 5
BUDGET = 20_000_000                          # 20 ms


@pytest.fixture(scope="module")
def mmv():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2506_23906_b200 as m
    m.debug_configure(0, -1)
    return m


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("heads,kv,dim,lens", [(8, 2, 64, [300, 77, 4000, 1]), (4, 1, 128, [9000]), (32, 2, 256, [40, 0, 700])])
def test_attention(mmv, code, heads, kv, dim, lens):
    q, caches, scales, table, lens = paged_case(7, lens, heads, kv, dim, 16, torch.bfloat16, code)
    ws = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    want, wlse = mmv.paged_attention_q8(q, *caches, *scales, table, lens, workspace=ws)
    assert mmv.last_async_status(ws) == 0
    try:
        for block in (0, 3):
            mmv.debug_configure(BUDGET, block)
            mmv.paged_attention_q8(q, *caches, *scales, table, lens, workspace=ws)
            assert mmv.last_async_status(ws) == TIMEOUT
    finally:
        mmv.debug_configure(0, -1)
    out, lse = mmv.paged_attention_q8(q, *caches, *scales, table, lens, workspace=ws)
    assert mmv.last_async_status(ws) == 0 and torch.equal(out, want) and torch.equal(lse, wlse)


@pytest.mark.parametrize("kernel", [0, 1 << 32])
@pytest.mark.parametrize("hk,rep,dk,dv,lens", [(2, 2, 64, 64, [300, 5, 700]), (3, 1, 128, 96, [65, 64]), (36, 1, 64, 64, [9000])])
def test_delta(mmv, kernel, hk, rep, dk, dv, lens):
    """The last case goes in parts: the ones behind the one that gave up find their operands and end."""
    q, k, v, off, g, beta, state = delta_case(5, lens, hk, rep, dk, dv, odd=False)
    ws = torch.zeros(max(256, mmv.gated_delta_workspace_bytes(q, k, v, g, beta, len(lens))), dtype=torch.uint8, device="cuda")
    want, last = mmv.gated_delta(q, k, v, ints(off), g, beta, state=state, workspace=ws)
    assert mmv.last_async_status(ws) == 0
    try:
        for block in (0, 2):
            mmv.debug_configure(BUDGET, kernel + block)
            mmv.gated_delta(q, k, v, ints(off), g, beta, state=state, workspace=ws)
            assert mmv.last_async_status(ws) == TIMEOUT
    finally:
        mmv.debug_configure(0, -1)
    out, s = mmv.gated_delta(q, k, v, ints(off), g, beta, state=state, workspace=ws)
    assert mmv.last_async_status(ws) == 0 and torch.equal(out, want) and torch.equal(s, last)
