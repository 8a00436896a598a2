"""Attention over the 16-bit paged cache with scores of millions: finite inputs give finite results."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

E = 2.0 ** -24


@pytest.fixture(scope="module")
def mmv():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2506_23906_b200 as m
    m.debug_configure(0, -1)
    return m


@pytest.mark.parametrize("dtype,u", [(torch.float16, 2.0 ** -11), (torch.bfloat16, 2.0 ** -8)])
@pytest.mark.parametrize("heads,kv", [(16, 2), (40, 2)])
@pytest.mark.parametrize("bits", [10.0, 23.0, 24.0, 24.5, 27.0, 31.0])
@pytest.mark.parametrize("sign", [1, -1])
def test_large_scores(mmv, dtype, u, heads, kv, bits, sign):
    """One token of each request is ahead by more than 32 bits can hold of the others' weights, so that the result is its value: the weight is a sum of two 16-bit values,
    2^-16 of it at most, and the sum of the weights divides it, a few e.  The logarithm is the score, products of a few factors in fp32."""
    lens, dim, block = [1, 2, 33, 300, 17, 9000, 0, 200], 64, 16
    gen = torch.Generator("cuda").manual_seed(int(bits))
    pages = [-(-n // block) for n in lens]
    k, v = (torch.zeros(sum(pages), block, kv, dim, dtype=dtype, device="cuda") for _ in range(2))
    v.normal_(generator=gen)
    q = torch.zeros(len(lens), heads, dim, dtype=dtype, device="cuda")
    q[..., 0] = 1.0 + torch.arange(heads, device="cuda") / 64
    far, near = (48.0, 96.0) if sign > 0 else (-96.0, -48.0)
    k[..., 0] = far
    table = torch.zeros(len(lens), max(pages), dtype=torch.int32, device="cuda")
    ids, at, rng = torch.randperm(sum(pages), device="cuda", generator=gen).to(torch.int32), 0, np.random.default_rng(int(bits))
    want = torch.zeros(len(lens), heads, dim, dtype=torch.float64, device="cuda")
    for r, n in enumerate(lens):
        table[r, :pages[r]] = ids[at:at + pages[r]]
        at += pages[r]
        if n:
            j = int(rng.integers(0, n))
            k[table[r, j // block].long(), j % block, :, 0] = near
            want[r] = v[table[r, j // block].long(), j % block].double().repeat_interleave(heads // kv, 0)
    scale = 2.0 ** bits * float(np.log(2.0)) / abs(near)
    out, lse = mmv.paged_attention(q, k, v, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), scale=scale)
    score = float(np.float32(scale)) * near * q[..., 0].double()
    score[6] = -float("inf")
    assert bool(((out.double() - want).abs() <= (u + 2.0 ** -15) * want.abs()).all())
    assert torch.equal(lse[6], torch.full_like(lse[6], -float("inf")))
    on = torch.tensor([n > 0 for n in lens], device="cuda")
    assert bool(((lse.double() - score)[on].abs() <= 8 * E * score[on].abs()).all())
