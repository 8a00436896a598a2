"""The serving example with its cache in 8 bits and with the gated delta rule, against its dense form."""
import importlib.util
from pathlib import Path

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("serve_ragged_batch", Path(__file__).resolve().parent.parent / "examples" / "serve_ragged_batch.py")
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    return ex


@pytest.mark.parametrize("cache", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("delta", [False, True])
def test_example_serves_a_ragged_batch(example, cache, delta):
    """Last logits against the dense fp32 model on the whole sequences: no further off than twice what the dense model itself makes of rounding its
    activations, and its keys and values to 8 bits, at the same places (the server's roundings are others, and as many; a code that is converted when
    its block's scale grows is rounded once more)."""
    off, own = example.difference(*example.serve(4, 5, seed=3, cache=cache, delta=delta))
    assert off < 2 * own
    off, own = example.difference(*example.serve(1, 0, seed=4, cache=cache, delta=delta))
    assert off < 2 * own


@pytest.mark.parametrize("cache,delta", [("int8", True), ("e4m3", False)])
def test_example_serves_pieces(example, cache, delta):
    """Steps in which some requests add no token and others several; the bound as above."""
    server, texts, last = example.serve_in_pieces(example.PIECES, seed=5, cache=cache, delta=delta)
    there = [r for r, t in enumerate(texts) if t.numel()]
    off, own = example.difference(server, [texts[r] for r in there], last[there])
    assert off < 2 * own
