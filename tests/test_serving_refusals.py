"""What the serving operators refuse, through the C ABI and without a GPU: argument errors are reported before any device work."""
import ctypes
import importlib.util
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
I64, I32, VP, SZ, F32 = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
OK, INVALID, SMALL = 0, 1, 3
F16, I8, BF16 = 0, 1, 2


class Cache(ctypes.Structure):
    _fields_ = [("k", VP), ("v", VP), ("num_blocks", I64), ("stride_block", I64), ("stride_token", I64), ("stride_head", I64),
                ("block_size", I32), ("heads", I32), ("dim", I32), ("dtype", I32)]


class Inputs(ctypes.Structure):
    _fields_ = [("q", VP), ("k", VP), ("v", VP)] + [(f"{x}_stride_{y}", I64) for x in "qkv" for y in ("token", "head")] + [
        ("heads", I32), ("kv_heads", I32), ("dim_k", I32), ("dim_v", I32), ("dtype", I32)]


@pytest.fixture(scope="module")
def lib():
    spec = importlib.util.spec_from_file_location("_mmv_build", ROOT / "paper_2506_23906_b200" / "build.py")
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    lib = ctypes.CDLL(str(mod.build()))
    for f in ("mmv_block_tables_workspace_bytes", "mmv_paged_attention_workspace_bytes", "mmv_linear_attention_workspace_bytes"):
        getattr(lib, f).restype = SZ
    lib.mmv_block_tables_workspace_bytes.argtypes = [I64]
    lib.mmv_paged_attention_workspace_bytes.argtypes = [I32, VP]
    lib.mmv_linear_attention_workspace_bytes.argtypes = [VP, I64, I64]
    lib.mmv_block_tables.argtypes = [VP, VP, I64, I32, VP, I64, VP, I64, I64, VP, VP, VP, I64, VP, VP, SZ, VP]
    lib.mmv_kv_append.argtypes = [VP, I64, I64, VP, I64, I64, VP, I64, VP, VP]
    lib.mmv_paged_attention.argtypes = [VP, I64, I64, I32, VP, VP, I64, I64, VP, I64, F32, I64, VP, VP, VP, SZ, VP]
    lib.mmv_linear_attention.argtypes = [VP, VP, I64, I64, VP, F32, VP, VP, VP, VP, SZ, VP]
    lib.mmv_linear_attention_step.argtypes = [VP, I64, VP, F32, VP, VP, VP, I64, VP, VP]
    return lib


def cache(**change):
    c = dict(k=1 << 20, v=1 << 24, num_blocks=9, stride_block=16 * 2 * 64, stride_token=2 * 64, stride_head=64, block_size=16, heads=2, dim=64,
             dtype=F16)
    c.update(change)
    return Cache(**c)


def inputs(**change):
    c = dict(q=1 << 20, k=1 << 21, v=1 << 22, heads=4, kv_heads=2, dim_k=64, dim_v=64, dtype=BF16)
    c.update({f"{x}_stride_{y}": {"token": 512, "head": 64}[y] for x in "qkv" for y in ("token", "head")})
    c.update(change)
    return Inputs(**c)


BAD_CACHES = [dict(dtype=I8), dict(dtype=7), dict(num_blocks=-1), dict(num_blocks=1 << 31), dict(block_size=0), dict(heads=0), dict(heads=1025), dict(dim=0),
              dict(dim=12), dict(dim=264), dict(stride_block=1001), dict(stride_token=132), dict(stride_head=60), dict(k=None), dict(v=None),
              dict(k=(1 << 20) + 8), dict(v=(1 << 24) + 2)]
BAD_INPUTS = [dict(dtype=I8), dict(heads=0), dict(heads=3), dict(kv_heads=0), dict(dim_k=0), dict(dim_k=60), dict(dim_k=136), dict(dim_v=4), dict(dim_v=256),
              dict(q_stride_token=511), dict(k_stride_head=30), dict(v_stride_token=4), dict(q=(1 << 20) + 4), dict(q=None), dict(k=None), dict(v=None)]


def test_block_tables(lib):
    ws = 1 << 30
    good = [16, 16, 4, 16, 16, 10, 16, 8, 8, 16, 16, 16, 100, 16, 256, ws, None]
    for at, value in [(0, None), (0, 18), (1, None), (2, -1), (2, 1 << 20), (3, 0), (3, -4), (4, None), (4, 2), (5, -1), (6, None), (6, 6), (7, 7), (8, -1),
                      (9, None), (9, 2), (10, None), (11, None), (11, 20), (12, -1), (13, None), (13, 6), (14, None), (14, 128)]:
        args = list(good)
        args[at] = value
        assert lib.mmv_block_tables(*args) == INVALID, (at, value)
    args = list(good)
    args[15] = 255
    assert lib.mmv_block_tables(*args) == SMALL
    assert lib.mmv_block_tables_workspace_bytes(-1) == 0 and lib.mmv_block_tables_workspace_bytes(1 << 20) == 0
    assert lib.mmv_block_tables_workspace_bytes(0) == 256
    assert lib.mmv_block_tables_workspace_bytes(100000) >= 256 + 400000


def test_block_tables_outputs_over_inputs(lib):
    """1000 requests; the first bytes or the last ones of an output meet an input that the kernels still read."""
    past, added, free, n = 1 << 20, 1 << 21, 1 << 22, 1000
    good = dict(past=past, added=added, nreq=n, block=16, free=free, nfree=n, table=1 << 23, stride=8, columns=8, offsets=1 << 24, total=1 << 25,
                slots=1 << 26, nslots=n, used=1 << 27, ws=1 << 28, bytes=1 << 20, stream=None)
    for name, size in [("offsets", 4 * (n + 1)), ("total", 4 * n), ("used", 4), ("slots", 8 * n)]:
        for at in (past, added, free):
            for where in (at + 8, at - size + 8, at if name != "total" or at == free else at + 4 * n - 8):
                if where % 8 == 0 or name != "slots":
                    assert lib.mmv_block_tables(*dict(good, **{name: where}).values()) == INVALID, (name, where - at)


@pytest.mark.parametrize("change", BAD_CACHES)
def test_caches(lib, change):
    c = cache(**change)
    assert lib.mmv_kv_append(16, 128, 64, 16, 128, 64, 16, 3, ctypes.byref(c), None) == INVALID
    assert lib.mmv_paged_attention(16, 256, 64, 4, ctypes.byref(c), 16, 8, 8, 16, 3, 1.0, 0, 16, None, 256, 1 << 30, None) == INVALID
    assert lib.mmv_paged_attention_workspace_bytes(4, ctypes.byref(c)) == 0


def test_kv_append(lib):
    c = ctypes.byref(cache())
    good = [16, 128, 64, 16, 128, 64, 16, 3, c, None]
    for at, value in [(0, None), (0, 8), (1, 100), (2, 3), (3, None), (3, 24), (4, 4), (5, 68), (6, None), (6, 12), (7, -1), (8, None)]:
        args = list(good)
        args[at] = value
        assert lib.mmv_kv_append(*args) == INVALID, (at, value)
    assert lib.mmv_kv_append(None, 0, 0, None, 0, 0, None, 0, c, None) == OK                                # nothing to write
    assert lib.mmv_kv_append(16, 0, 0, 16, 0, 0, 16, 5, ctypes.byref(cache(num_blocks=0, k=None, v=None)), None) == OK


def test_paged_attention(lib):
    c = ctypes.byref(cache())
    need = lib.mmv_paged_attention_workspace_bytes(4, c)
    assert 256 < need < 16 << 20
    good = [16, 256, 64, 4, c, 16, 8, 8, 16, 3, 1.0, 0, 16, 16, 256, need, None]
    for at, value in [(0, None), (0, 8), (1, 100), (2, 3), (3, 0), (3, 5), (3, 2048), (4, None), (5, None), (5, 2), (6, 7), (7, -1), (8, None), (8, 6), (9, -1),
                      (9, 1 << 20), (11, -1), (12, None), (12, 24), (13, 18), (14, None), (14, 64)]:
        args = list(good)
        args[at] = value
        assert lib.mmv_paged_attention(*args) == INVALID, (at, value)
    args = list(good)
    args[15] = need - 1
    assert lib.mmv_paged_attention(*args) == SMALL
    assert lib.mmv_paged_attention_workspace_bytes(5, c) == 0 and lib.mmv_paged_attention_workspace_bytes(0, c) == 0


@pytest.mark.parametrize("change", BAD_INPUTS)
def test_linear_inputs(lib, change):
    i = ctypes.byref(inputs(**change))
    assert lib.mmv_linear_attention(i, 16, 2, 70, 16, 1.0, 16, 16, 16, 256, 1 << 30, None) == INVALID
    assert lib.mmv_linear_attention_step(i, 3, 16, 1.0, 16, 16, None, 3, 16, None) == INVALID


def test_linear_attention(lib):
    i = ctypes.byref(inputs())
    need = lib.mmv_linear_attention_workspace_bytes(i, 2, 70)
    assert need >= 256
    good = [i, 16, 2, 70, 16, 1.0, 16, 16, 16, 256, need, None]
    for at, value in [(0, None), (1, None), (1, 6), (2, -1), (2, 1 << 20), (3, -1), (3, 1 << 31), (4, None), (4, 2), (6, 24), (7, 8), (8, None), (8, 24), (9, None),
                      (9, 128)]:
        args = list(good)
        args[at] = value
        assert lib.mmv_linear_attention(*args) == INVALID, (at, value)
    half = ctypes.byref(inputs(dtype=F16))                                                                 # bfloat16 only
    assert lib.mmv_linear_attention(half, *good[1:]) == INVALID
    args = list(good)
    args[10] = need - 1
    assert lib.mmv_linear_attention(*args) == SMALL
    assert lib.mmv_linear_attention_workspace_bytes(i, -1, 5) == 0 and lib.mmv_linear_attention_workspace_bytes(i, 1, 1 << 31) == 0


def test_linear_attention_states_that_overlap(lib):
    i, size = ctypes.byref(inputs()), 4 * 5 * 4 * 64 * 64
    need = lib.mmv_linear_attention_workspace_bytes(i, 5, 70)
    for gap in (0, 16, size - 16, 16 - size, -16):
        assert lib.mmv_linear_attention(i, 1 << 23, 5, 70, 1 << 24, 1.0, 1 << 25, (1 << 25) + gap, 1 << 27, 1 << 28, need, None) == INVALID, gap


def test_linear_attention_step(lib):
    i = ctypes.byref(inputs())
    good = [i, 3, 16, 1.0, 16, 16, 16, 9, 16, None]
    for at, value in [(0, None), (1, -1), (1, 1 << 40), (2, None), (2, 2), (4, None), (4, 24), (5, None), (5, 20), (6, 6), (7, -1), (8, None), (8, 8)]:
        args = list(good)
        args[at] = value
        assert lib.mmv_linear_attention_step(*args) == INVALID, (at, value)
    assert lib.mmv_linear_attention_step(i, 3, 16, 1.0, 16, 16, None, 2, 16, None) == INVALID              # fewer states than requests
    assert lib.mmv_linear_attention_step(i, 0, None, 1.0, None, None, None, 0, None, None) == OK           # nothing to do


def test_linear_attention_step_states_that_overlap(lib):
    i, size = ctypes.byref(inputs()), 4 * 5 * 4 * 64 * 64
    for gap in (16, size - 16, 16 - size, -16):
        assert lib.mmv_linear_attention_step(i, 3, 1 << 24, 1.0, 1 << 25, (1 << 25) + gap, None, 5, 1 << 27, None) == INVALID, gap


def test_strides_of_axes_with_one_entry_do_not_matter(lib):
    c = cache(num_blocks=1, block_size=1, heads=1, stride_block=3, stride_token=5, stride_head=7)
    assert lib.mmv_paged_attention_workspace_bytes(4, ctypes.byref(c)) > 0
    i = inputs(heads=1, kv_heads=1, q_stride_head=3, k_stride_head=1, v_stride_head=5, q_stride_token=1, k_stride_token=3, v_stride_token=9)
    assert lib.mmv_linear_attention_workspace_bytes(ctypes.byref(i), 1, 1) >= 256


def test_binding_refuses_what_is_no_cuda_tensor():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("for a machine without a GPU")
    import paper_2506_23906_b200 as mmv
    x = torch.zeros(2, 1, 8, dtype=torch.bfloat16)
    with pytest.raises((RuntimeError, ValueError)):
        mmv.linear_attention_step(x, x, x, torch.zeros(1), torch.zeros(2, 1, 8, 8))
