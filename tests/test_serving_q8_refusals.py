"""What the operators on a cache in 8 bits refuse, through the C ABI and without a GPU: argument errors are reported before any device work."""
import ctypes
import importlib.util
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
I64, I32, VP, SZ, F32 = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
OK, INVALID, SMALL = 0, 1, 3
F16, I8, BF16 = 0, 1, 2


class Cache(ctypes.Structure):
    _fields_ = [("k", VP), ("v", VP), ("k_scale", VP), ("v_scale", VP), ("num_blocks", I64), ("stride_block", I64), ("stride_token", I64), ("stride_head", I64),
                ("scale_stride_block", I64), ("scale_stride_head", I64), ("block_size", I32), ("heads", I32), ("dim", I32), ("code", I32)]


@pytest.fixture(scope="module")
def lib():
    spec = importlib.util.spec_from_file_location("_mmv_build", ROOT / "paper_2506_23906_b200" / "build.py")
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    lib = ctypes.CDLL(str(mod.build()))
    lib.mmv_paged_attention_q8_workspace_bytes.restype = SZ
    lib.mmv_paged_attention_q8_workspace_bytes.argtypes = [I32, VP]
    lib.mmv_kv_append_q8.argtypes = [VP, I64, I64, VP, I64, I64, I32, I64, VP, VP, I64, VP, I64, I64, VP, VP]
    lib.mmv_kv_read_q8.argtypes = [VP, VP, I64, I64, VP, I64, I64, I32, VP, VP, VP]
    lib.mmv_paged_attention_q8.argtypes = [VP, I64, I64, I32, I32, VP, VP, I64, I64, VP, I64, F32, I64, VP, VP, VP, SZ, VP]
    return lib


def cache(**change):
    c = dict(k=1 << 20, v=1 << 24, k_scale=1 << 26, v_scale=1 << 27, num_blocks=9, stride_block=16 * 2 * 64, stride_token=2 * 64, stride_head=64,
             scale_stride_block=2, scale_stride_head=1, block_size=16, heads=2, dim=64, code=0)
    c.update(change)
    return Cache(**c)


APPEND = [16, 128, 64, 16, 128, 64, F16, 3, 16, 16, 2, 16, 8, 8, None, None]
READ = [None, 16, 8, 8, 16, 2, 100, BF16, 16, 16, None]
ATTEND = [16, 256, 64, 4, BF16, None, 16, 8, 8, 16, 3, 1.0, 0, 16, 16, 256, 1 << 30, None]


@pytest.mark.parametrize("change", [
    dict(code=2), dict(code=-1), dict(num_blocks=-1), dict(num_blocks=1 << 31), dict(block_size=0), dict(block_size=1 << 27), dict(heads=0), dict(heads=1025), dict(dim=0), dict(dim=8),
    dict(dim=72), dict(dim=272), dict(stride_block=1000), dict(stride_token=136), dict(stride_head=60), dict(k=None), dict(v=None), dict(k=(1 << 20) + 8),
    dict(v=(1 << 24) + 2), dict(k_scale=None), dict(v_scale=None), dict(k_scale=(1 << 26) + 2), dict(v_scale=(1 << 27) + 1)])
def test_caches(lib, change):
    c = ctypes.byref(cache(**change))
    assert lib.mmv_kv_append_q8(*APPEND[:14], c, None) == INVALID
    assert lib.mmv_kv_read_q8(c, *READ[1:]) == INVALID
    assert lib.mmv_paged_attention_q8(*ATTEND[:5], c, *ATTEND[6:]) == INVALID
    assert lib.mmv_paged_attention_q8_workspace_bytes(4, c) == 0


def test_kv_append_q8(lib):
    c = ctypes.byref(cache())
    for at, value in [(0, None), (0, 8), (1, 100), (2, 3), (3, None), (3, 24), (4, 4), (5, 68), (6, I8), (6, 9), (7, -1), (7, 1 << 31), (8, None), (8, 6), (9, None), (9, 2),
                      (10, -1), (10, 1 << 20), (11, None), (11, 2), (12, 7), (13, -1)]:
        args = APPEND[:14] + [c, None]
        args[at] = value
        assert lib.mmv_kv_append_q8(*args) == INVALID, (at, value)
    assert lib.mmv_kv_append_q8(None, 0, 0, None, 0, 0, F16, 0, None, None, 0, None, 0, 0, c, None) == OK                  # nothing to write
    assert lib.mmv_kv_append_q8(16, 0, 0, 16, 0, 0, F16, 5, 16, 16, 1, 16, 8, 0, c, None) == OK                            # a table without columns
    empty = ctypes.byref(cache(num_blocks=0, k=None, v=None, k_scale=None, v_scale=None))
    assert lib.mmv_kv_append_q8(*APPEND[:14], empty, None) == OK


def test_kv_read_q8(lib):
    c = ctypes.byref(cache())
    for at, value in [(1, None), (1, 2), (2, 7), (3, -1), (4, None), (4, 6), (5, -1), (5, 1 << 20), (6, -1), (6, 1 << 31), (7, I8), (7, 5), (8, None), (8, 24), (9, None), (9, 8)]:
        args = [c] + READ[1:]
        args[at] = value
        assert lib.mmv_kv_read_q8(*args) == INVALID, (at, value)
    assert lib.mmv_kv_read_q8(c, None, 0, 0, None, 0, 0, BF16, None, None, None) == OK


def test_paged_attention_q8(lib):
    c = ctypes.byref(cache())
    need = lib.mmv_paged_attention_q8_workspace_bytes(4, c)
    assert 256 < need < 16 << 20
    good = ATTEND[:5] + [c] + ATTEND[6:16] + [need, None]
    for at, value in [(0, None), (0, 8), (1, 100), (2, 3), (3, 0), (3, 5), (3, 2048), (4, I8), (4, 4), (5, None), (6, None), (6, 2), (7, 7), (8, -1), (9, None), (9, 6),
                      (10, -1), (10, 1 << 20), (12, -1), (13, None), (13, 24), (14, 18), (15, None), (15, 64)]:
        args = list(good)
        args[at] = value
        assert lib.mmv_paged_attention_q8(*args) == INVALID, (at, value)
    args = list(good)
    args[16] = need - 1
    assert lib.mmv_paged_attention_q8(*args) == SMALL
    assert lib.mmv_paged_attention_q8_workspace_bytes(5, c) == 0 and lib.mmv_paged_attention_q8_workspace_bytes(0, c) == 0


def test_strides_of_axes_with_one_entry_do_not_matter(lib):
    c = cache(num_blocks=1, block_size=1, heads=1, stride_block=3, stride_token=5, stride_head=7, scale_stride_block=0, scale_stride_head=-3)
    assert lib.mmv_paged_attention_q8_workspace_bytes(4, ctypes.byref(c)) > 0
