"""What the gated delta rule refuses, through the C ABI and without a GPU: argument errors are reported before any device work."""
import ctypes
import importlib.util
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
I64, I32, VP, SZ, F32 = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
OK, INVALID, SMALL = 0, 1, 3
F16, I8, BF16 = 0, 1, 2


class Inputs(ctypes.Structure):
    _fields_ = [(x, VP) for x in ("q", "k", "v", "log_decay", "beta")] + [(f"{x}_stride_{y}", I64) for x in "qkv" for y in ("token", "head")] + [
        ("log_decay_stride_token", I64), ("beta_stride_token", I64)] + [(x, I32) for x in ("heads", "key_heads", "dim_k", "dim_v", "dtype")]


@pytest.fixture(scope="module")
def lib():
    spec = importlib.util.spec_from_file_location("_mmv_build", ROOT / "paper_2506_23906_b200" / "build.py")
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    lib = ctypes.CDLL(str(mod.build()))
    lib.mmv_gated_delta_workspace_bytes.restype = SZ
    lib.mmv_gated_delta_workspace_bytes.argtypes = [VP, I64, I64]
    lib.mmv_gated_delta.argtypes = [VP, VP, I64, I64, F32, VP, VP, VP, VP, SZ, VP]
    lib.mmv_gated_delta_step.argtypes = [VP, I64, F32, VP, VP, VP, I64, VP, VP]
    return lib


def inputs(**change):
    c = dict(q=1 << 20, k=1 << 21, v=1 << 22, log_decay=1 << 23, beta=1 << 24, heads=4, key_heads=2, dim_k=64, dim_v=64, dtype=BF16, log_decay_stride_token=7,
             beta_stride_token=4)
    c.update({f"{x}_stride_{y}": {"token": 512, "head": 64}[y] for x in "qkv" for y in ("token", "head")})
    c.update(change)
    return Inputs(**c)


@pytest.mark.parametrize("change", [
    dict(dtype=I8), dict(heads=0), dict(heads=3), dict(heads=1026), dict(key_heads=0), dict(dim_k=0), dict(dim_k=60), dict(dim_k=136), dict(dim_v=4), dict(dim_v=256),
    dict(q_stride_token=511), dict(k_stride_head=30), dict(v_stride_token=4), dict(q=(1 << 20) + 4), dict(q=None), dict(k=None), dict(v=None), dict(log_decay=None),
    dict(beta=None), dict(log_decay=(1 << 23) + 2), dict(beta=(1 << 24) + 1)])
def test_inputs(lib, change):
    i = ctypes.byref(inputs(**change))
    assert lib.mmv_gated_delta(i, 16, 2, 70, 1.0, 16, 1 << 26, 16, 256, 1 << 30, None) == INVALID
    assert lib.mmv_gated_delta_step(i, 3, 1.0, 16, 16, None, 3, 16, None) == INVALID


def test_gated_delta(lib):
    i = ctypes.byref(inputs())
    need = lib.mmv_gated_delta_workspace_bytes(i, 2, 70)
    assert need >= 256
    good = [i, 16, 2, 70, 1.0, 1 << 25, 1 << 26, 16, 256, need, None]
    for at, value in [(0, None), (1, None), (1, 6), (2, -1), (2, 1 << 20), (3, -1), (3, 1 << 31), (5, 24), (6, None), (6, 8), (7, None), (7, 24), (8, None), (8, 128)]:
        args = list(good)
        args[at] = value
        assert lib.mmv_gated_delta(*args) == INVALID, (at, value)
    half = ctypes.byref(inputs(dtype=F16))                                                                 # bfloat16 only
    assert lib.mmv_gated_delta(half, *good[1:]) == INVALID
    args = list(good)
    args[9] = need - 1
    assert lib.mmv_gated_delta(*args) == SMALL
    assert lib.mmv_gated_delta_workspace_bytes(i, -1, 5) == 0 and lib.mmv_gated_delta_workspace_bytes(i, 1, 1 << 31) == 0
    assert lib.mmv_gated_delta_workspace_bytes(i, 1, 1 << 30) <= 200 << 20                                 # (taken in parts)


def test_most_tokens(lib):
    """Positions past the last chunk's end are 32-bit numbers too."""
    i = ctypes.byref(inputs())
    most = (1 << 31) - 1 - 64
    need = lib.mmv_gated_delta_workspace_bytes(i, 2, most)
    assert need >= 256 and lib.mmv_gated_delta_workspace_bytes(i, 2, most + 1) == 0
    assert lib.mmv_gated_delta(i, 16, 2, most + 1, 1.0, 1 << 25, 1 << 26, 16, 256, need, None) == INVALID


def test_states_that_overlap_in_part(lib):
    i, size = ctypes.byref(inputs()), 4 * 5 * 4 * 64 * 64
    need = lib.mmv_gated_delta_workspace_bytes(i, 5, 70)
    for gap in (16, size - 16, 16 - size, -16):
        assert lib.mmv_gated_delta(i, 1 << 23, 5, 70, 1.0, 1 << 25, (1 << 25) + gap, 1 << 27, 1 << 28, need, None) == INVALID, gap
        assert lib.mmv_gated_delta_step(i, 3, 1.0, 1 << 25, (1 << 25) + gap, None, 5, 1 << 27, None) == INVALID, gap


def test_gated_delta_step(lib):
    i = ctypes.byref(inputs())
    good = [i, 3, 1.0, 16, 16, 16, 9, 16, None]
    for at, value in [(0, None), (1, -1), (1, 1 << 40), (3, None), (3, 24), (4, None), (4, 20), (5, 6), (6, -1), (7, None), (7, 8)]:
        args = list(good)
        args[at] = value
        assert lib.mmv_gated_delta_step(*args) == INVALID, (at, value)
    assert lib.mmv_gated_delta_step(i, 3, 1.0, 16, 16, None, 2, 16, None) == INVALID                       # fewer states than requests
    assert lib.mmv_gated_delta_step(i, 0, 1.0, None, None, None, 0, None, None) == OK                      # nothing to do


def test_strides_of_axes_with_one_entry_do_not_matter(lib):
    i = inputs(heads=1, key_heads=1, q_stride_head=3, k_stride_head=1, v_stride_head=5, q_stride_token=1, k_stride_token=3, v_stride_token=9, beta_stride_token=0)
    assert lib.mmv_gated_delta_workspace_bytes(ctypes.byref(i), 1, 1) >= 256
