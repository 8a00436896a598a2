"""Python binding of libmmv.so, the C-ABI CUDA library for segmented scan,
segmented sum and CSR SpMV on B200 (sm_100a).

The binding only marshals arguments (ctypes, and an extension for the serving
operators): torch supplies device memory and the current CUDA stream, every step of the computation runs in the library's own
kernels.  There is no CPU or PyTorch fallback: if the shared library is missing
the import of this module fails, and without the extension the first serving call does.
"""
from __future__ import annotations

import ctypes
import importlib.util
from pathlib import Path

import torch

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libmmv.so"
SERVE_PATH = _PKG / "_serve.so"

# enums of include/mmv.h
MMV_OK = 0
F16_TO_F32, I8_TO_I32, BF16_TO_F32 = 0, 1, 2
SEG_FLAGS_U8, SEG_OFFSETS_I32 = 0, 1
OP_SEG_SCAN, OP_SEG_SUM, OP_SPMV_CSR, OP_COMPRESS, OP_SEG_SCAN_MINMAX, OP_SEG_SCAN_WIDE, OP_MULT = 0, 1, 2, 3, 4, 5, 6

EXPORTS = (
    "mmv_workspace_bytes", "mmv_seg_scan", "mmv_seg_sum", "mmv_spmv_csr",
    "mmv_last_async_status", "mmv_status_string", "mmv_kernel_launch_count", "mmv_debug_configure",
    "mmv_seg_scan_static", "mmv_seg_scan_static_last_status", "mmv_debug_force_sum_groups",
    "mmv_seg_scan_host", "mmv_seg_scan_host_scratch_bytes", "mmv_seg_scan_exclusive", "mmv_compress",
    "mmv_seg_scan_minmax", "mmv_seg_scan_i8_i64", "mmv_seg_scan_shard", "mmv_seg_scan_shard_finish",
    "mmv_debug_force_scan_shape", "mmv_mult_i8",
    "mmv_block_tables_workspace_bytes", "mmv_block_tables", "mmv_kv_append", "mmv_linear_attention_step",
    "mmv_paged_attention_workspace_bytes", "mmv_paged_attention",
    "mmv_linear_attention_workspace_bytes", "mmv_linear_attention",
    "mmv_kv_append_q8", "mmv_kv_read_q8", "mmv_paged_attention_q8_workspace_bytes", "mmv_paged_attention_q8",
    "mmv_gated_delta_step", "mmv_gated_delta_workspace_bytes", "mmv_gated_delta",
)
SHARD_SUMMARY_BYTES = 16
STATIC_SCAN_MAX_N = 1 << 28


class MmvError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} (mmv_status {code})")


def _load() -> ctypes.CDLL:
    if not LIB_PATH.exists():
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python paper_2506_23906_b200/build.py` "
            "(nvcc, sm_100a).  There is no fallback path.")
    lib = ctypes.CDLL(str(LIB_PATH))
    vp, i64, sz, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int
    lib.mmv_workspace_bytes.restype = sz
    lib.mmv_workspace_bytes.argtypes = [ci, ci, ci, i64, i64]
    lib.mmv_seg_scan.restype = ci
    lib.mmv_seg_scan.argtypes = [vp, vp, ci, i64, i64, ci, vp, vp, sz, vp]
    lib.mmv_seg_scan_exclusive.restype = ci
    lib.mmv_seg_scan_exclusive.argtypes = [vp, vp, ci, i64, i64, ci, vp, vp, sz, vp]
    lib.mmv_seg_scan_minmax.restype = ci
    lib.mmv_seg_scan_minmax.argtypes = [vp, vp, i64, ci, ci, vp, vp, sz, vp]
    lib.mmv_seg_scan_i8_i64.restype = ci
    lib.mmv_seg_scan_i8_i64.argtypes = [vp, vp, i64, vp, vp, sz, vp]
    lib.mmv_compress.restype = ci
    lib.mmv_compress.argtypes = [vp, vp, i64, ci, vp, vp, vp, sz, vp]
    lib.mmv_seg_sum.restype = ci
    lib.mmv_seg_sum.argtypes = [vp, vp, ci, i64, i64, ci, vp, vp, vp, sz, vp]
    lib.mmv_spmv_csr.restype = ci
    lib.mmv_spmv_csr.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, vp, sz, vp]
    lib.mmv_last_async_status.restype = ci
    lib.mmv_last_async_status.argtypes = [vp, vp]
    lib.mmv_status_string.restype = ctypes.c_char_p
    lib.mmv_status_string.argtypes = [ci]
    lib.mmv_kernel_launch_count.restype = i64
    lib.mmv_kernel_launch_count.argtypes = []
    lib.mmv_seg_scan_static.restype = ci
    lib.mmv_seg_scan_static.argtypes = [vp, vp, i64, ci, vp, vp]
    lib.mmv_seg_scan_static_last_status.restype = ci
    lib.mmv_seg_scan_static_last_status.argtypes = [vp]
    lib.mmv_debug_configure.restype = None
    lib.mmv_debug_configure.argtypes = [i64, i64]
    lib.mmv_seg_scan_host_scratch_bytes.restype = sz
    lib.mmv_seg_scan_host_scratch_bytes.argtypes = [ci, i64]
    lib.mmv_seg_scan_host.restype = ci
    lib.mmv_seg_scan_host.argtypes = [vp, vp, i64, ci, vp, i64, vp, sz, vp]
    lib.mmv_seg_scan_shard.restype = ci
    lib.mmv_seg_scan_shard.argtypes = [vp, vp, i64, ci, ci, vp, vp, vp, sz, vp]
    lib.mmv_seg_scan_shard_finish.restype = ci
    lib.mmv_seg_scan_shard_finish.argtypes = [vp, ci, ci, vp, i64, ci, vp]
    lib.mmv_mult_i8.restype = ci
    lib.mmv_mult_i8.argtypes = [vp, vp, i64, vp, vp, sz, vp]
    lib.mmv_debug_force_scan_shape.restype = None
    lib.mmv_debug_force_scan_shape.argtypes = [ci]
    lib.mmv_debug_force_sum_groups.restype = None
    lib.mmv_debug_force_sum_groups.argtypes = [ci]
    return lib


_lib = _load()


def status_string(code: int) -> str:
    return _lib.mmv_status_string(int(code)).decode()


def kernel_launch_count() -> int:
    return int(_lib.mmv_kernel_launch_count())


def debug_configure(wait_budget_ns: int = 0, skip_publish_span: int = -1) -> None:
    _lib.mmv_debug_configure(int(wait_budget_ns), int(skip_publish_span))


def debug_force_scan_shape(shape: int = -1) -> None:
    _lib.mmv_debug_force_scan_shape(int(shape))


def debug_force_sum_groups(groups: int = 0) -> None:
    _lib.mmv_debug_force_sum_groups(int(groups))


def workspace_bytes(op: int, dt: int, sf: int, n: int, nseg: int = 0) -> int:
    return int(_lib.mmv_workspace_bytes(op, dt, sf, int(n), int(nseg)))


# (torch.cuda.current_stream() builds a Stream object, 5.7 us per call -- more than a small scan takes on the device;
#  the raw handle of the current stream comes back in a fraction of a microsecond where torch offers it)
_raw_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(stream) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    if _raw_current_stream is not None:
        return int(_raw_current_stream(torch.cuda.current_device()))
    return int(torch.cuda.current_stream().cuda_stream)


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _dtype_code(x: torch.Tensor) -> int:
    if x.dtype == torch.float16:
        return F16_TO_F32
    if x.dtype == torch.int8:
        return I8_TO_I32
    if x.dtype == torch.bfloat16:
        return BF16_TO_F32
    raise TypeError("values must be torch.float16, torch.bfloat16 or torch.int8")


def _seg_code(seg: torch.Tensor) -> int:
    if seg.dtype == torch.uint8:
        return SEG_FLAGS_U8
    if seg.dtype == torch.int32:
        return SEG_OFFSETS_I32
    raise TypeError("segments must be uint8 start flags or int32 offsets")


def _check_cuda(*ts):
    for t in ts:
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("tensors must be contiguous CUDA tensors")


def alloc_workspace(op: int, dt: int, sf: int, n: int, nseg: int = 0, device=None) -> torch.Tensor:
    nbytes = max(256, workspace_bytes(op, dt, sf, n, nseg))
    return torch.empty(nbytes, dtype=torch.uint8, device=device or "cuda")


def last_async_status(workspace: torch.Tensor, stream=None) -> int:
    return int(_lib.mmv_last_async_status(_ptr(workspace), _stream_ptr(stream)))


def seg_scan(x: torch.Tensor, seg: torch.Tensor | None, out: torch.Tensor | None = None,
             workspace: torch.Tensor | None = None, stream=None, exclusive: bool = False) -> torch.Tensor:
    """mmv_seg_scan: segmented inclusive scan (Problem 2.1, Eq. 1) of x over seg; seg = None is the
    plain inclusive scan (one segment, no flag vector is read).  exclusive=True calls
    mmv_seg_scan_exclusive: each element gets the sum of its segment's elements in front of it."""
    _check_cuda(x, seg, out, workspace)
    dt, sf = _dtype_code(x), (SEG_FLAGS_U8 if seg is None else _seg_code(seg))
    n = x.numel()
    nseg = seg.numel() - 1 if sf == SEG_OFFSETS_I32 else 0
    if out is None:
        out = torch.empty(n, dtype=torch.int32 if dt == I8_TO_I32 else torch.float32, device=x.device)
    if workspace is None:
        workspace = alloc_workspace(OP_SEG_SCAN, dt, sf, n, nseg, x.device)
    call = _lib.mmv_seg_scan_exclusive if exclusive else _lib.mmv_seg_scan
    rc = call(_ptr(x), _ptr(seg), sf, n, nseg, dt, _ptr(out), _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc != MMV_OK:
        raise MmvError(rc, "mmv_seg_scan_exclusive" if exclusive else "mmv_seg_scan")
    return out


def seg_scan_shard(x: torch.Tensor, flags: torch.Tensor | None, first_shard: bool, out: torch.Tensor, summary: torch.Tensor,
                   workspace: torch.Tensor, stream=None) -> torch.Tensor:
    """mmv_seg_scan_shard: scan of one contiguous shard of a longer vector, without the carry from the shards in
    front of it; `summary` (16 bytes on the device, e.g. two int64) receives the shard's record."""
    _check_cuda(x, flags, out, summary, workspace)
    if summary.numel() * summary.element_size() < SHARD_SUMMARY_BYTES:
        raise ValueError("summary needs 16 bytes")
    rc = _lib.mmv_seg_scan_shard(_ptr(x), _ptr(flags), x.numel(), _dtype_code(x), 1 if first_shard else 0, _ptr(out),
                                 _ptr(summary), _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc != MMV_OK:
        raise MmvError(rc, "mmv_seg_scan_shard")
    return out


def seg_scan_shard_finish(summaries: torch.Tensor, rank: int, world: int, out: torch.Tensor, x_dtype: torch.dtype,
                          stream=None) -> torch.Tensor:
    """mmv_seg_scan_shard_finish: fold the gathered records of the shards in front of `rank` and add the carry to
    this shard's elements in front of its first start."""
    _check_cuda(summaries, out)
    if summaries.numel() * summaries.element_size() < world * SHARD_SUMMARY_BYTES:
        raise ValueError("summaries needs 16 bytes per shard")
    dt = I8_TO_I32 if x_dtype == torch.int8 else (BF16_TO_F32 if x_dtype == torch.bfloat16 else F16_TO_F32)
    rc = _lib.mmv_seg_scan_shard_finish(_ptr(summaries), int(rank), int(world), _ptr(out), out.numel(), dt, _stream_ptr(stream))
    if rc != MMV_OK:
        raise MmvError(rc, "mmv_seg_scan_shard_finish")
    return out


def mult_i8(x: torch.Tensor, y: torch.Tensor, out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
            stream=None) -> torch.Tensor:
    """mmv_mult_i8: element-wise product of two int8 vectors through the segmented sum (Corollary 4.5), int32."""
    _check_cuda(x, y, out, workspace)
    if x.dtype != torch.int8 or y.dtype != torch.int8 or x.numel() != y.numel():
        raise TypeError("two int8 vectors of the same length expected")
    n = x.numel()
    if out is None:
        out = torch.empty(n, dtype=torch.int32, device=x.device)
    if workspace is None:
        workspace = alloc_workspace(OP_MULT, I8_TO_I32, SEG_OFFSETS_I32, n, 0, x.device)
    rc = _lib.mmv_mult_i8(_ptr(x), _ptr(y), n, _ptr(out), _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc != MMV_OK:
        raise MmvError(rc, "mmv_mult_i8")
    return out


def seg_scan_minmax(x: torch.Tensor, flags: torch.Tensor | None, want_min: bool = False, out: torch.Tensor | None = None,
                    workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """mmv_seg_scan_minmax: segmented running maximum (or minimum) of fp16 / int8 values; flags = None is one segment."""
    _check_cuda(x, flags, out, workspace)
    dt, n = _dtype_code(x), x.numel()
    if out is None:
        out = torch.empty(n, dtype=torch.int32 if dt == I8_TO_I32 else torch.float32, device=x.device)
    if workspace is None:
        workspace = alloc_workspace(OP_SEG_SCAN_MINMAX, dt, SEG_FLAGS_U8, n, 0, x.device)
    rc = _lib.mmv_seg_scan_minmax(_ptr(x), _ptr(flags), n, dt, int(bool(want_min)), _ptr(out), _ptr(workspace),
                                  workspace.numel(), _stream_ptr(stream))
    if rc != MMV_OK:
        raise MmvError(rc, "mmv_seg_scan_minmax")
    return out


def seg_scan_wide(x: torch.Tensor, flags: torch.Tensor | None, out: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """mmv_seg_scan_i8_i64: segmented inclusive scan of int8 values with int64 results (no wrap); flags = None is one segment."""
    _check_cuda(x, flags, out, workspace)
    if x.dtype != torch.int8:
        raise TypeError("seg_scan_wide takes int8 values")
    n = x.numel()
    if out is None:
        out = torch.empty(n, dtype=torch.int64, device=x.device)
    if workspace is None:
        workspace = alloc_workspace(OP_SEG_SCAN_WIDE, I8_TO_I32, SEG_FLAGS_U8, n, 0, x.device)
    rc = _lib.mmv_seg_scan_i8_i64(_ptr(x), _ptr(flags), n, _ptr(out), _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc != MMV_OK:
        raise MmvError(rc, "mmv_seg_scan_i8_i64")
    return out


def compress(x: torch.Tensor, flags: torch.Tensor, out: torch.Tensor | None = None, count: torch.Tensor | None = None,
             workspace: torch.Tensor | None = None, stream=None):
    """mmv_compress: COMPRESS of Section 2 -- the values x[i] with flags[i] != 0, in order.  Returns (out, count):
    out has room for n values of x's type, count is an int64 device tensor holding K; out[:K] is the result."""
    _check_cuda(x, flags, out, workspace)
    if flags.dtype != torch.uint8:
        raise TypeError("flags must be uint8")
    dt, n = _dtype_code(x), x.numel()
    if out is None:
        out = torch.empty(n, dtype=x.dtype, device=x.device)
    if count is None:
        count = torch.zeros(1, dtype=torch.int64, device=x.device)
    if workspace is None:
        workspace = alloc_workspace(OP_COMPRESS, dt, SEG_FLAGS_U8, n, 0, x.device)
    rc = _lib.mmv_compress(_ptr(x), _ptr(flags), n, dt, _ptr(out), _ptr(count), _ptr(workspace), workspace.numel(),
                           _stream_ptr(stream))
    if rc != MMV_OK:
        raise MmvError(rc, "mmv_compress")
    return out, count


def seg_scan_static(x: torch.Tensor, flags: torch.Tensor, out: torch.Tensor, stream=None) -> torch.Tensor:
    """mmv_seg_scan_static: the scan for callers that can pass only inputs and outputs.

    The carry words live in a buffer built into the library, so nothing is allocated by the
    call (here the caller supplies ``out`` too).  n is limited to STATIC_SCAN_MAX_N; calls on
    one device must not overlap on the GPU.
    """
    _check_cuda(x, flags, out)
    if flags.dtype != torch.uint8:
        raise TypeError("start flags must be uint8")
    rc = _lib.mmv_seg_scan_static(_ptr(x), _ptr(flags), x.numel(), _dtype_code(x), _ptr(out), _stream_ptr(stream))
    if rc != MMV_OK:
        raise MmvError(rc, "mmv_seg_scan_static")
    return out


def host_scan_scratch(dt: int, chunk: int, device=None) -> torch.Tensor:
    nbytes = int(_lib.mmv_seg_scan_host_scratch_bytes(dt, int(chunk)))
    if nbytes == 0:
        raise ValueError("chunk must be a positive multiple of 16384")
    return torch.empty(nbytes, dtype=torch.uint8, device=device or "cuda")


def seg_scan_host(x: torch.Tensor, flags: torch.Tensor | None, out: torch.Tensor | None = None, chunk: int = 1 << 26,
                  scratch: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """mmv_seg_scan_host: the scan of HOST tensors (pinned memory recommended), copies and kernels
    of neighbouring chunks overlapped.  Returns ``out`` (a pinned host tensor unless one is given);
    the results are complete once the stream has been synchronised."""
    if x.is_cuda or (flags is not None and flags.is_cuda) or (out is not None and out.is_cuda):
        raise ValueError("seg_scan_host takes host tensors")
    if not x.is_contiguous() or (flags is not None and (flags.dtype != torch.uint8 or not flags.is_contiguous())):
        raise TypeError("contiguous values and uint8 start flags expected")
    dt = _dtype_code(x)
    n = x.numel()
    if out is None:
        out = torch.empty(n, dtype=torch.int32 if dt == I8_TO_I32 else torch.float32, pin_memory=True)
    if scratch is None:
        scratch = host_scan_scratch(dt, chunk)
    rc = _lib.mmv_seg_scan_host(_ptr(x), _ptr(flags), n, dt, _ptr(out), int(chunk), _ptr(scratch), scratch.numel(),
                                _stream_ptr(stream))
    if rc != MMV_OK:
        raise MmvError(rc, "mmv_seg_scan_host")
    return out


def seg_scan_static_last_status(stream=None) -> int:
    return int(_lib.mmv_seg_scan_static_last_status(_stream_ptr(stream)))


def seg_sum(x: torch.Tensor, seg: torch.Tensor, out: torch.Tensor | None = None,
            num_segments: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
            stream=None) -> torch.Tensor:
    """mmv_seg_sum: per-segment sums (Section 2) of x over seg (CSR offsets or flags)."""
    _check_cuda(x, seg, out, workspace, num_segments)
    dt, sf = _dtype_code(x), _seg_code(seg)
    n = x.numel()
    nseg = seg.numel() - 1 if sf == SEG_OFFSETS_I32 else 0
    if out is None:
        cap = nseg if sf == SEG_OFFSETS_I32 else n
        out = torch.empty(cap, dtype=torch.int32 if dt == I8_TO_I32 else torch.float32, device=x.device)
    if workspace is None:
        workspace = alloc_workspace(OP_SEG_SUM, dt, sf, n, nseg, x.device)
    rc = _lib.mmv_seg_sum(_ptr(x), _ptr(seg), sf, n, nseg, dt, _ptr(out), _ptr(num_segments),
                          _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc != MMV_OK:
        raise MmvError(rc, "mmv_seg_sum")
    return out


def spmv_csr(rowptr: torch.Tensor, col: torch.Tensor, val: torch.Tensor, x: torch.Tensor,
             y: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """mmv_spmv_csr: y = A x for a CSR matrix (Algorithm 4.4), fp16 values, fp32 x and y."""
    _check_cuda(rowptr, col, val, x, y, workspace)
    if rowptr.dtype != torch.int32 or col.dtype != torch.int32 or val.dtype != torch.float16 or x.dtype != torch.float32:
        raise TypeError("rowptr/col int32, val float16, x float32 expected")
    rows, cols, nnz = rowptr.numel() - 1, x.numel(), val.numel()
    if y is None:
        y = torch.empty(rows, dtype=torch.float32, device=x.device)
    if workspace is None:
        workspace = alloc_workspace(OP_SPMV_CSR, F16_TO_F32, SEG_OFFSETS_I32, nnz, rows, x.device)
    rc = _lib.mmv_spmv_csr(_ptr(rowptr), _ptr(col), _ptr(val), _ptr(x), _ptr(y), rows, cols, nnz,
                           _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if rc != MMV_OK:
        raise MmvError(rc, "mmv_spmv_csr")
    return y


# ---------------------------------------------------------------------------
# Serving a language model over a ragged batch
#
# These calls take a few microseconds on the GPU in a decoding step; their tensors' metadata is read and checked by a
# small extension (csrc/torch_binding.cpp), which also allocates what is not handed in.  They have no backward pass: in grad mode
# a tensor that requires a gradient is refused (RuntimeError).
# ---------------------------------------------------------------------------
def _load_serve():
    if not SERVE_PATH.exists():
        raise ImportError(f"{SERVE_PATH} is missing: build it with `python paper_2506_23906_b200/build.py`.  There is no fallback path.")
    spec = importlib.util.spec_from_file_location(__name__ + "._serve", SERVE_PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    mod.set_error(MmvError)
    return mod


class _Serve:
    """The extension, loaded at the first serving call (it is tied to one version of torch, which the other operators are not);
    its functions are then this object's own attributes."""

    def __getattr__(self, name: str):
        if name.startswith("__"):
            raise AttributeError(name)
        mod = _load_serve()
        vars(self).update((f, getattr(mod, f)) for f in dir(mod) if not f.startswith("_"))
        return getattr(mod, name)


_serve = _Serve()


def _on_stream(call, stream, inputs, args):
    """A call on a stream other than the current one: what it allocates (and is handed) stays until that stream is done with it."""
    with torch.cuda.stream(stream):
        made = call(*args, None)
    for t in inputs:
        if t is not None:
            t.record_stream(stream)
    return made


def block_tables(past: torch.Tensor, added: torch.Tensor, free_blocks: torch.Tensor, table: torch.Tensor, slots: torch.Tensor,
                 block_size: int, offsets: torch.Tensor | None = None, total: torch.Tensor | None = None,
                 used: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """mmv_block_tables: token offsets, slots and new block-table entries of a packed batch from the requests' lengths.

    past, added: int32 [nreq]; free_blocks: int32; table: int32 [nreq, max_blocks] (rows may be strided), completed in
    place; slots: int64, written whole (-1 behind the last token); total may be past itself (lengths advanced in place).  Returns (offsets int32 [nreq + 1], total int32 [nreq],
    used int32 [1]: how many of free_blocks were taken)."""
    args = (past, added, free_blocks, table, slots, block_size, offsets, total, used, workspace)
    if stream is not None:
        return _on_stream(_serve.block_tables, stream, (past, added, free_blocks, table, slots, offsets, total, used, workspace), args)
    return _serve.block_tables(*args, None)


def kv_append(k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, stream=None) -> None:
    """mmv_kv_append: writes the keys and values k, v [tokens, heads, dim] of a packed batch (views are fine) to their slots
    (int64; negative: skipped) of the paged caches [blocks, block_size, heads, dim] (any order in memory, rows contiguous)."""
    if stream is not None:
        return _on_stream(_serve.kv_append, stream, (k, v, slots, k_cache, v_cache), (k, v, slots, k_cache, v_cache))
    return _serve.kv_append(k, v, slots, k_cache, v_cache, None)


def paged_attention_workspace_bytes(heads: int, k_cache: torch.Tensor, v_cache: torch.Tensor) -> int:
    """mmv_paged_attention_workspace_bytes of a call with `heads` query heads over these caches."""
    return _serve.paged_attention_workspace_bytes(heads, k_cache, v_cache)


def paged_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor, lens: torch.Tensor,
                    scale: float | None = None, window: int = 0, out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                    workspace: torch.Tensor | None = None, stream=None):
    """mmv_paged_attention: attention of one new token per request, q [requests, heads, dim], over the paged caches
    [blocks, block_size, kv_heads, dim] through table int32 [requests, max_blocks] (rows may be strided) and lens int32
    [requests].  scale None: dim ** -0.5; window > 0: the last `window` tokens only.  Returns (out [requests, heads, dim],
    lse fp32 [requests, heads])."""
    args = (q, k_cache, v_cache, table, lens, scale, window, out, lse, workspace)
    if stream is not None:
        return _on_stream(_serve.paged_attention, stream, (q, k_cache, v_cache, table, lens, out, lse, workspace), args)
    return _serve.paged_attention(*args, None)


def kv_append_q8(k: torch.Tensor, v: torch.Tensor, offsets: torch.Tensor, total: torch.Tensor, table: torch.Tensor, k_cache: torch.Tensor,
                 v_cache: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, stream=None) -> None:
    """mmv_kv_append_q8: quantises the keys and values k, v [tokens, heads, dim] of a packed batch (views are fine) into the paged
    caches [blocks, block_size, heads, dim] (int8 or float8_e4m3fn; any order in memory, rows contiguous), a code standing for
    code * scale with k_scale, v_scale fp32 [blocks, heads].

    offsets int32 [requests + 1], total int32 [requests] and table int32 [requests, max_blocks] as block_tables gives them: request
    r's rows are its last tokens, of total[r].  A block that a request goes on in keeps its scale where the new tokens fit; else the
    scale grows and the codes in front of them are converted."""
    args = (k, v, offsets, total, table, k_cache, v_cache, k_scale, v_scale)
    if stream is not None:
        return _on_stream(_serve.kv_append_q8, stream, args, args)
    return _serve.kv_append_q8(*args, None)


def kv_read_q8(k_cache: torch.Tensor, v_cache: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, table: torch.Tensor, offsets: torch.Tensor,
               tokens: int, dtype: torch.dtype = torch.bfloat16, k: torch.Tensor | None = None, v: torch.Tensor | None = None, stream=None):
    """mmv_kv_read_q8: the first offsets[r + 1] - offsets[r] tokens of every request r, read back from caches in 8 bits.

    table int32 [requests, max_blocks], offsets int32 [requests + 1].  Returns (k, v) [tokens, heads, dim] of `dtype` (float16 or bfloat16),
    request r's from row offsets[r] on; rows outside [offsets[0], offsets[requests]) are not written."""
    args = (k_cache, v_cache, k_scale, v_scale, table, offsets, tokens, dtype, k, v)
    if stream is not None:
        return _on_stream(_serve.kv_read_q8, stream, (k_cache, v_cache, k_scale, v_scale, table, offsets, k, v), args)
    return _serve.kv_read_q8(*args, None)


def paged_attention_q8_workspace_bytes(heads: int, k_cache: torch.Tensor, v_cache: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor) -> int:
    """mmv_paged_attention_q8_workspace_bytes of a call with `heads` query heads over these caches."""
    return _serve.paged_attention_q8_workspace_bytes(heads, k_cache, v_cache, k_scale, v_scale)


def paged_attention_q8(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, table: torch.Tensor,
                       lens: torch.Tensor, scale: float | None = None, window: int = 0, out: torch.Tensor | None = None,
                       lse: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """mmv_paged_attention_q8: paged_attention over caches in 8 bits (int8 or float8_e4m3fn [blocks, block_size, kv_heads, dim], scales
    fp32 [blocks, kv_heads]); q float16 or bfloat16.  Returns (out, lse) as paged_attention does."""
    args = (q, k_cache, v_cache, k_scale, v_scale, table, lens, scale, window, out, lse, workspace)
    if stream is not None:
        return _on_stream(_serve.paged_attention_q8, stream, (q, k_cache, v_cache, k_scale, v_scale, table, lens, out, lse, workspace), args)
    return _serve.paged_attention_q8(*args, None)


def linear_attention_workspace_bytes(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, sequences: int) -> int:
    """mmv_linear_attention_workspace_bytes of a call with these inputs."""
    return _serve.linear_attention_workspace_bytes(q, k, v, sequences)


def linear_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, offsets: torch.Tensor, log_decay: torch.Tensor,
                     scale: float = 1.0, state: torch.Tensor | None = None, out: torch.Tensor | None = None,
                     state_out: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """mmv_linear_attention: linear attention with a decay per head over packed sequences.

    q [tokens, heads, dim_k], k, v [tokens, kv_heads, dim_k / dim_v], bfloat16 (views are fine); offsets int32
    [sequences + 1]; log_decay fp32 [heads]; state fp32 [sequences, heads, dim_k, dim_v] in front of the first tokens (None:
    zero).  Returns (out [tokens, heads, dim_v], state_out: the states behind the last tokens).  Unlike the single-token form's,
    state_out must not overlap state."""
    args = (q, k, v, offsets, log_decay, scale, state, out, state_out, workspace)
    if stream is not None:
        return _on_stream(_serve.linear_attention, stream, (q, k, v, offsets, log_decay, state, out, state_out, workspace), args)
    return _serve.linear_attention(*args, None)


def linear_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor, state: torch.Tensor,
                          scale: float = 1.0, slots: torch.Tensor | None = None, state_out: torch.Tensor | None = None,
                          out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """mmv_linear_attention_step: one token of linear attention for every request.

    q [requests, heads, dim_k], k, v [requests, kv_heads, dim_k / dim_v]; log_decay fp32 [heads]; state fp32
    [states, heads, dim_k, dim_v], request r's at slots[r] (int32; None: at r), updated in place unless state_out is given.
    Returns out [requests, heads, dim_v]."""
    args = (q, k, v, log_decay, state, scale, slots, state_out, out)
    if stream is not None:
        return _on_stream(_serve.linear_attention_step, stream, (q, k, v, log_decay, state, slots, state_out, out), args)
    return _serve.linear_attention_step(*args, None)


def gated_delta_workspace_bytes(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor, beta: torch.Tensor, sequences: int) -> int:
    """mmv_gated_delta_workspace_bytes of a call with these inputs."""
    return _serve.gated_delta_workspace_bytes(q, k, v, log_decay, beta, sequences)


def gated_delta(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, offsets: torch.Tensor, log_decay: torch.Tensor, beta: torch.Tensor,
                scale: float = 1.0, state: torch.Tensor | None = None, out: torch.Tensor | None = None,
                state_out: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """mmv_gated_delta: the gated delta rule over packed sequences, S_t = a_t S_{t-1} + k_t u_t^T with
    u_t = beta_t (v_t - a_t S_{t-1}^T k_t), a_t = exp(log_decay_t), out_t = scale S_t^T q_t.

    q, k [tokens, key_heads, dim_k], v [tokens, heads, dim_v], bfloat16 (views are fine), keys normalised; log_decay, beta fp32
    [tokens, heads]; offsets int32 [sequences + 1]; state fp32 [sequences, heads, dim_k, dim_v] in front of the first tokens (None:
    zero).  Returns (out [tokens, heads, dim_v], state_out: the states behind the last tokens; it may be state itself)."""
    args = (q, k, v, offsets, log_decay, beta, scale, state, out, state_out, workspace)
    if stream is not None:
        return _on_stream(_serve.gated_delta, stream, (q, k, v, offsets, log_decay, beta, state, out, state_out, workspace), args)
    return _serve.gated_delta(*args, None)


def gated_delta_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor, beta: torch.Tensor, state: torch.Tensor,
                     scale: float = 1.0, slots: torch.Tensor | None = None, state_out: torch.Tensor | None = None,
                     out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """mmv_gated_delta_step: one token of the gated delta rule for every request.

    q, k [requests, key_heads, dim_k], v [requests, heads, dim_v]; log_decay, beta fp32 [requests, heads]; state fp32
    [states, heads, dim_k, dim_v], request r's at slots[r] (int32; None: at r), updated in place unless state_out is given.
    Returns out [requests, heads, dim_v]."""
    args = (q, k, v, log_decay, beta, state, scale, slots, state_out, out)
    if stream is not None:
        return _on_stream(_serve.gated_delta_step, stream, (q, k, v, log_decay, beta, state, slots, state_out, out), args)
    return _serve.gated_delta_step(*args, None)
