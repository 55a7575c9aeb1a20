"""Python binding of the pdyattn C-ABI (include/pdyattn.h).

Argument marshalling only: every step of the computation runs in the HIP
kernels of libpdyattn.so.  torch is used for device memory (outputs and the
workspace are torch allocations) and for the current stream.  There is no
fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
from typing import Optional, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("PDYATTN_LIB", os.path.join(_HERE, "libpdyattn.so"))

PDY_OK = 0
PDY_ERR_INVALID_ARG = -1
PDY_ERR_UNSUPPORTED = -2
PDY_ERR_WORKSPACE = -3
PDY_ERR_HIP = -4

# exported symbols, in the order include/pdyattn.h declares them
SYMBOLS = ("attn_fwd_workspace_size", "attn_bwd_workspace_size", "attn_fwd", "attn_bwd",
           "attn_fwd_chunk_workspace_size", "attn_bwd_chunk_workspace_size", "attn_fwd_chunk",
           "attn_bwd_chunk", "attn_fwd_chunk_shared", "attn_bwd_chunk_shared", "attn_merge",
           "attn_cross_fwd_workspace_size", "attn_cross_fwd", "attn_prefix_fwd_workspace_size",
           "attn_prefix_fwd", "attn_cross_bwd_workspace_size", "attn_cross_bwd",
           "attn_prefix_bwd_workspace_size", "attn_prefix_bwd", "attn_rotary_turns", "attn_rotary",
           "attn_paged_write", "attn_paged_fwd_workspace_size", "attn_paged_fwd",
           "attn_paged_evict_workspace_size", "attn_paged_evict",
           "attn_validate_cu_seqlens", "attn_bwd_noalloc", "pdy_launch_shapes",
           "pdy_chunk_launch_shapes", "pdy_cross_launch_shapes", "pdy_paged_launch_shapes",
           "pdy_status_string", "pdy_last_error",
           "pdy_kernel_count", "pdy_kernel_name", "pdy_profile_start", "pdy_profile_stop")


class PdyError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        self.status = status
        super().__init__(f"{where}: status {status}: {detail}")


_lib = None
_raw_stream = None


def lib() -> ctypes.CDLL:
    """Load libpdyattn.so (built in-tree by paper_2511_13198_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -m paper_2511_13198_amd.build` (no fallback exists)")
    L = ctypes.CDLL(LIB_PATH)
    i32, f32, vp, sz = ctypes.c_int32, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
    L.attn_fwd_workspace_size.argtypes = [i32] * 6
    L.attn_fwd_workspace_size.restype = sz
    L.attn_bwd_workspace_size.argtypes = [i32] * 6
    L.attn_bwd_workspace_size.restype = sz
    L.attn_fwd.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, f32, vp, vp, vp, sz, vp]
    L.attn_fwd.restype = i32
    L.attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, f32,
                           vp, vp, vp, vp, sz, vp]
    L.attn_bwd.restype = i32
    L.attn_fwd_chunk_workspace_size.argtypes = [i32] * 5
    L.attn_fwd_chunk_workspace_size.restype = sz
    L.attn_bwd_chunk_workspace_size.argtypes = [i32] * 5
    L.attn_bwd_chunk_workspace_size.restype = sz
    L.attn_fwd_chunk.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, f32, vp, vp,
                                 vp, sz, vp]
    L.attn_fwd_chunk.restype = i32
    L.attn_bwd_chunk.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32,
                                 f32, vp, vp, vp, i32, vp, sz, vp]
    L.attn_bwd_chunk.restype = i32
    L.attn_fwd_chunk_shared.argtypes = L.attn_fwd_chunk.argtypes + [i32]
    L.attn_fwd_chunk_shared.restype = i32
    L.attn_bwd_chunk_shared.argtypes = L.attn_bwd_chunk.argtypes + [i32]
    L.attn_bwd_chunk_shared.restype = i32
    L.attn_merge.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, vp]
    L.attn_merge.restype = i32
    L.attn_cross_fwd_workspace_size.argtypes = [i32] * 8
    L.attn_cross_fwd_workspace_size.restype = sz
    L.attn_cross_fwd.argtypes = [vp] * 6 + [i32] * 9 + [f32, vp, vp, vp, sz, vp]
    L.attn_cross_fwd.restype = i32
    L.attn_prefix_fwd_workspace_size.argtypes = [i32] * 9
    L.attn_prefix_fwd_workspace_size.restype = sz
    L.attn_prefix_fwd.argtypes = [vp] * 8 + [i32] * 10 + [f32, vp, vp, vp, sz, vp]
    L.attn_prefix_fwd.restype = i32
    L.attn_cross_bwd_workspace_size.argtypes = [i32] * 8
    L.attn_cross_bwd_workspace_size.restype = sz
    L.attn_cross_bwd.argtypes = [vp] * 9 + [i32] * 9 + [f32, i32, vp, vp, vp, vp, sz, vp]
    L.attn_cross_bwd.restype = i32
    L.attn_prefix_bwd_workspace_size.argtypes = [i32] * 9
    L.attn_prefix_bwd_workspace_size.restype = sz
    L.attn_prefix_bwd.argtypes = ([vp] * 11 + [i32] * 10 +
                                  [f32, i32, vp, vp, vp, vp, vp, vp, sz, vp])
    L.attn_prefix_bwd.restype = i32
    L.attn_rotary_turns.argtypes = [vp, i32, vp]
    L.attn_rotary_turns.restype = i32
    L.attn_rotary.argtypes = [vp] * 3 + [i32] * 6 + [vp] * 2 + [i32] * 4 + [vp] * 3
    L.attn_rotary.restype = i32
    L.attn_paged_write.argtypes = [vp] * 7 + [i32] * 8 + [vp] * 4
    L.attn_paged_write.restype = i32
    L.attn_paged_fwd_workspace_size.argtypes = [i32] * 8
    L.attn_paged_fwd_workspace_size.restype = sz
    L.attn_paged_fwd.argtypes = [vp] * 8 + [i32] * 12 + [f32, vp, vp, vp, vp, sz, vp]
    L.attn_paged_fwd.restype = i32
    L.attn_paged_evict_workspace_size.argtypes = [i32] * 4
    L.attn_paged_evict_workspace_size.restype = sz
    L.attn_paged_evict.argtypes = [vp] * 6 + [i32] * 12 + [vp, vp, vp, sz, vp]
    L.attn_paged_evict.restype = i32
    L.attn_validate_cu_seqlens.argtypes = [vp, i32, i32, ctypes.POINTER(i32), vp]
    L.attn_validate_cu_seqlens.restype = i32
    L.attn_bwd_noalloc.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32,
                                   f32, vp, vp, vp, vp]
    L.attn_bwd_noalloc.restype = i32
    L.pdy_launch_shapes.argtypes = [i32] * 7 + [ctypes.POINTER(i32)]
    L.pdy_launch_shapes.restype = i32
    L.pdy_chunk_launch_shapes.argtypes = [i32] * 9 + [ctypes.POINTER(i32)]
    L.pdy_chunk_launch_shapes.restype = i32
    L.pdy_cross_launch_shapes.argtypes = [i32] * 10 + [ctypes.POINTER(i32)]
    L.pdy_cross_launch_shapes.restype = i32
    L.pdy_paged_launch_shapes.argtypes = [i32] * 9 + [ctypes.POINTER(i32)]
    L.pdy_paged_launch_shapes.restype = i32
    L.pdy_status_string.argtypes = [i32]
    L.pdy_status_string.restype = ctypes.c_char_p
    L.pdy_last_error.argtypes = []
    L.pdy_last_error.restype = ctypes.c_char_p
    L.pdy_kernel_count.argtypes = []
    L.pdy_kernel_count.restype = i32
    L.pdy_kernel_name.argtypes = [i32]
    L.pdy_kernel_name.restype = ctypes.c_char_p
    L.pdy_profile_start.argtypes = []
    L.pdy_profile_start.restype = i32
    L.pdy_profile_stop.argtypes = [ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_double), i32]
    L.pdy_profile_stop.restype = i32
    _lib = L
    return L


def _check(status: int, where: str):
    if status != PDY_OK:
        L = lib()
        raise PdyError(status, where,
                       f"{L.pdy_status_string(status).decode()} ({L.pdy_last_error().decode()})")


def profile_start():
    """Start bracketing every kernel this thread launches with HIP events."""
    _check(lib().pdy_profile_start(), "pdy_profile_start")


def profile_stop() -> dict:
    """Stop timing; returns {kernel name: (launches, total ms)} for kernels
    launched since profile_start (waits for their events)."""
    L = lib()
    n = L.pdy_kernel_count()
    launches = (ctypes.c_int32 * n)()
    total = (ctypes.c_double * n)()
    _check(L.pdy_profile_stop(launches, total, n), "pdy_profile_stop")
    return {L.pdy_kernel_name(i).decode(): (int(launches[i]), float(total[i]))
            for i in range(n) if launches[i] > 0}


def last_error() -> str:
    return lib().pdy_last_error().decode()


def _shapes(st: int, where: str, out) -> dict:
    _check(st, where)
    return {n: tuple(out[3 * i:3 * i + 3])
            for i, n in enumerate(("fwd_kernel", "bwd_dq_kernel", "bwd_dkdv_kernel"))}


def launch_shapes(total_tokens, num_seqs, max_seqlen, hq, hkv, d, causal: bool = True) -> dict:
    """{kernel name: (waves, groups, parts)} of the launches that attn_fwd and
    attn_bwd take for these sizes in a workspace of the queried size."""
    out = (ctypes.c_int32 * 9)()
    return _shapes(lib().pdy_launch_shapes(total_tokens, num_seqs, max_seqlen, hq, hkv, d,
                                           int(bool(causal)), out), "pdy_launch_shapes", out)


def chunk_launch_shapes(tq, tk, q_offset, k_offset, hq, hkv, d, causal: bool = True,
                        launches: int = 1) -> dict:
    """The same for attn_fwd_chunk and attn_bwd_chunk."""
    out = (ctypes.c_int32 * 9)()
    return _shapes(lib().pdy_chunk_launch_shapes(tq, tk, q_offset, k_offset, hq, hkv, d,
                                                 int(bool(causal)), launches, out),
                   "pdy_chunk_launch_shapes", out)


def _stream_handle(device) -> int:
    import torch
    global _raw_stream
    if _raw_stream is None:
        # torch's stream handle without a Stream object around it, where the
        # installed torch has it (0.1 us instead of 2)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", False)
    if _raw_stream and device.index is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def fwd_workspace_size(total_tokens, num_seqs, max_seqlen, hq, hkv, d) -> int:
    return int(lib().attn_fwd_workspace_size(total_tokens, num_seqs, max_seqlen, hq, hkv, d))


def bwd_workspace_size(total_tokens, num_seqs, max_seqlen, hq, hkv, d) -> int:
    return int(lib().attn_bwd_workspace_size(total_tokens, num_seqs, max_seqlen, hq, hkv, d))


def validate_cu_seqlens(cu_seqlens, total_tokens: int) -> int:
    """Checks cu_seqlens on the host (synchronising) and returns the longest
    segment length."""
    out = ctypes.c_int32(0)
    st = lib().attn_validate_cu_seqlens(cu_seqlens.data_ptr(), cu_seqlens.numel() - 1,
                                        total_tokens, ctypes.byref(out),
                                        _stream_handle(cu_seqlens.device))
    _check(st, "attn_validate_cu_seqlens")
    return int(out.value)


def _check_tensor(t, name, dtype, ndim):
    if t.dtype == dtype and t.ndim == ndim and t.is_cuda and t.is_contiguous():
        return
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got shape {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _ws(nbytes: int, device):
    import torch
    return torch.empty(max(256, nbytes), dtype=torch.uint8, device=device)


def attn_fwd(q, k, v, cu_seqlens, max_seqlen: Optional[int] = None, causal: bool = True,
             scale: Optional[float] = None, out=None, lse=None, workspace=None):
    """O [T, Hq, d] bf16 and LSE [Hq, T] fp32 (natural log) of Eq. (2) over
    the packed batch described by cu_seqlens (int32 [N+1], on the device)."""
    import torch
    _check_tensor(q, "q", torch.bfloat16, 3)
    _check_tensor(k, "k", torch.bfloat16, 3)
    _check_tensor(v, "v", torch.bfloat16, 3)
    _check_tensor(cu_seqlens, "cu_seqlens", torch.int32, 1)
    T, hq, d = q.shape
    hkv = k.shape[1]
    if k.shape != (T, hkv, d) or v.shape != (T, hkv, d):
        raise ValueError("k and v must be [T, Hkv, d] with q's T and d")
    if max_seqlen is None:
        max_seqlen = validate_cu_seqlens(cu_seqlens, T)
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    n = cu_seqlens.numel() - 1
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((hq, T), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = _ws(fwd_workspace_size(T, n, max_seqlen, hq, hkv, d), q.device)
    st = lib().attn_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), cu_seqlens.data_ptr(), n, T,
                        int(max_seqlen), hq, hkv, d, int(bool(causal)), float(scale),
                        out.data_ptr(), lse.data_ptr(), workspace.data_ptr(),
                        workspace.numel() * workspace.element_size(),
                        _stream_handle(q.device))
    _check(st, "attn_fwd")
    return out, lse


def _bwd_args(q, k, v, o, lse, dout, cu_seqlens, max_seqlen, scale, dq, dk, dv):
    """Checked shapes and outputs of a backward call (outputs allocated by
    torch when not given)."""
    import torch
    for t, name in ((q, "q"), (k, "k"), (v, "v"), (o, "o"), (dout, "dout")):
        _check_tensor(t, name, torch.bfloat16, 3)
    _check_tensor(lse, "lse", torch.float32, 2)
    _check_tensor(cu_seqlens, "cu_seqlens", torch.int32, 1)
    T, hq, d = q.shape
    hkv = k.shape[1]
    if o.shape != (T, hq, d) or dout.shape != (T, hq, d):
        raise ValueError("o and dout must match q")
    if lse.shape != (hq, T):
        raise ValueError("lse must be [Hq, T]")
    if max_seqlen is None:
        max_seqlen = validate_cu_seqlens(cu_seqlens, T)
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    if dq is None:
        dq = torch.empty((T, hq, d), dtype=torch.float32, device=q.device)
    if dk is None:
        dk = torch.empty((T, hkv, d), dtype=torch.float32, device=q.device)
    if dv is None:
        dv = torch.empty((T, hkv, d), dtype=torch.float32, device=q.device)
    for t, name, shape in ((dq, "dq", (T, hq, d)), (dk, "dk", (T, hkv, d)),
                           (dv, "dv", (T, hkv, d))):
        _check_tensor(t, name, torch.float32, 3)
        if t.shape != shape:
            raise ValueError(f"{name} must be {list(shape)}")
    n = cu_seqlens.numel() - 1
    return T, hq, hkv, d, n, int(max_seqlen), float(scale), dq, dk, dv


def attn_bwd(q, k, v, o, lse, dout, cu_seqlens, max_seqlen: Optional[int] = None,
             causal: bool = True, scale: Optional[float] = None, dq=None, dk=None, dv=None,
             workspace=None) -> Tuple:
    """dQ [T, Hq, d], dK, dV [T, Hkv, d] (fp32) of sum(dout * O)."""
    T, hq, hkv, d, n, max_seqlen, scale, dq, dk, dv = _bwd_args(
        q, k, v, o, lse, dout, cu_seqlens, max_seqlen, scale, dq, dk, dv)
    if workspace is None:
        workspace = _ws(bwd_workspace_size(T, n, max_seqlen, hq, hkv, d), q.device)
    st = lib().attn_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
                        dout.data_ptr(), cu_seqlens.data_ptr(), n, T, max_seqlen, hq, hkv, d,
                        int(bool(causal)), scale, dq.data_ptr(), dk.data_ptr(),
                        dv.data_ptr(), workspace.data_ptr(),
                        workspace.numel() * workspace.element_size(), _stream_handle(q.device))
    _check(st, "attn_bwd")
    return dq, dk, dv


def attn_bwd_noalloc(q, k, v, o, lse, dout, cu_seqlens, max_seqlen: Optional[int] = None,
                     causal: bool = True, scale: Optional[float] = None, dq=None, dk=None,
                     dv=None) -> Tuple:
    """attn_bwd without a workspace: the library takes its scratch from a
    static device array of fixed size (PdyError with PDY_ERR_WORKSPACE when
    the sizes need more).  With dq, dk, dv given and max_seqlen known, this
    call allocates nothing.  Calls that overlap on one GPU share that
    scratch and must not run concurrently."""
    T, hq, hkv, d, n, max_seqlen, scale, dq, dk, dv = _bwd_args(
        q, k, v, o, lse, dout, cu_seqlens, max_seqlen, scale, dq, dk, dv)
    st = lib().attn_bwd_noalloc(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                lse.data_ptr(), dout.data_ptr(), cu_seqlens.data_ptr(), n, T,
                                max_seqlen, hq, hkv, d, int(bool(causal)), scale,
                                dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                _stream_handle(q.device))
    _check(st, "attn_bwd_noalloc")
    return dq, dk, dv


# ---------------------------------------------------------------------------
# One long sequence split into chunks (context parallelism)
# ---------------------------------------------------------------------------
def fwd_chunk_workspace_size(tq, tk, hq, hkv, d) -> int:
    return int(lib().attn_fwd_chunk_workspace_size(tq, tk, hq, hkv, d))


def bwd_chunk_workspace_size(tq, tk, hq, hkv, d) -> int:
    return int(lib().attn_bwd_chunk_workspace_size(tq, tk, hq, hkv, d))


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def attn_fwd_chunk(q, k, v, q_offset: int, k_offset: int, causal: bool = True,
                   scale: Optional[float] = None, out=None, lse=None, workspace=None,
                   launches: int = 1):
    """Partial O [Tq, Hq, d] bf16 and LSE [Hq, Tq] fp32 of the query chunk at
    positions q_offset.. over the key/value chunk at positions k_offset..;
    launches: how many such calls the caller runs at a time."""
    import torch
    _check_tensor(q, "q", torch.bfloat16, 3)
    _check_tensor(k, "k", torch.bfloat16, 3)
    _check_tensor(v, "v", torch.bfloat16, 3)
    tq, hq, d = q.shape
    tk, hkv = k.shape[0], k.shape[1]
    if tuple(v.shape) != tuple(k.shape) or k.shape[2] != d:
        raise ValueError("k and v must be [Tk, Hkv, d] with q's d")
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((hq, tq), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = _ws(fwd_chunk_workspace_size(tq, tk, hq, hkv, d), q.device)
    st = lib().attn_fwd_chunk_shared(
        q.data_ptr(), _ptr(k) if tk else 0, _ptr(v) if tk else 0, tq, tk, int(q_offset),
        int(k_offset), hq, hkv, d, int(bool(causal)), float(scale), out.data_ptr(),
        lse.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
        _stream_handle(q.device), int(launches))
    _check(st, "attn_fwd_chunk")
    return out, lse


def attn_bwd_chunk(q, k, v, o, lse, dout, q_offset: int, k_offset: int, causal: bool = True,
                   scale: Optional[float] = None, dq=None, dk=None, dv=None, workspace=None,
                   accumulate: bool = False, launches: int = 1):
    """This (query chunk, key chunk) pair's part of dQ [Tq, Hq, d] and dK, dV
    [Tk, Hkv, d] (fp32), given the final o and lse of the query rows; with
    accumulate=True it is added to the given dq, dk, dv.  launches: how many
    such calls the caller runs at a time."""
    import torch
    for t, name in ((q, "q"), (k, "k"), (v, "v"), (o, "o"), (dout, "dout")):
        _check_tensor(t, name, torch.bfloat16, 3)
    _check_tensor(lse, "lse", torch.float32, 2)
    tq, hq, d = q.shape
    tk, hkv = k.shape[0], k.shape[1]
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    dev = q.device if tq else k.device
    if dq is None:
        dq = torch.empty((tq, hq, d), dtype=torch.float32, device=dev)
    if dk is None:
        dk = torch.empty((tk, hkv, d), dtype=torch.float32, device=dev)
    if dv is None:
        dv = torch.empty((tk, hkv, d), dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = _ws(bwd_chunk_workspace_size(tq, tk, hq, hkv, d), dev)
    st = lib().attn_bwd_chunk_shared(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), dout.data_ptr(),
        tq, tk, int(q_offset), int(k_offset), hq, hkv, d, int(bool(causal)), float(scale),
        dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), int(bool(accumulate)), workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), _stream_handle(dev), int(launches))
    _check(st, "attn_bwd_chunk")
    return dq, dk, dv


def attn_merge(o_a, lse_a, o_b, lse_b, out=None, lse=None):
    """Combine two partial (O, LSE) of the same rows; out/lse may be o_a/lse_a."""
    import torch
    _check_tensor(o_a, "o_a", torch.bfloat16, 3)
    _check_tensor(o_b, "o_b", torch.bfloat16, 3)
    _check_tensor(lse_a, "lse_a", torch.float32, 2)
    _check_tensor(lse_b, "lse_b", torch.float32, 2)
    T, hq, d = o_a.shape
    if tuple(o_b.shape) != (T, hq, d) or tuple(lse_a.shape) != (hq, T) or \
            tuple(lse_b.shape) != (hq, T):
        raise ValueError("partials must share shapes [T, Hq, d] and [Hq, T]")
    if out is None:
        out = torch.empty_like(o_a)
    if lse is None:
        lse = torch.empty_like(lse_a)
    st = lib().attn_merge(o_a.data_ptr(), lse_a.data_ptr(), o_b.data_ptr(), lse_b.data_ptr(), T,
                          hq, d, out.data_ptr(), lse.data_ptr(), _stream_handle(o_a.device))
    _check(st, "attn_merge")
    return out, lse


# ---------------------------------------------------------------------------
# Keys of another length, and keys shared by the batch
# ---------------------------------------------------------------------------
def cross_fwd_workspace_size(total_q, total_k, num_seqs, max_seqlen_q, max_seqlen_k, hq, hkv,
                             d) -> int:
    return int(lib().attn_cross_fwd_workspace_size(total_q, total_k, num_seqs, max_seqlen_q,
                                                   max_seqlen_k, hq, hkv, d))


def prefix_fwd_workspace_size(prefix_len, total_q, total_k, num_seqs, max_seqlen_q, max_seqlen_k,
                              hq, hkv, d) -> int:
    return int(lib().attn_prefix_fwd_workspace_size(prefix_len, total_q, total_k, num_seqs,
                                                    max_seqlen_q, max_seqlen_k, hq, hkv, d))


def cross_bwd_workspace_size(total_q, total_k, num_seqs, max_seqlen_q, max_seqlen_k, hq, hkv,
                             d) -> int:
    return int(lib().attn_cross_bwd_workspace_size(total_q, total_k, num_seqs, max_seqlen_q,
                                                   max_seqlen_k, hq, hkv, d))


def prefix_bwd_workspace_size(prefix_len, total_q, total_k, num_seqs, max_seqlen_q, max_seqlen_k,
                              hq, hkv, d) -> int:
    return int(lib().attn_prefix_bwd_workspace_size(prefix_len, total_q, total_k, num_seqs,
                                                    max_seqlen_q, max_seqlen_k, hq, hkv, d))


def cross_launch_shapes(prefix_len, total_q, total_k, num_seqs, max_seqlen_q, max_seqlen_k, hq, hkv,
                        d, causal: bool = False) -> dict:
    """{kernel name: (waves, groups, parts at most)} of the launches of attn_cross_*
    (prefix_len 0) and attn_prefix_*; "apart": whether the shared keys are a list of
    their own; "fwd_whole_first", "dq_whole_first": whether the first items stay whole and
    the last ones alone are cut."""
    out = (ctypes.c_int32 * 12)()
    _check(lib().pdy_cross_launch_shapes(prefix_len, total_q, total_k, num_seqs, max_seqlen_q,
                                         max_seqlen_k, hq, hkv, d, int(bool(causal)), out),
           "pdy_cross_launch_shapes")
    names = ("cross_fwd_kernel", "cross_dq_kernel", "cross_dkdv_kernel")
    return {**{n: tuple(out[3 * i:3 * i + 3]) for i, n in enumerate(names)}, "apart": bool(out[9]),
            "fwd_whole_first": bool(out[10]), "dq_whole_first": bool(out[11])}


def _launch(name: str, device, *args):
    """Calls the library on the tensors' device and its current stream (the last
    argument); the library launches on the current device."""
    import torch
    index = device.index
    if index is None or torch.cuda.current_device() == index:
        st = getattr(lib(), name)(*args, _stream_handle(device))
    else:
        with torch.cuda.device(index):
            st = getattr(lib(), name)(*args, _stream_handle(device))
    if st != PDY_OK:
        _check(st, name)


def _fits(t, dtype, ndim: int, index) -> bool:
    """Whether t is what a call asks for: type, dims, layout, device (by its index)."""
    return (t.dtype is dtype and t.dim() == ndim and t.get_device() == index and
            t.is_contiguous())


def _refuse(device, *checks):
    """Raises for the first (tensor, name, dtype, dims) that is not what a call asks for,
    on a GPU and the one of the call's first tensor."""
    for t, name, dtype, ndim in checks:
        _check_tensor(t, name, dtype, ndim)
        if t.device != device:
            raise ValueError(f"{name} is on {t.device}, the call's first tensor on {device}")


def _longest(cu, name: str, total: int) -> int:
    """The longest sequence of cu (checked on the host, synchronising)."""
    c = cu.tolist()
    if c[0] != 0 or any(a > b for a, b in zip(c, c[1:])) or c[-1] > total:
        raise ValueError(f"{name} must rise from 0 to at most {total}")
    return max(b - a for a, b in zip(c, c[1:]))


def _cross_args(q, k, v, kp, vp, cu_q, cu_k, max_q, max_k, scale, seqlens_k):
    """Checked arguments of a call: the pointers and numbers of its inputs."""
    import torch
    bf16, i32 = torch.bfloat16, torch.int32
    dev = q.device
    index = dev.index
    shape_q, shape = q.shape, k.shape
    if not (len(shape_q) == 3 and len(shape) == 3 and q.dtype is bf16 and k.dtype is bf16 and
            v.dtype is bf16 and q.is_contiguous() and k.is_contiguous() and v.is_contiguous() and
            q.get_device() == index and k.get_device() == index and v.get_device() == index and
            _fits(cu_q, i32, 1, index) and _fits(cu_k, i32, 1, index)):
        _refuse(dev, (q, "q", bf16, 3), (k, "k", bf16, 3), (v, "v", bf16, 3),
                (cu_q, "cu_seqlens_q", i32, 1), (cu_k, "cu_seqlens_k", i32, 1))
    T, hq, d = shape_q
    tk, hkv, dk = shape
    if dk != d or v.shape != shape:
        raise ValueError("k and v must be [Tk, Hkv, d] with q's d")
    n = cu_q.numel() - 1
    if n < 1 or cu_k.numel() != n + 1:
        raise ValueError("cu_seqlens_q and cu_seqlens_k must have num_seqs + 1 >= 2 offsets each")
    used = 0
    if seqlens_k is not None:
        if not _fits(seqlens_k, i32, 1, index):
            _refuse(dev, (seqlens_k, "seqlens_k", i32, 1))
        if seqlens_k.numel() != n:
            raise ValueError("seqlens_k must have num_seqs lengths")
        used = seqlens_k.data_ptr()
    if max_q is None:  # (the library wants at least 1 where there are rows, of a sequence or not)
        max_q = max(_longest(cu_q, "cu_seqlens_q", T), min(1, T))
    max_k = _longest(cu_k, "cu_seqlens_k", tk) if max_k is None else max_k
    sizes = (n, T, tk, max_q, max_k, hq, hkv, d)
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    ptrs, offsets = (q.data_ptr(), k.data_ptr(), v.data_ptr()), (cu_q.data_ptr(), cu_k.data_ptr(), used)
    if kp is None:
        return dev, ptrs, offsets, (), sizes, scale
    shape = kp.shape
    if not (len(shape) == 3 and kp.dtype is bf16 and vp.dtype is bf16 and kp.is_contiguous() and
            vp.is_contiguous() and kp.get_device() == index and vp.get_device() == index):
        _refuse(dev, (kp, "k_prefix", bf16, 3), (vp, "v_prefix", bf16, 3))
    if shape[1] != hkv or shape[2] != d or vp.shape != shape:
        raise ValueError("k_prefix and v_prefix must be [P, Hkv, d]")
    return (dev, (*ptrs, kp.data_ptr(), vp.data_ptr()), (*offsets, shape[0]), (shape[0],), sizes,
            scale)


def _cross_workspace(kind: str, pre, sizes, device):
    """A workspace for a call of these sizes (kind "fwd" or "bwd")."""
    n, T, tk, max_q, max_k, hq, hkv, d = sizes
    name = f"attn_{'prefix' if pre else 'cross'}_{kind}_workspace_size"
    return _ws(getattr(lib(), name)(*pre, T, tk, n, max_q, max_k, hq, hkv, d), device)


def _check_outputs(dev, o, name: str, lse, workspace, T: int, hq: int, d: int):
    """o [T, Hq, d], lse [Hq, T], a workspace, all on the device."""
    import torch
    index = dev.index
    if not (o.dtype is torch.bfloat16 and lse.dtype is torch.float32 and o.is_contiguous() and
            lse.is_contiguous() and workspace.is_contiguous() and o.get_device() == index and
            lse.get_device() == index and workspace.get_device() == index):
        _refuse(dev, (o, name, torch.bfloat16, 3), (lse, "lse", torch.float32, 2),
                (workspace, "workspace", workspace.dtype, workspace.dim()))
    if o.shape != (T, hq, d) or lse.shape != (hq, T):
        raise ValueError(f"{name} must be q's shape, lse [Hq, T]")


def _cross_fwd(q, k, v, kp, vp, cu_q, cu_k, max_q, max_k, causal, scale, seqlens_k, out, lse,
               workspace):
    import torch
    dev, ptrs, offsets, pre, sizes, scale = _cross_args(q, k, v, kp, vp, cu_q, cu_k, max_q, max_k,
                                                        scale, seqlens_k)
    _, T, _, _, _, hq, _, d = sizes
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((hq, T), dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = _cross_workspace("fwd", pre, sizes, dev)
    _check_outputs(dev, out, "out", lse, workspace, T, hq, d)
    _launch("attn_prefix_fwd" if pre else "attn_cross_fwd", dev, *ptrs, *offsets, *sizes,
            1 if causal else 0, scale, out.data_ptr(), lse.data_ptr(), workspace.data_ptr(),
            workspace.nbytes)
    return out, lse


def attn_cross_fwd(q, k, v, cu_seqlens_q, cu_seqlens_k, max_seqlen_q: Optional[int] = None,
                   max_seqlen_k: Optional[int] = None, causal: bool = False,
                   scale: Optional[float] = None, seqlens_k=None, out=None, lse=None,
                   workspace=None):
    """O [Tq, Hq, d] bf16 and LSE [Hq, Tq] fp32 of every sequence's queries over
    its own keys: q [Tq, Hq, d] cut by cu_seqlens_q, k, v [Tk, Hkv, d] by
    cu_seqlens_k (int32 [N + 1]).  seqlens_k (int32 [N]): only the first so many
    keys of each are in use.  max_seqlen_q, max_seqlen_k: upper bounds of the
    lengths, max_seqlen_k with seqlens_k of these alone (None: read from the
    offsets, waiting for them); a sequence that is longer loses results of its own.
    causal aligns the ends: the last query sees every key.  Rows without a key get
    O = 0, LSE = -inf; rows of no sequence are left."""
    return _cross_fwd(q, k, v, None, None, cu_seqlens_q, cu_seqlens_k, max_seqlen_q,
                      max_seqlen_k, causal, scale, seqlens_k, out, lse, workspace)


def attn_prefix_fwd(q, k, v, k_prefix, v_prefix, cu_seqlens_q, cu_seqlens_k,
                    max_seqlen_q: Optional[int] = None, max_seqlen_k: Optional[int] = None,
                    causal: bool = True, scale: Optional[float] = None, seqlens_k=None, out=None,
                    lse=None, workspace=None):
    """attn_cross_fwd of rows that also see the keys k_prefix, v_prefix [P, Hkv, d],
    which the whole batch shares."""
    if k_prefix is None or v_prefix is None:
        raise ValueError("attn_prefix_fwd needs k_prefix and v_prefix")
    return _cross_fwd(q, k, v, k_prefix, v_prefix, cu_seqlens_q, cu_seqlens_k, max_seqlen_q,
                      max_seqlen_k, causal, scale, seqlens_k, out, lse, workspace)


def _cross_bwd(q, k, v, kp, vp, o, lse, dout, cu_q, cu_k, max_q, max_k, causal, scale, seqlens_k,
               grads, grad_dtype, workspace):
    import torch
    dev, ptrs, offsets, pre, sizes, scale = _cross_args(q, k, v, kp, vp, cu_q, cu_k, max_q, max_k,
                                                        scale, seqlens_k)
    given = [g for g in grads if g is not None]
    dtype = given[0].dtype if given else grad_dtype or torch.float32
    if dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"gradients must be torch.float32 or torch.bfloat16, got {dtype}")
    _, T, tk, _, _, hq, hkv, d = sizes
    index, own = dev.index, (tk, hkv, d)
    shapes = ((T, hq, d), own, own, (pre[0], hkv, d), (pre[0], hkv, d)) if pre else ((T, hq, d), own, own)
    out = []
    for i, shape in enumerate(shapes):
        g = grads[i]
        if g is None:
            g = torch.empty(shape, dtype=dtype, device=dev)
        elif not (g.dtype is dtype and g.shape == shape and g.is_contiguous() and
                  g.get_device() == index):
            name = ("dq", "dk", "dv", "dk_prefix", "dv_prefix")[i]
            _refuse(dev, (g, name, dtype, 3))
            raise ValueError(f"{name} must be {list(shape)}")
        out.append(g)
    if workspace is None:
        workspace = _cross_workspace("bwd", pre, sizes, dev)
    if not _fits(dout, torch.bfloat16, 3, index):
        _refuse(dev, (dout, "dout", torch.bfloat16, 3))
    if dout.shape != shapes[0]:
        raise ValueError("dout must match q")
    _check_outputs(dev, o, "o", lse, workspace, T, hq, d)
    _launch("attn_prefix_bwd" if pre else "attn_cross_bwd", dev, *ptrs, o.data_ptr(),
            lse.data_ptr(), dout.data_ptr(), *offsets, *sizes, 1 if causal else 0, scale,
            1 if dtype is torch.bfloat16 else 0, *[g.data_ptr() for g in out],
            workspace.data_ptr(), workspace.nbytes)
    return tuple(out)


def attn_cross_bwd(q, k, v, o, lse, dout, cu_seqlens_q, cu_seqlens_k,
                   max_seqlen_q: Optional[int] = None, max_seqlen_k: Optional[int] = None,
                   causal: bool = False, scale: Optional[float] = None, seqlens_k=None, dq=None,
                   dk=None, dv=None, grad_dtype=None, workspace=None) -> Tuple:
    """dQ [Tq, Hq, d], dK, dV [Tk, Hkv, d] of sum(dout * O) of attn_cross_fwd, in the
    dtype of the given gradients, else grad_dtype (torch.float32, the default, or
    torch.bfloat16).  Keys not in use get 0; rows of no sequence are left."""
    return _cross_bwd(q, k, v, None, None, o, lse, dout, cu_seqlens_q, cu_seqlens_k,
                      max_seqlen_q, max_seqlen_k, causal, scale, seqlens_k,
                      (dq, dk, dv, None, None), grad_dtype, workspace)


def attn_prefix_bwd(q, k, v, k_prefix, v_prefix, o, lse, dout, cu_seqlens_q, cu_seqlens_k,
                    max_seqlen_q: Optional[int] = None, max_seqlen_k: Optional[int] = None,
                    causal: bool = True, scale: Optional[float] = None, seqlens_k=None, dq=None,
                    dk=None, dv=None, dk_prefix=None, dv_prefix=None, grad_dtype=None,
                    workspace=None) -> Tuple:
    """attn_cross_bwd of attn_prefix_fwd: also dK, dV of the shared keys [P, Hkv, d],
    summed over the rows of all sequences."""
    if k_prefix is None or v_prefix is None:
        raise ValueError("attn_prefix_bwd needs k_prefix and v_prefix")
    return _cross_bwd(q, k, v, k_prefix, v_prefix, o, lse, dout, cu_seqlens_q, cu_seqlens_k,
                      max_seqlen_q, max_seqlen_k, causal, scale, seqlens_k,
                      (dq, dk, dv, dk_prefix, dv_prefix), grad_dtype, workspace)


# ---------------------------------------------------------------------------
# A paged key/value cache
# ---------------------------------------------------------------------------
def paged_fwd_workspace_size(total_q, num_seqs, max_seqlen_q, max_seqlen_k, hq, hkv, d,
                             with_scores: bool = False) -> int:
    return int(lib().attn_paged_fwd_workspace_size(total_q, num_seqs, max_seqlen_q, max_seqlen_k,
                                                   hq, hkv, d, 1 if with_scores else 0))


def paged_evict_workspace_size(num_seqs, max_seqlen_k, hkv, budget) -> int:
    return int(lib().attn_paged_evict_workspace_size(num_seqs, max_seqlen_k, hkv, budget))


def paged_launch_shapes(total_q, num_seqs, max_seqlen_q, max_seqlen_k, hq, hkv, d,
                        e4m3: bool = False, with_scores: bool = False) -> dict:
    """How attn_paged_fwd is launched: waves of a workgroup, rows of a tile, parts at most
    of its keys, and whether weights come from logits that the attention leaves."""
    out = (ctypes.c_int32 * 4)()
    _check(lib().pdy_paged_launch_shapes(total_q, num_seqs, max_seqlen_q, max_seqlen_k, hq, hkv, d,
                                         1 if e4m3 else 0, 1 if with_scores else 0, out),
           "pdy_paged_launch_shapes")
    return {"waves": out[0], "rows": out[1], "parts": out[2], "logits": bool(out[3])}


def _paged_pool(k_pages, v_pages, page_table, seqlens_k, scores, scales=None):
    """Checked pool and tables: (device, shape of the pages, 1 for e4m3, pointers of the
    scores and of scales, (k_scale, v_scale), where the call takes them)."""
    import torch
    dev, dtype, shape, i32 = k_pages.device, k_pages.dtype, k_pages.shape, torch.int32
    index = dev.index
    e4m3 = 1 if dtype is torch.float8_e4m3fn else 0
    if not e4m3 and dtype is not torch.bfloat16:
        raise TypeError(f"k_pages must be torch.bfloat16 or torch.float8_e4m3fn, got {dtype}")
    if not (len(shape) == 4 and v_pages.dtype is dtype and page_table.dtype is i32 and
            seqlens_k.dtype is i32 and page_table.dim() == 2 and seqlens_k.dim() == 1 and
            k_pages.is_contiguous() and v_pages.is_contiguous() and page_table.is_contiguous() and
            seqlens_k.is_contiguous() and k_pages.get_device() == index and
            v_pages.get_device() == index and page_table.get_device() == index and
            seqlens_k.get_device() == index):
        _refuse(dev, (k_pages, "k_pages", dtype, 4), (v_pages, "v_pages", dtype, 4),
                (page_table, "page_table", i32, 2), (seqlens_k, "seqlens_k", i32, 1))
    if v_pages.shape != shape:
        raise ValueError("v_pages must have k_pages' shape [pages, Hkv, page_size, d]")
    n = seqlens_k.numel()
    if n < 1 or page_table.shape[0] != n:
        raise ValueError("page_table and seqlens_k must have num_seqs >= 1 rows each")
    f32 = torch.float32
    ks = vs = sc = 0
    k_scale, v_scale = scales or (None, None)
    if e4m3 and scales:
        if k_scale is None or v_scale is None:
            raise ValueError("an e4m3 cache needs k_scale and v_scale")
        if not (_fits(k_scale, f32, 1, index) and _fits(v_scale, f32, 1, index)):
            _refuse(dev, (k_scale, "k_scale", f32, 1), (v_scale, "v_scale", f32, 1))
        if k_scale.numel() != shape[1] or v_scale.numel() != shape[1]:
            raise ValueError("k_scale and v_scale must have one value a kv head")
        ks, vs = k_scale.data_ptr(), v_scale.data_ptr()
    elif k_scale is not None or v_scale is not None:
        raise ValueError("k_scale and v_scale are of an e4m3 cache (a bf16 one has none)")
    if scores is not None:
        if not (scores.dtype is f32 and scores.is_contiguous() and scores.get_device() == index):
            _refuse(dev, (scores, "scores", f32, 3))
        if scores.shape != shape[:3]:
            raise ValueError("scores must be [pages, Hkv, page_size]")
        sc = scores.data_ptr()
    return dev, shape, e4m3, sc, ks, vs


def attn_paged_write(k, v, k_pages, v_pages, page_table, cu_seqlens, seqlens_k, k_scale=None,
                     v_scale=None, scores=None):
    """New keys and values k, v [T, Hkv, d] bf16 into k_pages, v_pages [pages, Hkv,
    page_size, d], bf16 or torch.float8_e4m3fn (divided by k_scale, v_scale, fp32 [Hkv]):
    the tokens cu_seqlens[i] .. cu_seqlens[i + 1] - 1 become the last of the seqlens_k[i]
    keys (with them) of sequence i, whose pages page_table[i] names (int32 [N, max
    pages]).  scores [pages, Hkv, page_size]: 0 for the new keys."""
    import torch
    dev, shape, e4m3, sc, ks, vs = _paged_pool(k_pages, v_pages, page_table, seqlens_k, scores,
                                               (k_scale, v_scale))
    index, (pages, hkv, page, d), bf16, i32 = dev.index, shape, torch.bfloat16, torch.int32
    if not (k.dtype is bf16 and v.dtype is bf16 and cu_seqlens.dtype is i32 and
            k.is_contiguous() and v.is_contiguous() and cu_seqlens.is_contiguous() and
            k.get_device() == index and v.get_device() == index and
            cu_seqlens.get_device() == index):
        _refuse(dev, (k, "k", bf16, 3), (v, "v", bf16, 3), (cu_seqlens, "cu_seqlens", i32, 1))
    rows = k.shape
    T, (n, width) = rows[0], page_table.shape
    if rows != (T, hkv, d) or v.shape != rows:
        raise ValueError("k and v must be [T, Hkv, d] with the pages' Hkv and d")
    if cu_seqlens.shape != (n + 1,):
        raise ValueError("cu_seqlens must have num_seqs + 1 offsets")
    _launch("attn_paged_write", dev, k.data_ptr(), v.data_ptr(), cu_seqlens.data_ptr(),
            page_table.data_ptr(), seqlens_k.data_ptr(), ks, vs, n, T, pages, page, width, hkv, d,
            e4m3, k_pages.data_ptr(), v_pages.data_ptr(), sc)


def attn_paged_fwd(q, k_pages, v_pages, page_table, cu_seqlens_q, seqlens_k,
                   max_seqlen_q: Optional[int] = None, max_seqlen_k: Optional[int] = None,
                   causal: bool = True, scale: Optional[float] = None, k_scale=None, v_scale=None,
                   scores=None, out=None, lse=None, workspace=None):
    """O [Tq, Hq, d] bf16 and LSE [Hq, Tq] fp32 of every sequence's queries over its
    first seqlens_k[i] keys in the pages page_table[i] of k_pages, v_pages [pages, Hkv,
    page_size, d] (bf16, or torch.float8_e4m3fn with k_scale, v_scale fp32 [Hkv]); q [Tq,
    Hq, d] is cut by cu_seqlens_q.  max_seqlen_q, max_seqlen_k: upper bounds of the
    lengths (None: max_seqlen_q read from the offsets, waiting for them, max_seqlen_k the
    table's room; with scores the workspace grows with it, up to 1 GiB).  causal aligns
    the ends: the last query sees every key.  scores fp32 [pages, Hkv, page_size]: each
    key's attention weight, summed over the sequence's rows and its group's heads, is
    added (at most 65,535 sequences then, and no page in use may be shared by two: sums
    would be lost).  Rows without a key get O = 0, LSE = -inf; rows of no sequence are
    left."""
    import torch
    dev, shape, e4m3, sc, ks, vs = _paged_pool(k_pages, v_pages, page_table, seqlens_k, scores,
                                               (k_scale, v_scale))
    index, (pages, hkv, page, d) = dev.index, shape
    if not (_fits(q, torch.bfloat16, 3, index) and _fits(cu_seqlens_q, torch.int32, 1, index)):
        _refuse(dev, (q, "q", torch.bfloat16, 3), (cu_seqlens_q, "cu_seqlens_q", torch.int32, 1))
    T, hq, dq = q.shape
    n, width = page_table.shape
    if dq != d:
        raise ValueError("q must have the pages' head dimension")
    if cu_seqlens_q.numel() != n + 1:
        raise ValueError("cu_seqlens_q must have num_seqs + 1 offsets")
    if max_seqlen_q is None:
        max_seqlen_q = max(_longest(cu_seqlens_q, "cu_seqlens_q", T), min(1, T))
    if max_seqlen_k is None:
        max_seqlen_k = width * page
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((hq, T), dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = _ws(paged_fwd_workspace_size(T, n, max_seqlen_q, max_seqlen_k, hq, hkv, d,
                                                 scores is not None), dev)
    _check_outputs(dev, out, "out", lse, workspace, T, hq, d)
    _launch("attn_paged_fwd", dev, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
            page_table.data_ptr(), cu_seqlens_q.data_ptr(), seqlens_k.data_ptr(), ks, vs, n, T,
            pages, page, width, max_seqlen_q, max_seqlen_k, hq, hkv, d, e4m3, 1 if causal else 0,
            1.0 / math.sqrt(d) if scale is None else scale, out.data_ptr(), lse.data_ptr(), sc,
            workspace.data_ptr(), workspace.nbytes)
    return out, lse


def attn_paged_evict(k_pages, v_pages, scores, page_table, seqlens_k, new_table, budget: int,
                     recent: int = 0, first: int = 0, max_seqlen_k: Optional[int] = None,
                     kept=None, new_lens=None, workspace=None):
    """Shortens every sequence to at most `budget` keys: each kv head keeps its first
    `first` and last `recent` ones and, of those between, the ones of the highest scores
    (equal ones: the earlier).  Keys, values and scores that stay are copied in their order
    to the pages of new_table (int32 [N, max pages]), none of which the sequences use;
    it is the table of the calls after this one.  At most 65,535 sequences.  Returns kept int32 [N, Hkv, budget], the old number of each key (-1 behind the last),
    and the new lengths int32 [N] (new_lens may be seqlens_k)."""
    import torch
    if scores is None:
        raise ValueError("attn_paged_evict needs scores")
    dev, shape, e4m3, sc, _, _ = _paged_pool(k_pages, v_pages, page_table, seqlens_k, scores)
    i32, index, (pages, hkv, page, d) = torch.int32, dev.index, shape
    n, width = page_table.shape
    if not _fits(new_table, i32, 2, index):
        _refuse(dev, (new_table, "new_table", i32, 2))
    if new_table.shape[0] != n:
        raise ValueError("new_table must have num_seqs rows")
    if max_seqlen_k is None:
        max_seqlen_k = width * page
    if kept is None:
        kept = torch.empty((n, hkv, budget), dtype=i32, device=dev)
    if new_lens is None:
        new_lens = torch.empty((n,), dtype=i32, device=dev)
    if workspace is None:
        workspace = _ws(paged_evict_workspace_size(n, max_seqlen_k, hkv, budget), dev)
    if not (_fits(kept, i32, 3, index) and _fits(new_lens, i32, 1, index) and
            workspace.is_contiguous() and workspace.get_device() == index):
        _refuse(dev, (kept, "kept", i32, 3), (new_lens, "new_lens", i32, 1),
                (workspace, "workspace", workspace.dtype, workspace.dim()))
    if kept.shape != (n, hkv, budget) or new_lens.shape != (n,):
        raise ValueError("kept must be [N, Hkv, budget], new_lens [N]")
    _launch("attn_paged_evict", dev, k_pages.data_ptr(), v_pages.data_ptr(), sc,
            page_table.data_ptr(), seqlens_k.data_ptr(), new_table.data_ptr(), n, pages, page,
            width, new_table.shape[1], max_seqlen_k, hkv, d, e4m3, budget, recent, first,
            kept.data_ptr(), new_lens.data_ptr(), workspace.data_ptr(), workspace.nbytes)
    return kept, new_lens


# ---------------------------------------------------------------------------
# Rotary positions with several axes
# ---------------------------------------------------------------------------
@functools.lru_cache(maxsize=64)
def _rotary_tables(sections: Tuple[int, ...], base: float, freqs: Optional[Tuple[float, ...]]):
    """(pairs, turns, axes): the pairs' frequencies as fractions of a turn and their
    axes, as C arrays, and the arrays' addresses."""
    if any(n < 0 for n in sections):
        raise ValueError(f"sections must be >= 0, got {sections}")
    pairs = sum(sections)
    if freqs is None:
        freqs = tuple(base ** (-p / pairs) for p in range(pairs))
    elif len(freqs) != pairs:
        raise ValueError(f"freqs must have {pairs} values, one a pair, got {len(freqs)}")
    turns = (ctypes.c_uint64 * pairs)()
    axes = (ctypes.c_int32 * pairs)(*(a for a, n in enumerate(sections) for _ in range(n)))
    w = (ctypes.c_double * pairs)(*freqs)
    _check(lib().attn_rotary_turns(w, pairs, turns), "attn_rotary_turns")
    return pairs, ctypes.addressof(turns), ctypes.addressof(axes), (turns, axes)


def attn_rotary(q, k, positions, sections, base: float = 10000.0, freqs=None,
                interleaved: bool = False, inverse: bool = False, out_q=None, out_k=None,
                out_dtype=None):
    """q [T, Hq, d] and k [T, Hkv, d] rotated by their positions (int32 [T, axes], or
    [T] for one): sections[a] pairs of every head turn with axis a, in this order; the
    frequencies are base ** (-p / sum(sections)) for pair p, or freqs[p] (numbers).  A
    pair is elements p and p + sum(sections), or with interleaved 2 p and 2 p + 1;
    elements behind the pairs are copied.  inverse undoes it: the gradients of q and k
    from those of the rotated.  q or k may be None.  bf16, or float32 (out_dtype or
    out_q, out_k bf16 round to it); out_q may be q, out_k k."""
    import torch
    first = q if q is not None else k
    if first is None:
        raise ValueError("attn_rotary needs q or k")
    dev, tin = first.device, first.dtype
    index, types = dev.index, (torch.bfloat16, torch.float32)
    outs = out_q if out_q is not None else out_k
    tout = outs.dtype if outs is not None else out_dtype or tin
    if tin not in types or tout not in types:
        raise TypeError("q, k and the outputs must be torch.bfloat16 or torch.float32, got "
                        f"{tin}, {tout}")

    if (q is None and out_q is not None) or (k is None and out_k is not None):
        raise ValueError("out_q without q" if q is None else "out_k without k")

    T = d = None
    heads, ptrs, filled = [0, 0], [0, 0, 0, 0], [out_q, out_k]
    for i, t in enumerate((q, k)):
        if t is None:
            continue
        o = filled[i]
        if o is None:
            o = filled[i] = torch.empty(t.shape, dtype=tout, device=dev)
        shape = t.shape
        if not (len(shape) == 3 and t.dtype is tin and o.dtype is tout and t.is_contiguous() and
                o.is_contiguous() and t.get_device() == index and o.get_device() == index):
            name = "qk"[i]
            _refuse(dev, (t, name, tin, 3), (o, f"out_{name}", tout, 3))
        if o.shape != shape:
            raise ValueError(f"out_{'qk'[i]} must have {'qk'[i]}'s shape")
        if T is None:
            T, heads[i], d = shape
        elif shape[0] != T or shape[2] != d:
            raise ValueError("q and k must have the same tokens and head dimension")
        else:
            heads[i] = shape[1]
        ptrs[i], ptrs[2 + i] = t.data_ptr(), o.data_ptr()
    if positions.dim() == 1:
        positions = positions[:, None]
    if not _fits(positions, torch.int32, 2, index):
        _refuse(dev, (positions, "positions", torch.int32, 2))
    sections = tuple(sections)
    axes = len(sections)
    if positions.shape != (T, axes):
        raise ValueError(f"positions must be [{T}, {axes}] (tokens, sections), got "
                         f"{list(positions.shape)}")
    pairs, turns, pair_axes, _ = _rotary_tables(sections, base,
                                                None if freqs is None else tuple(freqs))
    _launch("attn_rotary", dev, ptrs[0], ptrs[1], positions.data_ptr(), T, axes, heads[0], heads[1],
            d, pairs, turns, pair_axes, 1 if interleaved else 0, 1 if inverse else 0,
            1 if tin is torch.float32 else 0, 1 if tout is torch.float32 else 0, ptrs[2], ptrs[3])
    return filled[0], filled[1]
