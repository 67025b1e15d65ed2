"""ctypes binding of libflashbias.so: argument marshalling only.

Function names and argument order mirror include/flashbias.h.  Tensors are torch CUDA
tensors used purely as device buffers (data_ptr, dtype, shape); every step of the
computation runs inside the library's HIP kernels.  There is no fallback: if the shared
library is missing or a call returns an error status, an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Callable, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libflashbias.so")

FB_F32, FB_BF16 = 0, 1
_lib_handle = None

EXPORTS = (
    "fb_version", "fb_status_string", "fb_tune_set", "fb_lowrank_attn_fwd", "fb_lowrank_xattn_fwd",
    "fb_alibi_attn_fwd", "fb_dense_bias_attn_fwd", "fb_lowrank_attn_bwd_workspace_bytes",
    "fb_lowrank_attn_bwd", "fb_lowrank_xattn_bwd_workspace_bytes", "fb_lowrank_xattn_bwd",
    "fb_dense_bias_attn_bwd_workspace_bytes", "fb_dense_bias_attn_bwd",
    "fb_lowrank_mulbias_attn_fwd_workspace_bytes", "fb_lowrank_mulbias_attn_fwd",
    "fb_lowrank_mulbias_attn_bwd_workspace_bytes", "fb_lowrank_mulbias_attn_bwd",
    "fb_alibi_attn_bwd_workspace_bytes", "fb_alibi_attn_bwd", "fb_lowrank_attn_bwd_noalloc",
    "fb_fold_batch", "fb_lowrank_xattn_fwd_workspace_bytes", "fb_lowrank_xattn_fwd_ws",
    "fb_attn_bwd_call_workspace_bytes", "fb_rotary_fwd", "fb_rotary_bwd", "fb_paged_plan", "fb_paged_append",
    "fb_paged_attn_fwd_workspace_bytes", "fb_paged_attn_fwd",
)

FB_STATIC_SCRATCH_BYTES = 64 << 20     # include/flashbias.h


class FlashBiasError(RuntimeError):
    pass


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load (once) and type the C-ABI.  Raises FlashBiasError if the library is not built."""
    global _lib_handle
    if _lib_handle is not None and path is None:
        return _lib_handle
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise FlashBiasError(
            f"{p} not found: build it first (python -m paper_2505_12044_amd.build or "
            "__graft_entry__.build()); there is no CPU fallback")
    lib = ctypes.CDLL(p)
    vp, ci, cf, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    lib.fb_version.restype = ci
    lib.fb_version.argtypes = []
    lib.fb_status_string.restype = ctypes.c_char_p
    lib.fb_status_string.argtypes = [ci]
    lib.fb_tune_set.restype = ci
    lib.fb_tune_set.argtypes = [ctypes.c_char_p, ci]
    lib.fb_lowrank_attn_fwd.restype = ci
    lib.fb_lowrank_attn_fwd.argtypes = [vp] * 7 + [ci] * 6 + [ci, ci, ci, cf, vp]
    lib.fb_lowrank_xattn_fwd.restype = ci
    lib.fb_lowrank_xattn_fwd.argtypes = [vp] * 7 + [ci] * 6 + [ci, ci, ci, cf, vp]
    lib.fb_alibi_attn_fwd.restype = ci
    lib.fb_alibi_attn_fwd.argtypes = [vp] * 6 + [ci] * 5 + [ci, cf, vp]
    lib.fb_dense_bias_attn_fwd.restype = ci
    lib.fb_dense_bias_attn_fwd.argtypes = [vp] * 6 + [ci] * 5 + [ci, ci, cf, vp]
    lib.fb_lowrank_attn_bwd_workspace_bytes.restype = sz
    lib.fb_lowrank_attn_bwd_workspace_bytes.argtypes = [ci] * 5 + [ci]
    lib.fb_lowrank_attn_bwd.restype = ci
    lib.fb_lowrank_attn_bwd.argtypes = [vp] * 13 + [ci] * 6 + [ci, ci, ci, cf, vp, sz, vp]
    lib.fb_lowrank_attn_bwd_noalloc.restype = ci
    lib.fb_lowrank_attn_bwd_noalloc.argtypes = [vp] * 13 + [ci] * 6 + [ci, ci, ci, cf, vp]
    lib.fb_dense_bias_attn_bwd_workspace_bytes.restype = sz
    lib.fb_dense_bias_attn_bwd_workspace_bytes.argtypes = [ci] * 4 + [ci]
    lib.fb_dense_bias_attn_bwd.restype = ci
    lib.fb_dense_bias_attn_bwd.argtypes = [vp] * 11 + [ci] * 5 + [ci, ci, cf, vp, sz, vp]
    lib.fb_attn_bwd_call_workspace_bytes.restype = sz
    lib.fb_attn_bwd_call_workspace_bytes.argtypes = [ci] * 7 + [ci]
    lib.fb_lowrank_xattn_bwd_workspace_bytes.restype = sz
    lib.fb_lowrank_xattn_bwd_workspace_bytes.argtypes = [ci] * 6 + [ci]
    lib.fb_lowrank_xattn_bwd.restype = ci
    lib.fb_lowrank_xattn_bwd.argtypes = [vp] * 13 + [ci] * 6 + [ci, ci, ci, cf, vp, sz, vp]
    lib.fb_lowrank_mulbias_attn_fwd_workspace_bytes.restype = sz
    lib.fb_lowrank_mulbias_attn_fwd_workspace_bytes.argtypes = [ci] * 5 + [ci]
    lib.fb_lowrank_mulbias_attn_fwd.restype = ci
    lib.fb_lowrank_mulbias_attn_fwd.argtypes = [vp] * 7 + [ci] * 6 + [ci, ci, ci, cf, vp, sz, vp]
    lib.fb_lowrank_mulbias_attn_bwd_workspace_bytes.restype = sz
    lib.fb_lowrank_mulbias_attn_bwd_workspace_bytes.argtypes = [ci] * 5 + [ci]
    lib.fb_lowrank_mulbias_attn_bwd.restype = ci
    lib.fb_lowrank_mulbias_attn_bwd.argtypes = [vp] * 13 + [ci] * 6 + [ci, ci, ci, cf, vp, sz, vp]
    lib.fb_alibi_attn_bwd_workspace_bytes.restype = sz
    lib.fb_alibi_attn_bwd_workspace_bytes.argtypes = [ci] * 4 + [ci]
    lib.fb_alibi_attn_bwd.restype = ci
    lib.fb_alibi_attn_bwd.argtypes = [vp] * 11 + [ci] * 5 + [ci, cf, vp, sz, vp]
    lib.fb_lowrank_xattn_fwd_workspace_bytes.restype = sz
    lib.fb_lowrank_xattn_fwd_workspace_bytes.argtypes = [ci] * 7
    lib.fb_lowrank_xattn_fwd_ws.restype = ci
    lib.fb_lowrank_xattn_fwd_ws.argtypes = [vp] * 7 + [ci] * 6 + [ci, ci, ci, cf, vp, sz, vp]
    lib.fb_fold_batch.restype = ci
    lib.fb_fold_batch.argtypes = [vp, vp, ctypes.c_longlong, vp, vp, ctypes.c_longlong, ci, ci, vp]
    for f in (lib.fb_rotary_fwd, lib.fb_rotary_bwd):
        f.restype = ci
        f.argtypes = [vp, vp, ci] * 2 + [vp, vp, ci, ci, vp, vp] + [ci] * 5 + [vp]
    lib.fb_paged_plan.restype = ci
    lib.fb_paged_plan.argtypes = [vp] * 9 + [ci] * 5 + [vp]
    lib.fb_paged_append.restype = ci
    lib.fb_paged_append.argtypes = [vp] * 8 + [ci] * 10 + [vp]
    lib.fb_paged_attn_fwd_workspace_bytes.restype = sz
    lib.fb_paged_attn_fwd_workspace_bytes.argtypes = [ci] * 8
    lib.fb_paged_attn_fwd.restype = ci
    lib.fb_paged_attn_fwd.argtypes = [vp] * 11 + [ci] * 13 + [cf, vp, sz, vp]
    if path is None:
        _lib_handle = lib
    return lib


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return FB_F32
    if t.dtype == torch.bfloat16:
        return FB_BF16
    raise FlashBiasError(f"unsupported tensor dtype {t.dtype}")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise FlashBiasError("tensors must be contiguous CUDA tensors")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:      # the raw handle of the current device's current stream, without a Stream object around it
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) or None
    h = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    return h or None


def _scratch(nbytes: int, device, stream, least: Optional[Callable[[], int]] = None) -> torch.Tensor:
    """A workspace the wrapper allocates itself, of `least()` bytes (what the call accepts at a pinch) where there is no
    memory for `nbytes`.  The kernels run on `stream` (a Stream or a raw handle); when
    that is not torch's current stream the caching allocator must be told, or it could hand the block to
    other work as soon as the tensor is dropped."""
    try:
        ws = torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device=device)
    except torch.OutOfMemoryError:
        if least is None or least() >= nbytes:
            raise
        ws = torch.empty(max(int(least()), 16), dtype=torch.uint8, device=device)
    if stream is not None and _stream(stream) != _stream(None):
        ws.record_stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), device=device))
    return ws


def _bwd_scratch(lib, B, H, N, M, C, R, causal, dtype_code, device, stream) -> torch.Tensor:
    """Workspace of one low-rank backward: with the room for dS that it uses (up to 1 GiB), without where memory is short."""
    need = lib.fb_attn_bwd_call_workspace_bytes(B, H, N, M, C, R, 1 if causal else 0, dtype_code)
    return _scratch(need, device, stream, lambda: lib.fb_attn_bwd_call_workspace_bytes(B, H, N, M, C, R, -1, dtype_code))


def _check(status: int, what: str) -> None:
    if status != 0:
        msg = load_library().fb_status_string(status).decode()
        raise FlashBiasError(f"{what} failed: status {status} ({msg})")


def fb_version() -> int:
    return load_library().fb_version()


def fb_tune_set(name: str, value: int) -> None:
    _check(load_library().fb_tune_set(name.encode(), int(value)), "fb_tune_set")


def fb_lowrank_attn_fwd(q, k, v, phi_q, phi_k, out=None, lse=None, causal=False,
                        scale: float = 0.0, phi_batch_broadcast: Optional[bool] = None,
                        stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """out, lse = attention(q, k, v) with bias phi_q phi_k^T.  q, k, v: [B,H,N,C];
    phi_q, phi_k: [B or 1,H,N,R] (None for R = 0)."""
    lib = load_library()
    B, H, N, C = q.shape
    R = 0 if phi_q is None else phi_q.shape[-1]
    if phi_batch_broadcast is None:
        phi_batch_broadcast = phi_q is not None and phi_q.shape[0] == 1 and B > 1
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    phi_code = _dtype_code(phi_q) if phi_q is not None else _dtype_code(q)
    st = lib.fb_lowrank_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(phi_q), _ptr(phi_k), _ptr(out),
                                 _ptr(lse), B, H, N, C, R, int(bool(causal)), _dtype_code(q),
                                 phi_code, int(bool(phi_batch_broadcast)), float(scale),
                                 _stream(stream))
    _check(st, "fb_lowrank_attn_fwd")
    return out, lse


def fb_lowrank_xattn_fwd_workspace_bytes(B, H, N, M, C, R, dtype_code=FB_BF16) -> int:
    return int(load_library().fb_lowrank_xattn_fwd_workspace_bytes(B, H, N, M, C, R, dtype_code))


def fb_lowrank_xattn_fwd(q, k, v, phi_q, phi_k, out=None, lse=None, scale: float = 0.0,
                         phi_batch_broadcast: Optional[bool] = None, stream=None, workspace=None):
    """Cross-attention: q [B,H,N,C], k, v [B,H,M,C], phi_q [B or 1,H,N,R], phi_k [B or 1,H,M,R].
    A few queries against many keys (decode) use scratch of fb_lowrank_xattn_fwd_workspace_bytes: the caller's
    workspace, else the binding's own.  A call that is given out and lse but no workspace allocates nothing and does
    without (the keys of a head are then not split over the GPU)."""
    lib = load_library()
    B, H, N, C = q.shape
    M = k.shape[2]
    R = 0 if phi_q is None else phi_q.shape[-1]
    if phi_batch_broadcast is None:
        phi_batch_broadcast = phi_q is not None and phi_q.shape[0] == 1 and B > 1
    # only a few queries against many keys ever need scratch
    if workspace is None and N <= 8 and (out is None or lse is None):
        need = int(lib.fb_lowrank_xattn_fwd_workspace_bytes(B, H, N, M, C, R, _dtype_code(q)))
        workspace = _scratch(need, q.device, stream) if need else None
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    phi_code = _dtype_code(phi_q) if phi_q is not None else _dtype_code(q)
    st = lib.fb_lowrank_xattn_fwd_ws(_ptr(q), _ptr(k), _ptr(v), _ptr(phi_q), _ptr(phi_k), _ptr(out),
                                     _ptr(lse), B, H, N, M, C, R, _dtype_code(q), phi_code,
                                     int(bool(phi_batch_broadcast)), float(scale), _ptr(workspace), ws_bytes,
                                     _stream(stream))
    _check(st, "fb_lowrank_xattn_fwd")
    return out, lse


def fb_alibi_attn_bwd_workspace_bytes(B, H, N, C, dtype_code=FB_BF16) -> int:
    return int(load_library().fb_alibi_attn_bwd_workspace_bytes(B, H, N, C, dtype_code))


def fb_alibi_attn_bwd(q, k, v, slopes, out, lse, dout, causal=False, scale: float = 0.0, workspace=None,
                      grads=None, dslope_rows=None, stream=None):
    """dq, dk, dv of the attention with the in-kernel ALiBi bias -slopes[h] * (i - j).  dslope_rows: optional
    [B,H,N] float32 tensor that receives each query row's contribution to dL/dslope[h]."""
    lib = load_library()
    B, H, N, C = q.shape
    if slopes.dtype != torch.float32 or slopes.numel() != H:
        raise FlashBiasError("slopes must be a float32 tensor with one entry per head")
    if workspace is None:
        workspace = _bwd_scratch(lib, B, H, N, N, C, 2, causal, _dtype_code(q), q.device, stream)
    if grads is None:
        grads = (torch.empty_like(q), torch.empty_like(k), torch.empty_like(v))
    dq, dk, dv = grads
    st = lib.fb_alibi_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(slopes), _ptr(out), _ptr(lse), _ptr(dout),
                               _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dslope_rows), B, H, N, C, int(bool(causal)),
                               _dtype_code(q), float(scale), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "fb_alibi_attn_bwd")
    return dq, dk, dv


def fb_lowrank_mulbias_attn_fwd_workspace_bytes(B, H, N, C, R, dtype_code=FB_BF16) -> int:
    return int(load_library().fb_lowrank_mulbias_attn_fwd_workspace_bytes(B, H, N, C, R, dtype_code))


def fb_lowrank_mulbias_attn_fwd(q, k, v, phi_q, phi_k, out=None, lse=None, causal=False,
                                scale: float = 0.0, phi_batch_broadcast: Optional[bool] = None,
                                workspace=None, stream=None):
    """out, lse = softmax((q k^T scale) * (phi_q phi_k^T)) v, the multiplicative-bias form.
    q, k, v: [B,H,N,C] bf16; phi_q, phi_k: [B or 1,H,N,R], R >= 1, C (R - 1) <= 128 for C <= 64 (R = 1 at C = 128)."""
    lib = load_library()
    B, H, N, C = q.shape
    R = phi_q.shape[-1]
    if phi_batch_broadcast is None:
        phi_batch_broadcast = phi_q.shape[0] == 1 and B > 1
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    need = fb_lowrank_mulbias_attn_fwd_workspace_bytes(B, H, N, C, R)
    if workspace is None:
        workspace = _scratch(need, q.device, stream)
    st = lib.fb_lowrank_mulbias_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(phi_q), _ptr(phi_k), _ptr(out),
                                         _ptr(lse), B, H, N, C, R, int(bool(causal)), _dtype_code(q),
                                         _dtype_code(phi_q), int(bool(phi_batch_broadcast)), float(scale),
                                         _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "fb_lowrank_mulbias_attn_fwd")
    return out, lse


def fb_lowrank_mulbias_attn_bwd_workspace_bytes(B, H, N, C, R, dtype_code=FB_BF16) -> int:
    return int(load_library().fb_lowrank_mulbias_attn_bwd_workspace_bytes(B, H, N, C, R, dtype_code))


def fb_lowrank_mulbias_attn_bwd(q, k, v, phi_q, phi_k, out, lse, dout, causal=False, scale: float = 0.0,
                                phi_batch_broadcast: Optional[bool] = None, workspace=None, grads=None,
                                stream=None):
    """dq, dk, dv, dphi_q, dphi_k of the multiplicative-bias attention (dphi_*: [B,H,N,R] in the
    factors' dtype, per batch element)."""
    lib = load_library()
    B, H, N, C = q.shape
    R = phi_q.shape[-1]
    if phi_batch_broadcast is None:
        phi_batch_broadcast = phi_q.shape[0] == 1 and B > 1
    if workspace is None:
        need = least = fb_lowrank_mulbias_attn_bwd_workspace_bytes(B, H, N, C, R)
        if C == 128:      # the query holds the room for dS of either mask
            full, masked, plain = (lib.fb_attn_bwd_call_workspace_bytes(B, H, N, N, C, 0, m, FB_BF16) for m in (0, 1, -1))
            least -= max(full, masked) - plain
            need = least + (masked if causal else full) - plain
        workspace = _scratch(need, q.device, stream, lambda: least)
    if grads is None:
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        dpq = torch.empty((B, H, N, R), dtype=phi_q.dtype, device=q.device)
        dpk = torch.empty((B, H, N, R), dtype=phi_k.dtype, device=q.device)
    else:
        dq, dk, dv, dpq, dpk = grads
    st = lib.fb_lowrank_mulbias_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(phi_q), _ptr(phi_k), _ptr(out), _ptr(lse),
                                         _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dpq), _ptr(dpk),
                                         B, H, N, C, R, int(bool(causal)), _dtype_code(q), _dtype_code(phi_q),
                                         int(bool(phi_batch_broadcast)), float(scale), _ptr(workspace),
                                         workspace.numel(), _stream(stream))
    _check(st, "fb_lowrank_mulbias_attn_bwd")
    return dq, dk, dv, dpq, dpk


def fb_alibi_attn_fwd(q, k, v, slopes, out=None, lse=None, causal=False, scale: float = 0.0,
                      stream=None):
    """out, lse = attention(q, k, v) with the bias -slopes[h] * (i - j) generated in the kernel.
    slopes: [H] float32 CUDA tensor."""
    lib = load_library()
    B, H, N, C = q.shape
    if slopes.dtype != torch.float32 or slopes.numel() != H:
        raise FlashBiasError("slopes must be a float32 tensor with one entry per head")
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    st = lib.fb_alibi_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(slopes), _ptr(out), _ptr(lse),
                               B, H, N, C, int(bool(causal)), _dtype_code(q), float(scale),
                               _stream(stream))
    _check(st, "fb_alibi_attn_fwd")
    return out, lse


def fb_dense_bias_attn_fwd(q, k, v, bias, out=None, lse=None, causal=False, scale: float = 0.0,
                           bias_batch_broadcast: Optional[bool] = None, stream=None):
    """out, lse = attention(q, k, v) with a dense bias [B or 1,H,N,N] of q's dtype."""
    lib = load_library()
    B, H, N, C = q.shape
    if bias_batch_broadcast is None:
        bias_batch_broadcast = bias.shape[0] == 1 and B > 1
    if bias.dtype != q.dtype:
        raise FlashBiasError("dense bias must have q's dtype")
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    st = lib.fb_dense_bias_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(bias), _ptr(out), _ptr(lse),
                                    B, H, N, C, int(bool(causal)), _dtype_code(q),
                                    int(bool(bias_batch_broadcast)), float(scale), _stream(stream))
    _check(st, "fb_dense_bias_attn_fwd")
    return out, lse


def fb_lowrank_attn_bwd_workspace_bytes(B, H, N, C, R, dtype_code=FB_BF16) -> int:
    return int(load_library().fb_lowrank_attn_bwd_workspace_bytes(B, H, N, C, R, dtype_code))


def fb_lowrank_attn_bwd(q, k, v, phi_q, phi_k, out, lse, dout, causal=False, scale: float = 0.0,
                        phi_batch_broadcast: Optional[bool] = None, workspace=None, grads=None,
                        stream=None):
    """dq, dk, dv, dphi_q, dphi_k for an upstream gradient dout.  dphi_* are [B,H,N,R]
    (per batch element) in the factors' dtype; None when R = 0.  Without a workspace of the caller's the binding
    allocates one for the call: linear in B H N, and up to 1 GiB more for dS (bf16 at C = 128, fp32 from C = 32 on)
    where the call uses it and the memory is there; any workspace from the linear size on is taken."""
    lib = load_library()
    B, H, N, C = q.shape
    R = 0 if phi_q is None else phi_q.shape[-1]
    if phi_batch_broadcast is None:
        phi_batch_broadcast = phi_q is not None and phi_q.shape[0] == 1 and B > 1
    phi_code = _dtype_code(phi_q) if phi_q is not None else _dtype_code(q)
    if workspace is None:
        workspace = _bwd_scratch(lib, B, H, N, N, C, R, causal, _dtype_code(q), q.device, stream)
    if grads is None:
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        dpq = dpk = None
        if R:
            dpq = torch.empty((B, H, N, R), dtype=phi_q.dtype, device=q.device)
            dpk = torch.empty((B, H, N, R), dtype=phi_q.dtype, device=q.device)
    else:
        dq, dk, dv, dpq, dpk = grads
    st = lib.fb_lowrank_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(phi_q), _ptr(phi_k), _ptr(out),
                                 _ptr(lse), _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dpq),
                                 _ptr(dpk), B, H, N, C, R, int(bool(causal)), _dtype_code(q),
                                 phi_code, int(bool(phi_batch_broadcast)), float(scale),
                                 _ptr(workspace), workspace.numel() * workspace.element_size(),
                                 _stream(stream))
    _check(st, "fb_lowrank_attn_bwd")
    return dq, dk, dv, dpq, dpk


def fb_lowrank_attn_bwd_noalloc(q, k, v, phi_q, phi_k, out, lse, dout, grads, causal=False, scale: float = 0.0,
                                phi_batch_broadcast: Optional[bool] = None, stream=None):
    """fb_lowrank_attn_bwd on the library's static scratch: the caller passes every output tensor
    (grads = (dq, dk, dv, dphi_q, dphi_k); the last two None when R = 0 or not wanted) and this
    wrapper allocates nothing either."""
    lib = load_library()
    B, H, N, C = q.shape
    R = 0 if phi_q is None else phi_q.shape[-1]
    if phi_batch_broadcast is None:
        phi_batch_broadcast = phi_q is not None and phi_q.shape[0] == 1 and B > 1
    phi_code = _dtype_code(phi_q) if phi_q is not None else _dtype_code(q)
    dq, dk, dv, dpq, dpk = grads
    st = lib.fb_lowrank_attn_bwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(phi_q), _ptr(phi_k), _ptr(out),
                                         _ptr(lse), _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dpq),
                                         _ptr(dpk), B, H, N, C, R, int(bool(causal)), _dtype_code(q),
                                         phi_code, int(bool(phi_batch_broadcast)), float(scale),
                                         _stream(stream))
    _check(st, "fb_lowrank_attn_bwd_noalloc")
    return dq, dk, dv, dpq, dpk


def fb_lowrank_xattn_bwd(q, k, v, phi_q, phi_k, out, lse, dout, scale: float = 0.0,
                         phi_batch_broadcast: Optional[bool] = None, workspace=None, stream=None):
    """Cross-attention backward: returns dq [B,H,N,C], dk, dv [B,H,M,C], dphi_q [B,H,N,R],
    dphi_k [B,H,M,R] (None when R = 0)."""
    lib = load_library()
    B, H, N, C = q.shape
    M = k.shape[2]
    R = 0 if phi_q is None else phi_q.shape[-1]
    if phi_batch_broadcast is None:
        phi_batch_broadcast = phi_q is not None and phi_q.shape[0] == 1 and B > 1
    phi_code = _dtype_code(phi_q) if phi_q is not None else _dtype_code(q)
    if workspace is None:
        workspace = _bwd_scratch(lib, B, H, N, M, C, R, False, _dtype_code(q), q.device, stream)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    dpq = dpk = None
    if R:
        dpq = torch.empty((B, H, N, R), dtype=phi_q.dtype, device=q.device)
        dpk = torch.empty((B, H, M, R), dtype=phi_q.dtype, device=q.device)
    st = lib.fb_lowrank_xattn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(phi_q), _ptr(phi_k), _ptr(out),
                                  _ptr(lse), _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dpq),
                                  _ptr(dpk), B, H, N, M, C, R, _dtype_code(q), phi_code,
                                  int(bool(phi_batch_broadcast)), float(scale), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "fb_lowrank_xattn_bwd")
    return dq, dk, dv, dpq, dpk


def fb_dense_bias_attn_bwd_workspace_bytes(B, H, N, C, dtype_code=FB_BF16) -> int:
    return int(load_library().fb_dense_bias_attn_bwd_workspace_bytes(B, H, N, C, dtype_code))


def fb_lowrank_xattn_bwd_workspace_bytes(B, H, N, M, C, R, dtype_code=FB_BF16) -> int:
    return int(load_library().fb_lowrank_xattn_bwd_workspace_bytes(B, H, N, M, C, R, dtype_code))


def fb_dense_bias_attn_bwd(q, k, v, bias, out, lse, dout, causal=False, scale: float = 0.0,
                           bias_batch_broadcast: Optional[bool] = None, workspace=None, grads=None,
                           stream=None):
    """dq, dk, dv, dbias ([B,H,N,N], q's dtype) for the dense-bias attention."""
    lib = load_library()
    B, H, N, C = q.shape
    if bias_batch_broadcast is None:
        bias_batch_broadcast = bias.shape[0] == 1 and B > 1
    need = int(lib.fb_dense_bias_attn_bwd_workspace_bytes(B, H, N, C, _dtype_code(q)))
    if workspace is None:
        workspace = _scratch(need, q.device, stream)
    if grads is None:
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        dbias = torch.empty((B, H, N, N), dtype=q.dtype, device=q.device)
    else:
        dq, dk, dv, dbias = grads
    st = lib.fb_dense_bias_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(bias), _ptr(out), _ptr(lse),
                                    _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dbias),
                                    B, H, N, C, int(bool(causal)), _dtype_code(q),
                                    int(bool(bias_batch_broadcast)), float(scale), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "fb_dense_bias_attn_bwd")
    return dq, dk, dv, dbias


def fb_fold_batch(*grads, stream=None):
    """Sums over the batch (dimension 0, kept) of one or two contiguous gradient tensors of one dtype and
    batch size, in one launch: fp32 sums, one rounding to the tensors' dtype."""
    lib = load_library()
    if not 1 <= len(grads) <= 2:
        raise FlashBiasError("one or two tensors")
    g0 = grads[0]
    g1 = grads[1] if len(grads) == 2 else None
    shape0 = g0.shape
    B, dtype = shape0[0], _dtype_code(g0)
    o0 = g0.new_empty((1, *shape0[1:]))
    n0 = o0.numel()
    if g1 is None:
        st = lib.fb_fold_batch(_ptr(g0), o0.data_ptr(), n0, None, None, 0, B, dtype, _stream(stream))
        _check(st, "fb_fold_batch")
        return (o0,)
    shape1 = g1.shape
    if shape1[0] != B or g1.dtype != g0.dtype:
        raise FlashBiasError("the tensors must have one batch size and dtype")
    o1 = g1.new_empty((1, *shape1[1:]))
    st = lib.fb_fold_batch(_ptr(g0), o0.data_ptr(), n0, _ptr(g1), o1.data_ptr(), o1.numel(), B, dtype, _stream(stream))
    _check(st, "fb_fold_batch")
    return o0, o1


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise FlashBiasError(what)


def _here(stream, *tensors: Optional[torch.Tensor]) -> Optional[int]:
    """The stream's raw handle; all tensors of the call have to live on the current device, whose stream it is."""
    dev = tensors[0].get_device()
    if dev < 0 or dev != torch._C._cuda_getDevice():
        raise FlashBiasError("tensors must be CUDA tensors of the current device")
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise FlashBiasError("tensors must be CUDA tensors of the current device")
    return torch._C._cuda_getCurrentRawStream(dev) or None if stream is None else _stream(stream)


def _ints(name: str, t: torch.Tensor, *shape: int) -> int:
    """Address of a contiguous int32 tensor of this shape."""
    if t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous():
        raise FlashBiasError(f"{name} must be a contiguous int32 tensor of shape {shape}")
    return t.data_ptr()


def _shared_factors(phi: torch.Tensor, B: int, flag: Optional[bool]) -> bool:
    """Whether factors [B or 1, ...] are shared over the batch: their shape says so, and a flag that says otherwise is refused
    (False for one set of factors would read past it, True for B sets would use the first for every request)."""
    shared = phi.shape[0] == 1
    if flag is not None and B > 1 and bool(flag) != shared:
        raise FlashBiasError(f"phi_batch_broadcast={bool(flag)} contradicts factors of batch {phi.shape[0]} in a batch of {B}")
    return shared and B > 1


_Six = ctypes.c_longlong * 6


def _row_strides(x: torch.Tensor, y: Optional[torch.Tensor]):
    """Batch, head and row strides of one or two [B,H,N,C] tensors whose channels are adjacent."""
    xs = x.stride()
    ys = (0, 0, 0, 1) if y is None else y.stride()
    if len(xs) != 4 or len(ys) != 4 or xs[3] != 1 or ys[3] != 1:
        raise FlashBiasError("tensors must be [B,H,N,C] with adjacent channels")
    return _Six(xs[0], xs[1], xs[2], ys[0], ys[1], ys[2])


@functools.lru_cache(maxsize=64)
def _sections(sections: Tuple[int, ...]):
    """(axes, pairs, the C array) of the pairs of each axis."""
    _need(1 <= len(sections) <= 4, "one to four axes")
    return len(sections), sum(sections), (ctypes.c_int * 4)(*sections)


def _rotary(lib_fn, what, x0, x1, positions, freqs, sections, interleaved, out, stream):
    strides = _row_strides(x0, x1)
    handle = _here(stream, x0, x1, positions, freqs)
    B, H0, N, C = x0.shape
    dtype = x0.dtype
    axes, pairs, c_sections = _sections(tuple(sections))
    H1 = 0
    if x1 is not None:
        H1 = x1.shape[1]
        _need(x1.dtype is dtype and x1.shape == (B, H1, N, C), "both tensors must have one dtype, batch, length and head dimension")
    f32_pos = positions.dtype is torch.float32
    shape = positions.shape
    _need((f32_pos or positions.dtype is torch.int32) and (shape == (axes, B, N) or shape == (axes, 1, N)) and positions.is_contiguous(),
          "positions must be a contiguous int32 or float32 tensor [axes, B or 1, N]")
    _need(freqs.dtype is torch.float32 and freqs.numel() == pairs and freqs.is_contiguous(),
          "freqs must be a contiguous float32 tensor with one entry per pair")
    if out is None:
        y0 = x0.new_empty((B, H0, N, C))
        y1 = None if x1 is None else x0.new_empty((B, H1, N, C))
    else:
        y0, y1 = out
        for x, y in ((x0, y0), (x1, y1)):
            _need((x is None) == (y is None) and (x is None or (y.shape == x.shape and y.dtype is dtype and y.is_contiguous())),
                  "outputs must be contiguous, with their inputs' shapes and dtype")
        _here(stream, y0, y1)
    st = lib_fn(x0.data_ptr(), y0.data_ptr(), H0, None if x1 is None else x1.data_ptr(), None if y1 is None else y1.data_ptr(), H1,
                strides, positions.data_ptr(), f32_pos, shape[1] == 1, freqs.data_ptr(), c_sections, B, N, C, bool(interleaved),
                _dtype_code(x0), handle)
    _check(st, what)
    return y0, y1


def fb_rotary_fwd(q, k, positions, freqs, sections, interleaved: bool = False, out=None, stream=None):
    """q [B,H,N,C] and k [B,Hkv,N,C] (or None) turned by their positions: pair p by positions[axis of p] * freqs[p] radians.
    positions: [axes, B or 1, N] int32 or float32; freqs: float32, one per pair; sections: pairs of each axis, in order.
    Pairs are the channels (p, P + p), P = sum(sections), or (2p, 2p + 1) when interleaved; other channels are copied.  q and k
    may be slices of a fused projection (any strides with adjacent channels); the results are contiguous.  out: a pair of
    contiguous tensors, q and k themselves where these are contiguous."""
    return _rotary(load_library().fb_rotary_fwd, "fb_rotary_fwd", q, k, positions, freqs, sections, interleaved, out, stream)


def fb_rotary_bwd(dq, dk, positions, freqs, sections, interleaved: bool = False, out=None, stream=None):
    """The gradients of fb_rotary_fwd's q and k from those of its results (the inverse turn); same arguments."""
    return _rotary(load_library().fb_rotary_bwd, "fb_rotary_bwd", dq, dk, positions, freqs, sections, interleaved, out, stream)


def fb_paged_plan(lens, new_lens, table, ring, state, n_new: int, page: int, lens_out=None, state_out=None, slots=None,
                  positions=None, stream=None):
    """Moves B requests from lens to new_lens tokens: pages are given back and taken (table [B, max_blocks] and the ring of
    free pages, int32, in place), and the up to n_new new tokens of each are mapped.  Returns lens [B] and state [2]
    (ring head, free pages) afterwards, slots [B, n_new] (-1: no token) and positions [B, n_new]."""
    args, out = _plan_call(lens, new_lens, table, ring, state, n_new, page, lens_out, state_out, slots, positions, stream)
    _run_plan(args)
    return out


def _plan_call(lens, new_lens, table, ring, state, n_new, page, lens_out=None, state_out=None, slots=None, positions=None,
               stream=None):
    """The checked arguments of the entry point, and the tensors it writes."""
    handle = _here(stream, lens, new_lens, table, ring, state, lens_out, state_out, slots, positions)
    _need(lens.dim() == 1 and table.dim() == 2 and ring.dim() == 1, "lens, ring: one dimension, table: [B, max_blocks]")
    B, blocks, n_pages = lens.shape[0], table.shape[1], ring.shape[0]
    new = lens.new_empty
    if lens_out is None:
        lens_out = new(B)
    if state_out is None:
        state_out = new(2)
    if slots is None:
        slots = new((B, n_new))
    if positions is None:
        positions = new((B, n_new))
    return ((_ints("lens", lens, B), _ints("new_lens", new_lens, B), _ints("table", table, B, blocks), _ints("ring", ring, n_pages),
             _ints("state", state, 2), _ints("lens_out", lens_out, B), _ints("state_out", state_out, 2),
             _ints("slots", slots, B, n_new), _ints("positions", positions, B, n_new), B, n_new, page, n_pages, blocks, handle),
            (lens_out, state_out, slots, positions))


def _run_plan(args) -> None:
    _check(load_library().fb_paged_plan(*args), "fb_paged_plan")


def _check_pages(k_pages, v_pages, phi_pages, factors):
    """(n_pages, Hkv, page, C, R) of a cache and the factors that meet it."""
    shape = k_pages.shape
    _need(len(shape) == 4 and v_pages.shape == shape and v_pages.dtype is k_pages.dtype,
          "k_pages and v_pages must be [n_pages, Hkv, page, C] of one dtype")
    if factors is None:
        _need(phi_pages is None, "factors need their pages")
        return (*shape, 0)
    R = factors.shape[-1]
    _need(phi_pages is not None and phi_pages.shape == (*shape[:3], R) and phi_pages.dtype is factors.dtype,
          "phi_pages must be [n_pages, Hkv, page, R] of the factors' dtype")
    return (*shape, R)


def fb_paged_append(k, v, slots, k_pages, v_pages, phi_k=None, phi_pages=None, phi_batch_broadcast: Optional[bool] = None,
                    stream=None) -> None:
    """Stores k, v [B,Hkv,N,C] (any strides with adjacent channels) and phi_k [B or 1,Hkv,N,R] in the rows slots [B,N] of
    k_pages, v_pages [n_pages,Hkv,page,C] and phi_pages [n_pages,Hkv,page,R].  Slots of -1 are left out; the others must differ.
    phi_batch_broadcast follows from phi_k's shape; a value that contradicts it is refused."""
    lib = load_library()
    strides = _row_strides(k, v)
    shared = phi_k is not None and _shared_factors(phi_k, k.shape[0], phi_batch_broadcast)
    handle = _here(stream, k, v, slots, k_pages, v_pages, phi_k, phi_pages)
    B, Hkv, N, C = k.shape
    n_pages, hp, page, cp, R = _check_pages(k_pages, v_pages, phi_pages, phi_k)
    _need(v.shape == k.shape and k.dtype is v.dtype and k.dtype is k_pages.dtype and hp == Hkv and cp == C,
          "k, v and their pages must have one dtype, head count and head dimension")
    code = phi_code = _dtype_code(k)
    if R:
        _need(phi_k.shape == (B, Hkv, N, R) or phi_k.shape == (1, Hkv, N, R), "phi_k must be [B or 1,Hkv,N,R]")
        phi_code = _dtype_code(phi_k)
    st = lib.fb_paged_append(k.data_ptr(), v.data_ptr(), _ptr(phi_k), _ints("slots", slots, B, N), _ptr(k_pages), _ptr(v_pages),
                             _ptr(phi_pages), strides, B, Hkv, N, C, R, page, n_pages, code, phi_code, shared, handle)
    _check(st, "fb_paged_append")


@functools.lru_cache(maxsize=256)
def _paged_attn_workspace(device, B, H, Hkv, N, C, page, max_blocks, dtype_code) -> int:
    """The size query, once for each shape (it depends on the device's CU count too)."""
    return int(load_library().fb_paged_attn_fwd_workspace_bytes(B, H, Hkv, N, C, page, max_blocks, dtype_code))


def fb_paged_attn_fwd_workspace_bytes(B, H, Hkv, N, C, page, max_blocks, dtype_code=FB_BF16) -> int:
    return int(load_library().fb_paged_attn_fwd_workspace_bytes(B, H, Hkv, N, C, page, max_blocks, dtype_code))


def fb_paged_attn_fwd(q, k_pages, v_pages, table, lens, starts=None, phi_q=None, phi_pages=None, slopes=None,
                      causal: bool = True, scale: float = 0.0, out=None, lse=None,
                      phi_batch_broadcast: Optional[bool] = None, workspace=None, stream=None):
    """out, lse = attention of q [B,H,N,C], the N newest tokens of each request, over its pages: lens [B] keys each, the
    first new token at position starts[b] (None: lens - N).  k_pages, v_pages [n_pages,Hkv,page,C], H a multiple of Hkv.
    Bias: phi_q [B or 1,H,N,R] with phi_pages [n_pages,Hkv,page,R] (phi_batch_broadcast follows from phi_q's shape; a value that
    contradicts it is refused), or slopes [H] (ALiBi), or none.  causal=False: every
    query sees all keys (an encoder's states).  Queries that see nothing get out = 0, lse = -inf.  Scratch of
    fb_paged_attn_fwd_workspace_bytes: the caller's workspace, else the binding's own; a call that is given out and lse but no
    workspace allocates nothing and does without (a key head is then not split over the GPU)."""
    lib = load_library()
    shared = phi_q is not None and _shared_factors(phi_q, q.shape[0], phi_batch_broadcast)
    handle = _here(stream, q, k_pages, v_pages, table, lens, starts, phi_q, phi_pages, slopes, out, lse, workspace)
    _need(q.dim() == 4 and table.dim() == 2, "q must be [B,H,N,C], table [B, max_blocks]")
    B, H, N, C = q.shape
    blocks = table.shape[1]
    n_pages, Hkv, page, cp, R = _check_pages(k_pages, v_pages, phi_pages, phi_q)
    _need(k_pages.dtype is q.dtype and cp == C, "q and the pages must have one dtype and head dimension")
    code = phi_code = _dtype_code(q)
    if R:
        _need(phi_q.shape == (B, H, N, R) or phi_q.shape == (1, H, N, R), "phi_q must be [B or 1,H,N,R]")
        phi_code = _dtype_code(phi_q)
    if slopes is not None:
        _need(slopes.dtype is torch.float32 and slopes.numel() == H, "slopes must be a float32 tensor with one entry per head")
    ws_bytes = 0
    if workspace is not None:
        ws_bytes = workspace.numel() * workspace.element_size()
    elif out is None or lse is None:
        ws_bytes = _paged_attn_workspace(q.get_device(), B, H, Hkv, N, C, page, blocks, code)
        if ws_bytes:
            workspace = _scratch(ws_bytes, q.device, stream)
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out.shape == q.shape and out.dtype is q.dtype, "out must be like q")
    if lse is None:
        lse = q.new_empty((B, H, N), dtype=torch.float32)
    else:
        _need(lse.shape == (B, H, N) and lse.dtype is torch.float32, "lse must be [B,H,N] float32")
    st = lib.fb_paged_attn_fwd(_ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(phi_q), _ptr(phi_pages), _ptr(slopes),
                               _ints("table", table, B, blocks), _ints("lens", lens, B), None if starts is None else _ints("starts", starts, B),
                               _ptr(out), _ptr(lse), B, H, Hkv, N, C, R, page, n_pages, blocks, bool(causal), code, phi_code,
                               shared, float(scale), _ptr(workspace), ws_bytes, handle)
    _check(st, "fb_paged_attn_fwd")
    return out, lse
