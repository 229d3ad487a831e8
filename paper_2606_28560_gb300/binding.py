"""Thin ctypes binding of the C ABI in ``include/fibattn.h``.

Argument marshalling only: tensors are passed as raw device pointers with the
caller's current CUDA stream, or the torch stream given as ``stream=`` (see
``_on_stream`` for what it then does with memory); every step of the computation runs in the CUDA
library.  The binding raises ``RuntimeError`` when the library is missing or
a call returns a non-OK status -- there is no fallback.
"""
from __future__ import annotations

import array
import ctypes
import functools
import operator
import os
import threading

import numpy as np
import torch

from . import build as _build

FIBATTN_F32 = 0
FIBATTN_BF16 = 1
FIBATTN_ERR_UNSUPPORTED = 2
_STATUS = {0: "OK", 1: "INVALID_ARG", 2: "UNSUPPORTED", 3: "CUDA", 4: "INTERNAL"}

_lock = threading.Lock()
_lib = None


class FibattnError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"fibattn {_STATUS.get(status, status)}: {message}")
        self.status = status


class Opts(ctypes.Structure):
    _fields_ = [("rope_base", ctypes.c_float), ("scale", ctypes.c_float),
                ("Hkv", ctypes.c_int), ("no_dedup", ctypes.c_int), ("fwd_kernel", ctypes.c_int),
                ("bwd_kernel", ctypes.c_int), ("rotated_k", ctypes.c_void_p), ("residuals", ctypes.c_void_p),
                ("round_offsets", ctypes.c_int)]


class CacheStruct(ctypes.Structure):
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("page_stride", ctypes.c_longlong), ("row_stride", ctypes.c_longlong),
                ("head_stride", ctypes.c_longlong), ("pages", ctypes.c_int), ("page_rows", ctypes.c_int),
                ("Hkv", ctypes.c_int), ("seqs", ctypes.c_int), ("pages_per_seq", ctypes.c_int),
                ("dtype", ctypes.c_int), ("ready", ctypes.c_uint), ("phase", ctypes.c_ulonglong * 32)]


def library_path() -> str:
    return _build.LIB


def lib():
    """Load the CUDA library (it must have been built: ``__graft_entry__.build()``)."""
    global _lib
    with _lock:
        if _lib is None:
            path = _build.LIB
            if not os.path.exists(path):
                raise RuntimeError(f"CUDA library not built ({path} missing); run __graft_entry__.build()")
            L = ctypes.CDLL(path)
            vp, sz, ci, cf = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float
            fp = ctypes.POINTER(ctypes.c_float)
            ip = ctypes.POINTER(ctypes.c_int)
            op = ctypes.POINTER(Opts)
            L.fibattn_fwd_workspace_bytes.argtypes = [ci] * 7 + [op]
            L.fibattn_fwd_workspace_bytes.restype = sz
            L.fibattn_fwd.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, cf, vp, ci, ci, op, vp, sz, vp]
            L.fibattn_fwd.restype = ci
            L.fibattn_bwd_workspace_bytes.argtypes = [ci] * 7 + [op]
            L.fibattn_bwd_workspace_bytes.restype = sz
            L.fibattn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, cf, vp, ci, ci,
                                      op, vp, sz, vp]
            L.fibattn_bwd.restype = ci
            L.fibattn_last_error.argtypes = []
            L.fibattn_last_error.restype = ctypes.c_char_p
            L.fibattn_rung_params.argtypes = [cf, fp, ci, ci, ci, ci, fp, ip, fp, ip]
            L.fibattn_rung_params.restype = ci
            L.fibattn_base.argtypes = [ci, ci, fp]
            L.fibattn_base.restype = ci
            L.fibattn_alpha_schedule.argtypes = [ci, ci, fp, ci, fp]
            L.fibattn_alpha_schedule.restype = ci
            L.fibattn_theta_of_alpha.argtypes = [ci, fp, fp]
            L.fibattn_theta_of_alpha.restype = ci
            L.fibattn_residual_bytes.argtypes = [ci] * 7
            L.fibattn_residual_bytes.restype = sz
            L.fibattn_check_status.argtypes = [vp, ctypes.POINTER(ctypes.c_uint)]
            L.fibattn_check_status.restype = ci
            L.fibattn_test_wait_timeout.argtypes = [ctypes.c_uint, vp]
            L.fibattn_test_wait_timeout.restype = ci
            ll = ctypes.c_longlong
            L.fibattn_linear_xent_fwd_workspace_bytes.argtypes = [ci] * 4
            L.fibattn_linear_xent_fwd_workspace_bytes.restype = sz
            L.fibattn_linear_xent_fwd.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ll, ci, vp, sz, vp]
            L.fibattn_linear_xent_fwd.restype = ci
            L.fibattn_linear_xent_bwd_workspace_bytes.argtypes = [ci] * 4
            L.fibattn_linear_xent_bwd_workspace_bytes.restype = sz
            L.fibattn_linear_xent_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ll, ci, vp, sz, vp]
            L.fibattn_linear_xent_bwd.restype = ci
            L.fibattn_clip_grads_workspace_bytes.argtypes = [ci]
            L.fibattn_clip_grads_workspace_bytes.restype = sz
            L.fibattn_clip_grads.argtypes = [ci, vp, vp, vp, vp, cf, vp, vp, sz, vp]
            L.fibattn_clip_grads.restype = ci
            L.fibattn_cache_init.argtypes = [vp, vp, vp, ci, ci, ci, ci, ll, ll, ll, vp, ci, ci, ci, cf]
            L.fibattn_cache_init.restype = ci
            L.fibattn_cache_append.argtypes = [vp, vp, ll, ll, vp, ll, ll, vp, vp, vp, ci, vp]
            L.fibattn_cache_append.restype = ci
            L.fibattn_cached_fwd.argtypes = [vp, vp, ll, ll, vp, vp, vp, vp, ci, ci, ci, cf, vp, ci, vp, vp]
            L.fibattn_cached_fwd.restype = ci
            L.fibattn_tree_fwd.argtypes = [vp, vp, ll, ll, vp, vp, vp, vp, vp, vp, ci, ci, ci, cf, vp, ci, vp, vp]
            L.fibattn_tree_fwd.restype = ci
            _lib = L
    return _lib


def _check(rc: int):
    if rc != 0:
        raise FibattnError(rc, lib().fibattn_last_error().decode(errors="replace"))


def _fptr(a: np.ndarray):
    return a.ctypes.data_as(ctypes.POINTER(ctypes.c_float))


def _iptr(a: np.ndarray):
    return a.ctypes.data_as(ctypes.POINTER(ctypes.c_int))


FWD_KERNELS = {"auto": 0, "gather": 1, "mma": 3}
BWD_KERNELS = {"auto": 0, "gather": 1, "mma": 2}


def _opts(rope_base=1e4, scale=None, Hkv=None, dedup=True, fwd_kernel="auto", bwd_kernel="auto",
          rotated_k=None, residuals=None, round_offsets=False) -> Opts:
    return Opts(float(rope_base), float(scale) if scale else 0.0, int(Hkv or 0), 0 if dedup else 1,
                FWD_KERNELS[fwd_kernel], BWD_KERNELS[bwd_kernel],
                rotated_k.data_ptr() if rotated_k is not None else None,
                residuals.data_ptr() if residuals is not None else None, 1 if round_offsets else 0)


@functools.lru_cache(maxsize=256)
def _residual_bytes(B, H, T, W, K, bf16, D) -> int:
    return int(lib().fibattn_residual_bytes(B, H, T, D, W, K, FIBATTN_BF16 if bf16 else FIBATTN_F32))


def residual_bytes(B, H, T, W, K, dtype=torch.bfloat16, D=64) -> int:
    """Size of the forward residuals (``residuals=``); 0 for fp32 I/O."""
    return _residual_bytes(int(B), int(H), int(T), int(W), int(K), dtype == torch.bfloat16, int(D))


def residuals_like(q: torch.Tensor, W: int, K: int) -> torch.Tensor:
    """A buffer for the forward residuals of queries like q (bf16 I/O): the
    forward fills it, the backward of the same inputs reads it."""
    B, H, T, D = q.shape
    n = residual_bytes(B, H, T, W, K, q.dtype, D)
    if n == 0:
        raise ValueError("forward residuals need bf16 I/O")
    return torch.empty(n, dtype=torch.uint8, device=q.device)


def residual_views(res: torch.Tensor, B, H, T, W, K):
    """Views of a residual buffer: rotated q (bf16 [B,H,T,64]), the
    unnormalised softmax weight exp(s - max) per slot (fp32 [B,H,W+1+K,T]),
    far-minus-floor rung scores (fp32 [B,H,K,T]) and 1 / (sum of the weights)
    per query (fp32 [B,H,T]; p = weight * that); the arrays follow one another,
    each from the next multiple of 256 bytes."""
    def up(x):
        return (x + 255) // 256 * 256
    n = B * H * T
    S = W + 1 + K
    o_p = up(n * 64 * 2)
    o_sd = o_p + up(n * S * 4)
    o_il = o_sd + up(n * K * 4)
    qt = res[:n * 128].view(torch.bfloat16).view(B, H, T, 64)
    P = res[o_p:o_p + n * S * 4].view(torch.float32).view(B, H, S, T)
    sd = res[o_sd:o_sd + n * K * 4].view(torch.float32).view(B, H, K, T)
    il = res[o_il:o_il + n * 4].view(torch.float32).view(B, H, T)
    return qt, P, sd, il


def _check_residuals(res, q, W, K):
    if res is None:
        return
    B, H, T, D = q.shape
    if not (res.is_cuda and res.is_contiguous() and res.numel() * res.element_size() >=
            residual_bytes(B, H, T, W, K, q.dtype, D)):
        raise ValueError("residuals must be a contiguous CUDA buffer of residual_bytes(...) bytes")


def rotated_k_like(k: torch.Tensor) -> torch.Tensor:
    """A buffer for the rotated keys (``rotated_k=``): fp16 for bf16 k, fp32 for fp32 k."""
    return torch.empty(k.shape, dtype=torch.float16 if k.dtype == torch.bfloat16 else torch.float32,
                       device=k.device)


def _check_rotated(rk, k):
    if rk is None:
        return
    want = torch.float16 if k.dtype == torch.bfloat16 else torch.float32
    if not (rk.is_cuda and rk.is_contiguous() and rk.dtype == want and rk.shape == k.shape):
        raise ValueError(f"rotated_k must be a contiguous CUDA {want} tensor of k's shape")


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return FIBATTN_F32
    if t.dtype == torch.bfloat16:
        return FIBATTN_BF16
    raise TypeError(f"unsupported dtype {t.dtype}: fp32 or bf16")


def _check_device(index: int, *tensors):
    """The tensors (None: not given) are on device ``index`` and that is the
    current one, where the library puts its work: it cannot follow the pointers
    of another."""
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError("all tensors must be on one CUDA device")
    current = _current_device()
    if index != current:
        raise ValueError(f"the tensors are on cuda:{index} and the current device is cuda:{current}: "
                         f"make the call under torch.cuda.device({index})")


def _check_workspace(workspace, index: int):
    """Of a workspace that the caller gives; its size is checked by the library."""
    if workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous buffer on the tensors' CUDA device")


def _stream_ptr(stream) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return int(s.cuda_stream)


# The current device, and the current stream of a device by its index, without
# the looks at the state of torch.cuda and the Stream object that the calls of
# torch.cuda cost (some 4 us of every call).
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else \
    lambda index: torch.cuda.current_stream(index).cuda_stream


def _record(values, stream):
    for t in values:
        if torch.is_tensor(t):
            t.record_stream(stream)
        elif isinstance(t, PagedCache):
            _record((t.k_pages, t.v_pages, t.block_table), stream)
        elif isinstance(t, (list, tuple)):
            _record(t, stream)


def _on_stream(stream, call, *args, **kw):
    """call(*args, **kw) for a caller that gave ``stream=``, the torch stream its
    kernels are to run on: made with that stream current, so that what it allocates
    belongs to that stream and is not handed to other work while the kernels use
    it.  Given tensors are recorded with that stream, results with the caller's:
    dropping them frees nothing that the other stream still uses.  That inputs are
    ready, and results finished, is the caller's to order, as between any two
    streams."""
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream.cuda_stream))
    if stream.device_index == _current_device() and stream.cuda_stream == _raw_stream(stream.device_index):
        return call(*args, **kw)                  # it is the current one
    caller = torch.cuda.current_stream(stream.device)
    with torch.cuda.stream(stream):
        results = call(*args, **kw)
    _record(args, stream)
    _record(kw.values(), stream)
    _record(results if isinstance(results, tuple) else (results,), caller)
    return results


def _offsets(offsets) -> np.ndarray:
    if isinstance(offsets, np.ndarray) and offsets.dtype == np.float32 and offsets.flags.c_contiguous:
        return offsets
    return np.ascontiguousarray(np.asarray(offsets, dtype=np.float32))


# ------------------------------------------------------------- host prep ----

def base(kind: str, K: int) -> np.ndarray:
    f = np.zeros(K, dtype=np.float32)
    _check(lib().fibattn_base({"fib": 0, "pow2": 1}[kind], K, _fptr(f)))
    return f


def alpha_schedule(kind: str, L: int = 16, theta=None, stride: int = 7) -> np.ndarray:
    code = {"fixed": 0, "learned": 1, "linear": 2, "coprime": 3}[kind]
    out = np.zeros(L, dtype=np.float32)
    th = np.ascontiguousarray(np.asarray(theta, dtype=np.float32)) if theta is not None else None
    _check(lib().fibattn_alpha_schedule(code, L, _fptr(th) if th is not None else None, stride, _fptr(out)))
    return out


def theta_of_alpha_array(alpha) -> np.ndarray:
    """theta with 0.5 + sigmoid(theta) = alpha, per entry (fibattn_theta_of_alpha)."""
    a = np.ascontiguousarray(np.atleast_1d(np.asarray(alpha, dtype=np.float32)))
    out = np.zeros(len(a), dtype=np.float32)
    _check(lib().fibattn_theta_of_alpha(len(a), _fptr(a), _fptr(out)))
    return out


def coverage(alphas, offsets, W: int, T: int, dedup: bool = True) -> dict:
    """Distinct key distances of a layer stack (see fibattn_coverage)."""
    al = np.ascontiguousarray(np.asarray(alphas, dtype=np.float32))
    f = _offsets(offsets)
    L = lib()
    ip = ctypes.POINTER(ctypes.c_int)
    L.fibattn_coverage.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_float),
                                   ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ip, ip, ip, ip]
    L.fibattn_coverage.restype = ctypes.c_int
    per = np.zeros(len(al), dtype=np.int32)
    u, bw, hop = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check(L.fibattn_coverage(len(al), _fptr(al), _fptr(f), len(f), int(W), int(T), 0 if dedup else 1,
                              _iptr(per), ctypes.byref(u), ctypes.byref(bw), ctypes.byref(hop)))
    return dict(per_layer=per, union=u.value, beyond_window=bw.value, two_hop=hop.value)


def staging_layout(kind: str, T: int, W: int, alpha: float, offsets, dedup: bool = True) -> dict:
    """Shared-memory staging layout of the tensor-core kernels (see
    fibattn_staging_layout): kind "query" (forward, backward query pass) or
    "key" (backward key pass).  Returns the merged intervals (start, len,
    smem arrays) and slab_row per rung (-1 when not staged)."""
    f = _offsets(offsets)
    K = len(f)
    L = lib()
    ip = ctypes.POINTER(ctypes.c_int)
    L.fibattn_staging_layout.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_float,
                                         ctypes.POINTER(ctypes.c_float), ctypes.c_int, ctypes.c_int, ip, ip, ip, ip, ip]
    L.fibattn_staging_layout.restype = ctypes.c_int
    n = ctypes.c_int()
    st, ln, sm = (np.zeros(64, np.int32) for _ in range(3))
    slab = np.zeros(max(K, 1), np.int32)
    _check(L.fibattn_staging_layout({"query": 0, "key": 1}[kind], int(T), int(W), float(alpha), _fptr(f), K,
                                    0 if dedup else 1, ctypes.byref(n), _iptr(st), _iptr(ln), _iptr(sm), _iptr(slab)))
    m = n.value
    return dict(start=st[:m].copy(), len=ln[:m].copy(), smem=sm[:m].copy(), slab_row=slab[:K].copy())


def rung_params(alpha: float, offsets, W: int, dedup: bool = True, round_offsets: bool = False):
    f = _offsets(offsets)
    K = len(f)
    d = np.zeros(K, np.float32); w = np.zeros(K, np.float32)
    s0 = np.zeros(K, np.int32); act = np.zeros(K, np.int32)
    _check(lib().fibattn_rung_params(float(alpha), _fptr(f), K, int(W), 0 if dedup else 1, 1 if round_offsets else 0,
                                     _fptr(d), _iptr(s0), _fptr(w), _iptr(act)))
    return dict(d=d, s0=s0, w=w, active=act.astype(bool))


# --------------------------------------------------------------- compute ----

def fwd_workspace_bytes(B, H, T, W, K, dtype, Hkv=None, D=64) -> int:
    o = _opts(Hkv=Hkv)
    code = FIBATTN_BF16 if dtype == torch.bfloat16 else FIBATTN_F32
    return int(lib().fibattn_fwd_workspace_bytes(B, H, T, D, W, K, code, ctypes.byref(o)))


def bwd_workspace_bytes(B, H, T, W, K, dtype, Hkv=None, D=64) -> int:
    o = _opts(Hkv=Hkv)
    code = FIBATTN_BF16 if dtype == torch.bfloat16 else FIBATTN_F32
    return int(lib().fibattn_bwd_workspace_bytes(B, H, T, D, W, K, code, ctypes.byref(o)))


def fwd(q, k, v, alpha: float, offsets, W: int, *, rope_base=1e4, scale=None, dedup=True,
        out=None, lse=None, workspace=None, stream=None, kernel="auto", rotated_k=None, residuals=None,
        round_offsets=False):
    """Forward pass.  q [B,H,T,64]; k, v [B,Hkv,T,64] (fp32 or bf16, CUDA,
    contiguous).  ``kernel``: "auto", "gather" or "mma".  ``round_offsets``:
    the integer-offset variants (rung distances rounded to integers).
    ``rotated_k``: optional buffer (``rotated_k_like(k)``) that receives the
    rotated keys for a later ``bwd(..., rotated_k=...)``.  ``residuals``:
    optional buffer (``residuals_like(q, W, K)``) that receives the rotated
    queries, p of every slot and the rung score differences for a later
    ``bwd(..., residuals=...)`` (tensor-core forward only).  Returns (out, lse)."""
    if stream is not None:
        return _on_stream(stream, fwd, q, k, v, alpha, offsets, W, rope_base=rope_base, scale=scale, dedup=dedup, out=out,
                          lse=lse, workspace=workspace, kernel=kernel, rotated_k=rotated_k, residuals=residuals,
                          round_offsets=round_offsets)
    B, H, T, D = q.shape
    Hkv = k.shape[1]
    f = _offsets(offsets)
    _check_rotated(rotated_k, k)
    _check_residuals(residuals, q, W, len(f))
    o = _opts(rope_base, scale, Hkv, dedup, kernel, rotated_k=rotated_k, residuals=residuals,
              round_offsets=round_offsets)
    code = _dtype_code(q)
    for t in (q, k, v):
        if not (t.is_cuda and t.is_contiguous() and t.dtype == q.dtype):
            raise ValueError("q, k, v must be contiguous CUDA tensors of one dtype")
    _check_device(q.get_device(), k, v, out, lse, rotated_k, residuals)
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((B, H, T), dtype=torch.float32, device=q.device)
    if workspace is not None:
        _check_workspace(workspace, q.get_device())
    else:
        need = int(lib().fibattn_fwd_workspace_bytes(B, H, T, D, W, len(f), code, ctypes.byref(o)))
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    _check(lib().fibattn_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                             B, H, T, D, int(W), float(alpha), f.ctypes.data, len(f), code, ctypes.byref(o),
                             workspace.data_ptr(), workspace.numel(), _raw_stream(q.get_device())))
    return out, lse


def bwd(q, k, v, lse, dout, alpha: float, offsets, W: int, *, out=None, rope_base=1e4, scale=None, dedup=True,
        dq=None, dk=None, dv=None, dtheta=None, dd=None, workspace=None, stream=None, kernel="auto",
        rotated_k=None, rung_grads=True, residuals=None, round_offsets=False):
    """Backward pass.  ``out``: the forward output (optional; enables the
    tensor-core query pass).  ``kernel``: "auto", "gather" or "mma".
    ``rotated_k``: the buffer the forward of the same k filled (skips rotating
    k again).  ``residuals``: the buffer the forward of the same inputs filled
    (the tensor-core passes then read p, the rung score differences and the
    rotated queries instead of recomputing them).  ``rung_grads=False`` skips
    dL/dtheta and dL/dd_k (a fixed schedule; required with ``round_offsets``).
    Returns (dq, dk, dv, dtheta [1], dd [K]) on the device (dtheta, dd None
    without rung_grads)."""
    if stream is not None:
        return _on_stream(stream, bwd, q, k, v, lse, dout, alpha, offsets, W, out=out, rope_base=rope_base, scale=scale,
                          dedup=dedup, dq=dq, dk=dk, dv=dv, dtheta=dtheta, dd=dd, workspace=workspace, kernel=kernel,
                          rotated_k=rotated_k, rung_grads=rung_grads, residuals=residuals, round_offsets=round_offsets)
    B, H, T, D = q.shape
    Hkv = k.shape[1]
    f = _offsets(offsets)
    K = len(f)
    _check_rotated(rotated_k, k)
    _check_residuals(residuals, q, W, K)
    o = _opts(rope_base, scale, Hkv, dedup, bwd_kernel=kernel, rotated_k=rotated_k, residuals=residuals,
              round_offsets=round_offsets)
    code = _dtype_code(q)
    for t in (q, k, v, dout) + ((out,) if out is not None else ()):
        if not (t.is_cuda and t.is_contiguous() and t.dtype == q.dtype):
            raise ValueError("q, k, v, dout, out must be contiguous CUDA tensors of one dtype")
    _check_device(q.get_device(), k, v, lse, dout, out, dq, dk, dv, dtheta, dd, rotated_k, residuals)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    if rung_grads:
        dtheta = torch.empty(4, dtype=torch.float32, device=q.device) if dtheta is None else dtheta
        dd = torch.empty(max(K, 1), dtype=torch.float32, device=q.device) if dd is None else dd
    if workspace is not None:
        _check_workspace(workspace, q.get_device())
    else:
        need = int(lib().fibattn_bwd_workspace_bytes(B, H, T, D, W, K, code, ctypes.byref(o)))
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    _check(lib().fibattn_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr() if out is not None else None,
                             lse.data_ptr(), dout.data_ptr(),
                             dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                             dtheta.data_ptr() if dtheta is not None else None,
                             dd.data_ptr() if dd is not None else None,
                             B, H, T, D, int(W), float(alpha), f.ctypes.data, K, code, ctypes.byref(o),
                             workspace.data_ptr(), workspace.numel(), _raw_stream(q.get_device())))
    if dtheta is None and dd is None:
        return dq, dk, dv, None, None
    return dq, dk, dv, (dtheta[:1] if dtheta is not None else None), (dd[:K] if dd is not None else None)


# ------------------------------------------- loss head, gradient clipping ----

def _check_xent(x, w, targets):
    if x.dim() != 2 or w.dim() != 2 or targets.dim() != 1:
        raise ValueError("linear cross entropy takes x [N, D], w [V, D] and targets [N]")
    (N, D), (V, Dw), dtype, index = x.shape, w.shape, x.dtype, x.get_device()
    if Dw != D or targets.shape[0] != N:
        raise ValueError("linear cross entropy takes x [N, D], w [V, D] and targets [N]")
    if index < 0 or w.dtype != dtype or w.get_device() < 0 or not (x.is_contiguous() and w.is_contiguous()):
        raise ValueError("x and w must be contiguous CUDA tensors of one dtype")
    if targets.get_device() < 0 or targets.dtype != torch.int64 or not targets.is_contiguous():
        raise ValueError("targets must be a contiguous CUDA int64 tensor")
    if w.get_device() != index or targets.get_device() != index:
        raise ValueError("x, w and targets must be on one device")
    _check_device(index)
    return N, D, V, _dtype_code(x), index


def _f32_row(t, N, index, name):
    if t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != N or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous fp32 tensor of N values on x's device")
    return t


def aligned(t):
    """t, or a copy of it where it does not start on a 16-byte boundary, which the
    library asks of every tensor (a view into a longer one may not)."""
    return t if t.data_ptr() % 16 == 0 else t.clone()


def linear_xent_fwd(x, w, targets, *, ignore_index: int = -100, loss=None, lse=None, workspace=None, stream=None):
    """Cross entropy of the linear head ``x @ w.T`` without forming it in
    memory (fibattn_linear_xent_fwd).  x [N, D], w [V, D] (fp32 or bf16, CUDA,
    contiguous), targets [N] int64; rows whose target is ``ignore_index`` have
    loss 0.  Returns (loss [N], lse [N]) in fp32; ``lse`` goes to
    ``linear_xent_bwd``."""
    if stream is not None:
        return _on_stream(stream, linear_xent_fwd, x, w, targets, ignore_index=ignore_index, loss=loss, lse=lse,
                          workspace=workspace)
    N, D, V, code, index = _check_xent(x, w, targets)
    loss = torch.empty(N, dtype=torch.float32, device=x.device) if loss is None else _f32_row(loss, N, index, "loss")
    lse = torch.empty_like(loss) if lse is None else _f32_row(lse, N, index, "lse")
    L = lib()
    if workspace is not None:
        _check_workspace(workspace, index)
    else:
        need = L.fibattn_linear_xent_fwd_workspace_bytes(N, D, V, code)
        workspace = torch.empty(need or 256, dtype=torch.uint8, device=x.device)
    _check(L.fibattn_linear_xent_fwd(x.data_ptr(), w.data_ptr(), targets.data_ptr(), loss.data_ptr(), lse.data_ptr(),
                                     N, D, V, ignore_index, code, workspace.data_ptr(), workspace.numel(),
                                     _raw_stream(index)))
    return loss, lse


def linear_xent_bwd(x, w, targets, lse, dloss, *, ignore_index: int = -100, dx=None, dw=None, want_dx: bool = True,
                    want_dw: bool = True, workspace=None, stream=None):
    """Gradients of ``sum(dloss * loss)`` by x and w (fibattn_linear_xent_bwd).
    lse [N] from ``linear_xent_fwd`` of the same inputs; dloss [N] fp32 (views at
    any offset).
    Returns (dx [N, D], dw [V, D]) in x's dtype; without ``want_dx`` or
    ``want_dw`` that product is not computed and None is returned for it."""
    if stream is not None:
        return _on_stream(stream, linear_xent_bwd, x, w, targets, lse, dloss, ignore_index=ignore_index, dx=dx, dw=dw,
                          want_dx=want_dx, want_dw=want_dw, workspace=workspace)
    N, D, V, code, index = _check_xent(x, w, targets)
    lse, dloss = aligned(_f32_row(lse, N, index, "lse")), aligned(_f32_row(dloss, N, index, "dloss"))
    if not (want_dx or want_dw):
        raise ValueError("neither dx nor dw is wanted")
    dx = None if not want_dx else torch.empty_like(x) if dx is None else _grad_like(dx, x)
    dw = None if not want_dw else torch.empty_like(w) if dw is None else _grad_like(dw, w)
    L = lib()
    if workspace is not None:
        _check_workspace(workspace, index)
    else:
        need = L.fibattn_linear_xent_bwd_workspace_bytes(N, D, V, code)
        workspace = torch.empty(need or 256, dtype=torch.uint8, device=x.device)
    _check(L.fibattn_linear_xent_bwd(x.data_ptr(), w.data_ptr(), targets.data_ptr(), lse.data_ptr(), dloss.data_ptr(),
                                     dx.data_ptr() if want_dx else None, dw.data_ptr() if want_dw else None, N, D, V,
                                     ignore_index, code, workspace.data_ptr(), workspace.numel(),
                                     _raw_stream(index)))
    return dx, dw


def _grad_like(t, of):
    if t.dtype != of.dtype or t.shape != of.shape or t.get_device() != of.get_device() or not t.is_contiguous():
        raise ValueError("dx and dw must be contiguous tensors like x and w")
    return t


_dtype_of = operator.attrgetter("dtype")


def _on_device(tensors, index) -> bool:
    return set(map(torch.Tensor.get_device, tensors)) == {index} and all(map(torch.Tensor.is_contiguous, tensors))


_CLIP_CODE = {torch.float32: FIBATTN_F32, torch.bfloat16: FIBATTN_BF16}


def clip_grads(grads, max_norm: float, *, out=None, norm=None, workspace=None, stream=None):
    """Scales tensors by min(1, max_norm / (norm + 1e-6)), norm being the square
    root of the sum of the squares of all their values (fibattn_clip_grads).
    grads: contiguous CUDA tensors on one device, fp32 and bf16 in any mix, any
    offset into a buffer.  ``out``: tensors of the same sizes and dtypes, or
    None to clip in place.  Returns norm, a 0-dim fp32 tensor on the device."""
    return _clip(list(grads), float(max_norm), None if out is None else list(out), norm, workspace, stream, True)


def grad_norm(grads, *, norm=None, workspace=None, stream=None):
    """The norm alone, as ``clip_grads`` computes it; nothing else is written."""
    return _clip(list(grads), float("inf"), None, norm, workspace, stream, False)


def _clip(grads, max_norm, out, norm, workspace, stream, scale):
    if stream is not None:
        return _on_stream(stream, _clip, grads, max_norm, out, norm, workspace, None, scale)
    # (a model has hundreds of tensors: each is looked at with few calls, made by map)
    n = len(grads)
    outs = grads if out is None else out
    if len(outs) != n:
        raise ValueError("out must hold one tensor for each gradient")
    index = grads[0].get_device() if n else torch.cuda.current_device()
    dtypes = list(map(_dtype_of, grads))
    if not _CLIP_CODE.keys() >= set(dtypes):
        raise TypeError("unsupported dtype: fp32 or bf16")
    sizes = list(map(torch.Tensor.numel, grads))
    if index < 0 or n and not _on_device(grads, index):
        raise ValueError("gradients must be contiguous CUDA tensors on one device")
    if out is not None and n and (list(map(_dtype_of, outs)) != dtypes or
                                  list(map(torch.Tensor.numel, outs)) != sizes or not _on_device(outs, index)):
        raise ValueError("out must hold contiguous tensors like the gradients")
    _check_device(index)
    device = grads[0].device if n else torch.device("cuda", index)
    if norm is None:
        norm = torch.empty((), dtype=torch.float32, device=device)
    elif norm.dtype != torch.float32 or norm.numel() != 1 or norm.get_device() != index:
        raise ValueError("norm must be one fp32 value on the gradients' device")
    L = lib()
    if workspace is not None:
        _check_workspace(workspace, index)
    else:
        workspace = torch.empty(L.fibattn_clip_grads_workspace_bytes(n), dtype=torch.uint8, device=device)
    ptrs = array.array("Q", map(torch.Tensor.data_ptr, grads))
    optrs = (ptrs if out is None else array.array("Q", map(torch.Tensor.data_ptr, outs))) if scale else None
    arrays = [ptrs, optrs, array.array("q", sizes), array.array("i", map(_CLIP_CODE.__getitem__, dtypes))]
    at = [a.buffer_info()[0] if a is not None else None for a in arrays]
    _check(L.fibattn_clip_grads(n, *at, max_norm, norm.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                _raw_stream(index)))
    return norm


# ------------------------------------------ generating: the paged cache ----

class PagedCache:
    """One layer's cache of keys and values in pages (fibattn_cache_init).

    k_pages, v_pages [pages, rows of a page, Hkv, 64]: pools on one device, of the
    same shape and strides; the rotated keys in fp16 and the values in bf16, or
    both in fp32.  Any strides that are multiples of 64, the last dimension
    contiguous (a layer of a larger pool, a transposed pool with the heads first);
    they start on 32 bytes.
    block_table [seqs, pages of a sequence] int32: where the pages of each sequence
    lie; entries may change between calls, unused ones are -1 or anything else.

    The object keeps the three tensors and what follows from them; their memory is
    the caller's.  The library is told of them once: they cannot be replaced (a wider
    table, another pool: make a new cache, some 10 us), and are
    not to be given other memory (``set_``, ``resize_``).  ``PagedCache.empty`` makes
    pools."""

    _fixed = frozenset({"k_pages", "v_pages", "block_table", "rope_base", "dtype", "Hkv", "index", "device", "unit", "_struct",
                        "_at"})

    def __setattr__(self, name, value):
        if name in self._fixed:
            raise AttributeError(f"{name} of a PagedCache cannot be replaced: make a new one")
        object.__setattr__(self, name, value)

    def __delattr__(self, name):
        if name in self._fixed:
            raise AttributeError(f"{name} of a PagedCache cannot be taken out: make a new one")
        object.__delattr__(self, name)

    def __init__(self, k_pages, v_pages, block_table, *, rope_base: float = 1e4):
        if hasattr(self, "_at"):
            raise AttributeError("a PagedCache cannot be set up again: make a new one")
        if k_pages.dim() != 4 or v_pages.shape != k_pages.shape or k_pages.shape[3] != 64:
            raise ValueError("k_pages and v_pages must be [pages, rows, Hkv, 64], alike")
        want = {torch.bfloat16: torch.float16, torch.float32: torch.float32}.get(v_pages.dtype)
        if want is None or k_pages.dtype != want:
            raise TypeError("a cache holds fp16 keys and bf16 values, or both in fp32")
        index = k_pages.get_device()
        if index < 0 or v_pages.get_device() != index or block_table.get_device() != index:
            raise ValueError("the pools and block_table must be on one CUDA device")
        if block_table.dim() != 2 or block_table.dtype != torch.int32 or not block_table.is_contiguous():
            raise ValueError("block_table must be a contiguous int32 tensor [seqs, pages of a sequence]")
        if max(*k_pages.shape, *block_table.shape) > _MOST:
            raise ValueError("the sizes of the pools and of block_table must be below 2^31")
        strides = _pool_strides(k_pages)
        if strides != _pool_strides(v_pages):
            raise ValueError("k_pages and v_pages must have the same strides")
        pages, rows, heads, D = k_pages.shape
        struct = CacheStruct()
        at = ctypes.addressof(struct)
        _check(lib().fibattn_cache_init(at, k_pages.data_ptr(), v_pages.data_ptr(), pages, rows, heads, D, *strides,
                                        block_table.data_ptr(), *block_table.shape, _dtype_code(v_pages), float(rope_base)))
        put = object.__setattr__                               # (past the refusal above)
        put(self, "k_pages", k_pages)
        put(self, "v_pages", v_pages)
        put(self, "block_table", block_table)
        put(self, "rope_base", float(rope_base) or 1e4)        # (0: the library's own)
        put(self, "dtype", v_pages.dtype)
        put(self, "Hkv", heads)
        put(self, "index", index)
        put(self, "device", k_pages.device)
        put(self, "unit", 16 // v_pages.element_size())        # strides of tokens are multiples of this
        put(self, "_struct", struct)
        put(self, "_at", at)

    @classmethod
    def empty(cls, pages: int, rows: int, Hkv: int, block_table, *, dtype=torch.bfloat16, rope_base: float = 1e4):
        """A cache over new pools on block_table's device, for tensors of ``dtype``."""
        if dtype not in (torch.bfloat16, torch.float32):
            raise TypeError(f"unsupported dtype {dtype}: fp32 or bf16")
        shape = (pages, rows, Hkv, 64)
        keys = torch.float16 if dtype == torch.bfloat16 else torch.float32
        return cls(torch.empty(shape, dtype=keys, device=block_table.device),
                   torch.empty(shape, dtype=dtype, device=block_table.device), block_table, rope_base=rope_base)


def _pool_strides(t):
    """Strides of a pool's first three dimensions; that of a dimension of one is of no matter."""
    if t.shape[3] > 1 and t.stride(3) != 1:
        raise ValueError("the last dimension of a pool must be contiguous")
    return tuple(64 if n == 1 else s for n, s in zip(t.shape[:3], t.stride()))


_MOST = 2 ** 31 - 1                     # of an int of the library: ctypes would cut a larger one short


def _tokens(t, cache, name):
    """(pointer, token stride, head stride) of tokens [N, heads, 64] as the library takes them."""
    shape = t.shape
    if len(shape) != 3 or shape[2] != 64 or t.dtype is not cache.dtype or t.get_device() != cache.index:
        raise ValueError(f"{name} must be [tokens, heads, 64] of the cache's dtype, on its device")
    token, head, last = t.stride()
    if shape[0] == 1:
        token = 0
    if shape[1] == 1:
        head = 0
    if last != 1 or token % cache.unit or head % cache.unit:
        raise ValueError(f"{name} must be contiguous in its last dimension, with strides of whole 16 bytes")
    return t.data_ptr(), token, head


def _ints(t, shape, index, name):
    """The pointer of a tensor with one int32 per token."""
    if t is None or t.dtype is not torch.int32 or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor of {shape[0]} values on the cache's device")
    return t.data_ptr()


# What the library reads on the host at a call on the cache, by value: finding a few
# numbers again takes a fraction of the time of handing them over anew.
_offset_tables, _opt_structs = {}, {}


def _offset_table(offsets):
    """(address of the offsets as floats, how many, what has to live meanwhile)"""
    f = _offsets(offsets)
    key = f.tobytes()
    got = _offset_tables.get(key)
    if got is None:
        if len(_offset_tables) > 255:
            _offset_tables.clear()
        f = f.copy()
        got = _offset_tables[key] = f.ctypes.data, f.size, f
    return got


def _opt_struct(scale, dedup, round_offsets):
    """(address of the options, or None for the library's own; what has to live meanwhile)"""
    if scale is None and dedup and not round_offsets:
        return None, None
    key = scale if scale is None else float(scale), bool(dedup), bool(round_offsets)
    got = _opt_structs.get(key)
    if got is None:
        if len(_opt_structs) > 255:
            _opt_structs.clear()
        o = _opts(0.0, scale, 0, dedup, round_offsets=round_offsets)
        got = _opt_structs[key] = ctypes.addressof(o), o
    return got


def cache_append(cache: PagedCache, k, v, positions, *, seqs=None, slots=None, stream=None):
    """Writes the keys and values of N tokens into the cache, the keys rotated on
    the way (fibattn_cache_append).  k, v [N, Hkv, 64]: views of a fused projection
    will do.  positions [N] int32: where each token stands; seqs [N] int32: whose
    it is (default: token n is sequence n's); slots [N] int32: where it is stored
    (default: at its position; drafted tokens lie elsewhere); two tokens of one call at
    one slot leave a mixture there.  A negative position or sequence is padding.
    Nothing is returned."""
    if stream is not None:
        return _on_stream(stream, cache_append, cache, k, v, positions, seqs=seqs, slots=slots)
    index, shape = cache.index, k.shape
    k_at, v_at = _tokens(k, cache, "k"), _tokens(v, cache, "v")
    if v.shape != shape or shape[1] != cache.Hkv:
        raise ValueError("k and v must be [tokens, the cache's Hkv, 64]")
    each, N = shape[:1], shape[0]
    if N > _MOST:
        raise ValueError("tokens times heads must be below 2^31")
    p = _ints(positions, each, index, "positions")
    b = None if seqs is None else _ints(seqs, each, index, "seqs")
    at = None if slots is None else _ints(slots, each, index, "slots")
    _check_device(index)
    rc = lib().fibattn_cache_append(cache._at, *k_at, *v_at, p, at, b, N, _raw_stream(index))
    if rc:
        _check(rc)


def cached_fwd(q, cache: PagedCache, alpha: float, offsets, W: int, positions, *, seqs=None, scale=None, dedup=True,
               round_offsets=False, out=None, lse=None, stream=None):
    """Attention of N tokens over the cache (fibattn_cached_fwd): ``fwd``'s window
    and rungs, read from the pages.  q [N, H, 64] (views of a fused projection will
    do), positions and seqs as for ``cache_append``; the tokens' own keys and values
    have to be in the cache.  One token per sequence, chunks of a prompt, or any mix.
    Returns (out [N, H, 64], lse [N, H] fp32), without gradients; padding has out 0 and
    lse -infinity.  A token has the same bits in whatever batch it is."""
    if stream is not None:
        return _on_stream(stream, cached_fwd, q, cache, alpha, offsets, W, positions, seqs=seqs, scale=scale, dedup=dedup,
                          round_offsets=round_offsets, out=out, lse=lse)
    return _attention(q, cache, alpha, offsets, W, positions, None, None, seqs, scale, dedup, round_offsets, out, lse)


def tree_fwd(q, cache: PagedCache, alpha: float, offsets, W: int, positions, parents, slots, *, seqs=None, scale=None,
             dedup=True, round_offsets=False, out=None, lse=None, stream=None):
    """Attention of drafted tokens that form trees (fibattn_tree_fwd): a token sees
    its ancestors in place of the positions they stand at, and the cached sequence
    behind the root.  parents [N] int32: the row of this batch, before n, that token
    n continues, or -1 (a parent is of its child's sequence, its position one less);
    slots [N] int32: where ``cache_append`` put each token.  The rest as for
    ``cached_fwd``.  Accepted tokens are appended again, at their positions."""
    if stream is not None:
        return _on_stream(stream, tree_fwd, q, cache, alpha, offsets, W, positions, parents, slots, seqs=seqs, scale=scale,
                          dedup=dedup, round_offsets=round_offsets, out=out, lse=lse)
    if parents is None or slots is None:
        raise ValueError("a tree needs parents and slots")
    return _attention(q, cache, alpha, offsets, W, positions, parents, slots, seqs, scale, dedup, round_offsets, out, lse)


def _attention(q, cache, alpha, offsets, W, positions, parents, slots, seqs, scale, dedup, round_offsets, out, lse):
    at, index, shape = _tokens(q, cache, "q"), cache.index, q.shape
    each, N, H = shape[:1], shape[0], shape[1]
    if N * H > _MOST:
        raise ValueError("tokens times heads must be below 2^31")
    p = _ints(positions, each, index, "positions")
    b = None if seqs is None else _ints(seqs, each, index, "seqs")
    _check_device(index)
    W = int(W)
    if not -_MOST <= W <= _MOST:
        raise ValueError(f"W must be in [0, 1024] (got {W})")
    f, K, alive = _offset_table(offsets)              # noqa: F841 (alive, kept: until the call is over)
    o, kept = _opt_struct(scale, dedup, round_offsets)   # noqa: F841
    if out is None:
        out = torch.empty(shape, dtype=cache.dtype, device=cache.device)
    elif out.dtype is not cache.dtype or out.shape != shape or out.get_device() != index or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor of q's shape and dtype on its device")
    if lse is None:
        lse = torch.empty((N, H), dtype=torch.float32, device=cache.device)
    elif lse.dtype is not torch.float32 or lse.shape != (N, H) or lse.get_device() != index or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous fp32 tensor [N, H] on q's device")
    if parents is None:
        rc = lib().fibattn_cached_fwd(cache._at, *at, out.data_ptr(), lse.data_ptr(), p, b, N, H, W, float(alpha), f, K,
                                      o, _raw_stream(index))
    else:
        rc = lib().fibattn_tree_fwd(cache._at, *at, out.data_ptr(), lse.data_ptr(), p, _ints(parents, each, index, "parents"),
                                    _ints(slots, each, index, "slots"), b, N, H, W, float(alpha), f, K, o,
                                    _raw_stream(index))
    if rc:
        _check(rc)
    return out, lse


# ---------------------------------------------------------- device status ----

def check_status(stream=None):
    """Synchronise ``stream`` and read and clear the device status word
    (fibattn_check_status).  Returns the flags; raises FibattnError when a
    kernel gave up a bounded wait (status 4), a rotated row overflowed fp16, a
    cross-entropy target was outside the vocabulary or a token named a part of a
    cache that does not exist (status 5)."""
    flags = ctypes.c_uint(0)
    rc = lib().fibattn_check_status(_stream_ptr(stream), ctypes.byref(flags))
    if rc != 0:
        e = FibattnError(rc, lib().fibattn_last_error().decode(errors="replace"))
        e.flags = flags.value
        raise e
    return flags.value


def test_wait_timeout(timeout_us: int, stream=None):
    """Launch the library's bounded-wait probe (a wait that no copy completes)."""
    _check(lib().fibattn_test_wait_timeout(int(timeout_us), _stream_ptr(stream)))


# ------------------------------------------------------------- profiling ----

def profile_enable(on: bool = True):
    L = lib()
    L.fibattn_profile_enable.argtypes = [ctypes.c_int]
    L.fibattn_profile_enable.restype = ctypes.c_int
    _check(L.fibattn_profile_enable(1 if on else 0))


def profile_summary() -> dict:
    """{kernel name: (total device ms, launches)} for launches since enable."""
    L = lib()
    L.fibattn_profile_summary.argtypes = [ctypes.c_int, ctypes.c_char_p, ctypes.c_int,
                                          ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int)]
    L.fibattn_profile_summary.restype = ctypes.c_int
    n = L.fibattn_profile_summary(-1, None, 0, None, None)
    out = {}
    for i in range(n):
        buf = ctypes.create_string_buffer(64)
        ms = ctypes.c_double()
        cnt = ctypes.c_int()
        _check(L.fibattn_profile_summary(i, buf, 64, ctypes.byref(ms), ctypes.byref(cnt)))
        out[buf.value.decode()] = (ms.value, cnt.value)
    return out
