"""Python binding of libfem.so (argument marshalling only).

Every function here checks shapes, dtypes and devices of torch tensors,
passes raw pointers and sizes to the C ABI of ``include/fem.h`` and raises on
a non-zero status.  All arithmetic of the read runs in the library's CUDA
kernels; there is no other implementation behind these names.  If the
library is not built, ``load()`` raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading
import types

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libfem.so")
_lock = threading.Lock()
_lib = None

STATUS = {0: "FEM_OK", 1: "FEM_ERR_INVALID_ARG", 2: "FEM_ERR_UNSUPPORTED", 3: "FEM_ERR_CUDA",
          4: "FEM_ERR_TIMEOUT", 5: "FEM_ERR_NO_MEMORY"}

EXPORTS = ["fem_fwd", "fem_fwd_ws", "fem_fwd_workspace_bytes", "fem_fwd_f32", "fem_fwd_host",
           "fem_check_device_error", "fem_last_fixup_rows", "fem_set_kernel_events", "fem_status_str",
           "fem_fwd_noalloc", "fem_fwd_gated", "fem_decode", "fem_gla_fwd", "fem_tdc_conv", "fem_bwd_f32",
           "fem_probe_wait_timeout", "fem_attn_fwd", "fem_gla_fwd_tc", "fem_cache_write", "fem_cache_gather",
           "fem_paged_read", "fem_rope_turns", "fem_rope", "fem_recur_fwd", "fem_recur_bwd", "fem_norm_fwd", "fem_norm_bwd"]


class FemError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} returned {STATUS.get(status, status)}")
        self.status = status


def library_path() -> str:
    return _LIB_PATH


def load(path: str | None = None):
    """Load libfem.so (built by ``paper_2602_07160_gb300.build``) and bind its ABI."""
    global _lib
    with _lock:
        if _lib is not None and path is None:
            return _lib
        p = path or _LIB_PATH
        if not os.path.exists(p):
            raise RuntimeError(f"{p} is not built; run `python -m paper_2602_07160_gb300.build`")
        lib = ctypes.CDLL(p)
        vp, i, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        sig = [vp, vp, vp, vp, vp, vp, i, i, i, i, i]
        lib.fem_fwd.argtypes = sig + [vp]
        lib.fem_fwd_ws.argtypes = sig + [vp, sz, vp]
        lib.fem_fwd_f32.argtypes = sig + [vp]
        lib.fem_fwd_host.argtypes = sig + [vp]
        lib.fem_fwd_noalloc.argtypes = sig + [vp]
        lib.fem_fwd_noalloc.restype = i
        lib.fem_fwd_gated.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, vp]
        lib.fem_fwd_gated.restype = i
        lib.fem_decode.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, vp]
        lib.fem_decode.restype = i
        lib.fem_gla_fwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, vp]
        lib.fem_gla_fwd.restype = i
        lib.fem_gla_fwd_tc.argtypes = [vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, vp]
        lib.fem_gla_fwd_tc.restype = i
        lib.fem_tdc_conv.argtypes = [vp, vp, vp, i, i, i, vp]
        lib.fem_tdc_conv.restype = i
        lib.fem_bwd_f32.argtypes = [vp] * 11 + [i, i, i, i, i, vp]
        lib.fem_bwd_f32.restype = i
        i64 = ctypes.c_int64
        lib.fem_cache_write.argtypes = [vp, vp, vp, i64, i64, i64, i64, vp, i, vp]
        lib.fem_cache_write.restype = i
        lib.fem_cache_gather.argtypes = [vp, vp, i, vp, vp, i, vp, vp, i, vp]
        lib.fem_cache_gather.restype = i
        lib.fem_paged_read.argtypes = [vp, vp, i64, i64, vp, vp, vp, vp, i, i, i, i, i, i, vp, vp, vp]
        lib.fem_paged_read.restype = i
        f32, f64 = ctypes.c_float, ctypes.c_double
        lib.fem_rope_turns.argtypes = [i, f64, i, f64, f64, f64, f64, vp]
        lib.fem_rope_turns.restype = i
        lib.fem_rope.argtypes = [vp, vp, i, vp, vp, i, i, i, i, i, vp, i, i, f32, vp, i, vp]
        lib.fem_rope.restype = i
        lib.fem_recur_fwd.argtypes = [vp, vp, i64, i64, vp, i, i, i, i, i, i, vp, vp, vp, i, vp, i64, vp]
        lib.fem_recur_fwd.restype = i
        lib.fem_recur_bwd.argtypes = [vp] * 4 + [i64] * 4 + [vp] + [i] * 6 + [vp] * 4 + [i64] * 2 + [vp] * 2
        lib.fem_recur_bwd.restype = i
        lib.fem_norm_fwd.argtypes = [vp] * 7
        lib.fem_norm_fwd.restype = i
        lib.fem_norm_bwd.argtypes = [vp] * 14
        lib.fem_norm_bwd.restype = i
        lib.fem_fwd_workspace_bytes.argtypes = [i, i, i, i, i]
        lib.fem_fwd_workspace_bytes.restype = sz
        lib.fem_check_device_error.argtypes = [vp]
        lib.fem_attn_fwd.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, vp]
        lib.fem_attn_fwd.restype = i
        lib.fem_probe_wait_timeout.argtypes = [ctypes.c_uint, vp]
        lib.fem_probe_wait_timeout.restype = i
        lib.fem_last_fixup_rows.argtypes = [vp]
        lib.fem_set_kernel_events.argtypes = [vp, vp]
        lib.fem_set_kernel_events.restype = i
        lib.fem_status_str.argtypes = [i]
        lib.fem_status_str.restype = ctypes.c_char_p
        for name in ("fem_fwd", "fem_fwd_ws", "fem_fwd_f32", "fem_fwd_host", "fem_check_device_error",
                     "fem_last_fixup_rows"):
            getattr(lib, name).restype = i
        if path is None:
            _lib = lib
        return lib


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream, device):
    if stream is None:
        stream = torch.cuda.current_stream(device)
    return ctypes.c_void_p(stream.cuda_stream)


def _check_qkvb(q, k, v, beta, dtype, device_type):
    if q.dim() != 4 or k.shape != q.shape or v.shape != q.shape:
        raise ValueError("q, k, v must share the shape [B, H, T, d]")
    B, H, T, d = q.shape
    if beta.shape != (H, d) or beta.dtype != torch.float32:
        raise ValueError("beta must be float32 [H, d]")
    for name, t in (("q", q), ("k", k), ("v", v), ("beta", beta)):
        if t.dtype != (torch.float32 if name == "beta" else dtype):
            raise ValueError(f"{name} has dtype {t.dtype}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if t.device.type != device_type:
            raise ValueError(f"{name} must be on {device_type}")
    return B, H, T, d


def _outputs(q, out, lse, device):
    B, H, T, d = q.shape
    if out is None:
        out = torch.empty((B, H, T, d), dtype=torch.float32, device=device)
    if lse is None:
        lse = torch.empty((B, H, T), dtype=torch.float32, device=device)
    if out.shape != (B, H, T, d) or out.dtype != torch.float32 or not out.is_contiguous():
        raise ValueError("out must be contiguous float32 [B, H, T, d]")
    if lse is not False and (lse.shape != (B, H, T) or lse.dtype != torch.float32 or not lse.is_contiguous()):
        raise ValueError("lse must be contiguous float32 [B, H, T]")
    return out, lse


def fem_fwd(q, k, v, beta, causal: bool = True, out=None, lse=None, stream=None):
    """The read on bf16 CUDA tensors (tensor-core path).  Returns (out, lse).

    Pass ``lse=False`` to skip the log-normaliser output."""
    B, H, T, d = _check_qkvb(q, k, v, beta, torch.bfloat16, "cuda")
    out, lse = _outputs(q, out, lse, q.device)
    rc = load().fem_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(out), None if lse is False else _ptr(lse),
                        B, H, T, d, int(bool(causal)), _stream(stream, q.device))
    if rc != 0:
        raise FemError("fem_fwd", rc)
    return out, (None if lse is False else lse)


def fem_attn_fwd(q, k, v, causal: bool = True, out=None, lse=None, stream=None):
    """Plain softmax attention on the same tensor-core kernel (the comparator; bf16 CUDA
    tensors).  Returns (out, lse)."""
    beta = torch.zeros((q.shape[1], q.shape[3]), dtype=torch.float32, device=q.device)  # shape check only
    B, H, T, d = _check_qkvb(q, k, v, beta, torch.bfloat16, "cuda")
    out, lse = _outputs(q, out, lse, q.device)
    rc = load().fem_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(out), None if lse is False else _ptr(lse),
                             B, H, T, d, int(bool(causal)), _stream(stream, q.device))
    if rc != 0:
        raise FemError("fem_attn_fwd", rc)
    return out, (None if lse is False else lse)


def workspace_bytes(B: int, H: int, T: int, d: int, causal: bool = True) -> int:
    return int(load().fem_fwd_workspace_bytes(B, H, T, d, int(bool(causal))))


def fem_fwd_ws(q, k, v, beta, workspace, causal: bool = True, out=None, lse=None, stream=None):
    """fem_fwd with a caller-owned uint8 CUDA workspace of ``workspace_bytes()`` bytes."""
    B, H, T, d = _check_qkvb(q, k, v, beta, torch.bfloat16, "cuda")
    out, lse = _outputs(q, out, lse, q.device)
    rc = load().fem_fwd_ws(_ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(out), None if lse is False else _ptr(lse),
                           B, H, T, d, int(bool(causal)), _ptr(workspace), workspace.numel() * workspace.element_size(),
                           _stream(stream, q.device))
    if rc != 0:
        raise FemError("fem_fwd_ws", rc)
    return out, (None if lse is False else lse)


def fem_fwd_gated(q, k, v, beta_max, lam, gate, causal: bool = True, out=None, lse=None, stream=None):
    """The two-level gated read on bf16 CUDA tensors: out = gate * ((1 - lam) mu + lam Fmax).

    lam and gate are float32 [B, H, T, d] (already activated); beta_max is float32 [H, d].
    Returns (out, lse)."""
    B, H, T, d = _check_qkvb(q, k, v, beta_max, torch.bfloat16, "cuda")
    for name, t in (("lam", lam), ("gate", gate)):
        if t.shape != q.shape or t.dtype != torch.float32 or not t.is_contiguous() or t.device != q.device:
            raise ValueError(f"{name} must be a contiguous float32 tensor shaped like q on its device")
    out, lse = _outputs(q, out, lse, q.device)
    rc = load().fem_fwd_gated(_ptr(q), _ptr(k), _ptr(v), _ptr(beta_max), _ptr(lam), _ptr(gate), _ptr(out),
                              None if lse is False else _ptr(lse), B, H, T, d, int(bool(causal)),
                              _stream(stream, q.device))
    if rc != 0:
        raise FemError("fem_fwd_gated", rc)
    return out, (None if lse is False else lse)


def fem_decode(q, k, v, beta, out=None, lse=None, stream=None):
    """Decode read on bf16 CUDA tensors: q [B, H, d] against the cache k, v [B, H, T, d].

    Returns (out [B, H, d] float32, lse [B, H] float32)."""
    if q.dim() != 3 or k.dim() != 4 or k.shape != v.shape or k.shape[:2] != q.shape[:2] or k.shape[3] != q.shape[2]:
        raise ValueError("q must be [B, H, d] and k, v [B, H, T, d]")
    B, H, T, d = k.shape
    for name, t in (("q", q), ("k", k), ("v", v)):
        if t.dtype != torch.bfloat16 or not t.is_contiguous() or t.device.type != "cuda":
            raise ValueError(f"{name} must be a contiguous bf16 CUDA tensor")
    if beta.shape != (H, d) or beta.dtype != torch.float32 or not beta.is_contiguous() or beta.device != q.device:
        raise ValueError("beta must be float32 [H, d] on q's device")
    if out is None:
        out = torch.empty((B, H, d), dtype=torch.float32, device=q.device)
    if lse is None:
        lse = torch.empty((B, H), dtype=torch.float32, device=q.device)
    rc = load().fem_decode(_ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(out), None if lse is False else _ptr(lse),
                           B, H, T, d, _stream(stream, q.device))
    if rc != 0:
        raise FemError("fem_decode", rc)
    return out, (None if lse is False else lse)


def fem_gla_fwd_tc(qf, kf, v, logdecay, beta, out=None, logz=None, stream=None):
    """fem_gla_fwd chunked on the tensor cores (m = d = 64; bf16 operands, fp32 state)."""
    return fem_gla_fwd(qf, kf, v, logdecay, beta, out=out, logz=logz, stream=stream, _entry="fem_gla_fwd_tc")


def fem_gla_fwd(qf, kf, v, logdecay, beta, out=None, logz=None, stream=None, _entry="fem_gla_fwd"):
    """The read over a GLA prior on fp32 CUDA tensors.

    qf, kf: [B, H, T, m] nonnegative features; v: [B, H, T, d]; logdecay: [B, H, T] (<= 0);
    beta: [H, d].  Returns (out [B, H, T, d], logz [B, H, T])."""
    if qf.dim() != 4 or kf.shape != qf.shape or v.dim() != 4 or v.shape[:3] != qf.shape[:3]:
        raise ValueError("qf, kf must be [B, H, T, m] and v [B, H, T, d]")
    B, H, T, m = qf.shape
    d = v.shape[3]
    for name, t in (("qf", qf), ("kf", kf), ("v", v), ("logdecay", logdecay), ("beta", beta)):
        if t.dtype != torch.float32 or not t.is_contiguous() or t.device != qf.device or t.device.type != "cuda":
            raise ValueError(f"{name} must be a contiguous float32 CUDA tensor on qf's device")
    if logdecay.shape != (B, H, T) or beta.shape != (H, d):
        raise ValueError("logdecay must be [B, H, T] and beta [H, d]")
    if out is None:
        out = torch.empty((B, H, T, d), dtype=torch.float32, device=qf.device)
    if logz is None:
        logz = torch.empty((B, H, T), dtype=torch.float32, device=qf.device)
    rc = getattr(load(), _entry)(_ptr(qf), _ptr(kf), _ptr(v), _ptr(logdecay), _ptr(beta), _ptr(out),
                                 None if logz is False else _ptr(logz), B, H, T, m, d, _stream(stream, qf.device))
    if rc != 0:
        raise FemError(_entry, rc)
    return out, (None if logz is False else logz)


def fem_tdc_conv(s, u, out=None, stream=None):
    """The time-decay conditioner's convolution h_t = exp(-s_t) h_{t-1} + u_t on fp32
    CUDA tensors s, u of shape [B, T, Hc] (s >= 0).  Returns h."""
    if s.dim() != 3 or u.shape != s.shape:
        raise ValueError("s and u must share the shape [B, T, Hc]")
    for name, t in (("s", s), ("u", u)):
        if t.dtype != torch.float32 or not t.is_contiguous() or t.device.type != "cuda" or t.device != s.device:
            raise ValueError(f"{name} must be a contiguous float32 CUDA tensor on s's device")
    B, T, Hc = s.shape
    _sizes("fem_tdc_conv", B, T, Hc)
    if out is None:
        out = torch.empty_like(s)
    rc = load().fem_tdc_conv(_ptr(s), _ptr(u), _ptr(out), B, T, Hc, _stream(stream, s.device))
    if rc != 0:
        raise FemError("fem_tdc_conv", rc)
    return out


def fem_bwd_f32(q, k, v, beta, out, lse, dout, causal: bool = True, stream=None):
    """Gradients of the fp32 read from its saved (out, lse) and the output cotangent dout.

    Returns (dq, dk, dv [B, H, T, d], dbeta [H, d] summed over batch and time)."""
    B, H, T, d = _check_qkvb(q, k, v, beta, torch.float32, "cuda")
    for name, t, shape in (("out", out, q.shape), ("dout", dout, q.shape), ("lse", lse, q.shape[:3])):
        if t.shape != shape or t.dtype != torch.float32 or not t.is_contiguous() or t.device != q.device:
            raise ValueError(f"{name} must be a contiguous float32 tensor of shape {tuple(shape)} on q's device")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    dbeta = torch.empty_like(beta)
    rc = load().fem_bwd_f32(_ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(out), _ptr(lse), _ptr(dout), _ptr(dq),
                            _ptr(dk), _ptr(dv), _ptr(dbeta), B, H, T, d, int(bool(causal)), _stream(stream, q.device))
    if rc != 0:
        raise FemError("fem_bwd_f32", rc)
    return dq, dk, dv, dbeta


def fem_fwd_f32(q, k, v, beta, causal: bool = True, out=None, lse=None, stream=None):
    """The read on fp32 CUDA tensors (CUDA-core path).  Returns (out, lse)."""
    B, H, T, d = _check_qkvb(q, k, v, beta, torch.float32, "cuda")
    out, lse = _outputs(q, out, lse, q.device)
    rc = load().fem_fwd_f32(_ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(out), None if lse is False else _ptr(lse),
                            B, H, T, d, int(bool(causal)), _stream(stream, q.device))
    if rc != 0:
        raise FemError("fem_fwd_f32", rc)
    return out, (None if lse is False else lse)


def fem_fwd_host(q, k, v, beta, causal: bool = True, out=None, lse=None, stream=None, device=None):
    """The read on HOST (ideally pinned) bf16 tensors: copies in, computes, copies out."""
    B, H, T, d = _check_qkvb(q, k, v, beta, torch.bfloat16, "cpu")
    # outputs it allocates are pinned: copies into pageable memory do not overlap the read
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32).pin_memory()
    if lse is None:
        lse = torch.empty(q.shape[:3], dtype=torch.float32).pin_memory()
    out, lse = _outputs(q, out, lse, "cpu")
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    rc = load().fem_fwd_host(_ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(out), None if lse is False else _ptr(lse),
                             B, H, T, d, int(bool(causal)), _stream(stream, dev))
    if rc != 0:
        raise FemError("fem_fwd_host", rc)
    return out, (None if lse is False else lse)


def fem_fwd_noalloc(q, k, v, beta, causal: bool = True, out=None, lse=None, stream=None):
    """fem_fwd without device allocation (the library's fixed 16 MiB scratch).

    For callers that may not allocate device memory during the read.  ``out``
    and ``lse`` should be passed preallocated by such callers.  Calls that
    overlap on the GPU share the scratch and race."""
    B, H, T, d = _check_qkvb(q, k, v, beta, torch.bfloat16, "cuda")
    out, lse = _outputs(q, out, lse, q.device)
    rc = load().fem_fwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(out),
                                None if lse is False else _ptr(lse), B, H, T, d, int(bool(causal)),
                                _stream(stream, q.device))
    if rc != 0:
        raise FemError("fem_fwd_noalloc", rc)
    return out, (None if lse is False else lse)


class _CacheStruct(ctypes.Structure):
    """fem_paged_cache of include/fem.h."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
                ("format", ctypes.c_int), ("num_pages", ctypes.c_int), ("H", ctypes.c_int), ("page_size", ctypes.c_int),
                ("d", ctypes.c_int)]


class PagedCache:
    """A paged key/value cache: k, v [num_pages, H, page_size, d] on one CUDA device.

    bf16 and float32 caches are the two tensors; float8_e4m3fn ones have the rows' scale
    exponents k_exp, v_exp (uint8 [num_pages, H, page_size]) beside them.  The object keeps
    the tensors, checks them once, and is what ``fem_cache_write``, ``fem_cache_gather`` and
    ``fem_paged_read`` take.  Those run on the cache's device, which has to be the current one."""

    FORMATS = {torch.bfloat16: 0, torch.float8_e4m3fn: 1, torch.float32: 2}

    def __init__(self, k, v, k_exp=None, v_exp=None):
        if k.dim() != 4 or v.shape != k.shape or v.dtype != k.dtype or v.device != k.device:
            raise ValueError("k and v must share the shape [num_pages, H, page_size, d], type and device")
        if k.dtype not in self.FORMATS:
            raise ValueError(f"a cache of {k.dtype} is not supported")
        pages, H, page_size, d = k.shape
        scaled = k.dtype == torch.float8_e4m3fn
        if scaled != (k_exp is not None) or scaled != (v_exp is not None):
            raise ValueError("k_exp and v_exp go with float8_e4m3fn caches, and only with them")
        for name, t in (("k", k), ("v", v)) + ((("k_exp", k_exp), ("v_exp", v_exp)) if scaled else ()):
            if not t.is_contiguous() or t.device.type != "cuda" or t.device != k.device:
                raise ValueError(f"{name} must be a contiguous CUDA tensor on k's device")
            if name.endswith("exp") and (t.dtype != torch.uint8 or t.shape != (pages, H, page_size)):
                raise ValueError(f"{name} must be uint8 [num_pages, H, page_size]")
        if page_size not in (16, 32, 64, 128, 256) or d % 16 or not 16 <= d <= 256 or pages < 1 or H < 1:
            raise ValueError("page_size must be 16, 32, 64, 128 or 256 and d a multiple of 16 up to 256")
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        self.num_pages, self.H, self.page_size, self.d = pages, H, page_size, d
        self.device, self.index = k.device, k.get_device()
        self.row_dtype = torch.float32 if k.dtype == torch.float32 else torch.bfloat16  # of k, v, q given to the calls
        self._struct = _CacheStruct(k.data_ptr(), v.data_ptr(), k_exp.data_ptr() if scaled else None,
                                    v_exp.data_ptr() if scaled else None, self.FORMATS[k.dtype], pages, H, page_size, d)
        self._ref = ctypes.addressof(self._struct)

    @classmethod
    def empty(cls, num_pages: int, H: int, d: int, page_size: int = 64, dtype=torch.bfloat16, device="cuda"):
        """A cache of zeros."""
        shape = (num_pages, H, page_size, d)
        k, v = (torch.zeros(shape, dtype=torch.uint8 if dtype == torch.float8_e4m3fn else dtype, device=device)
                for _ in range(2))
        if dtype != torch.float8_e4m3fn:
            return cls(k, v)
        exps = (torch.full(shape[:3], 127, dtype=torch.uint8, device=device) for _ in range(2))
        return cls(k.view(dtype), v.view(dtype), *exps)


def _check_device(cache):
    """The library launches on the current device, with its workspace and error word."""
    if torch.cuda.current_device() != cache.index:
        raise ValueError("the cache's device must be the current one")


def _raw_stream(stream, cache):
    """The stream a paged-cache call runs on, as a number."""
    return torch._C._cuda_getCurrentRawStream(cache.index) if stream is None else stream.cuda_stream


def _output(shape, dtype, cache, stream):
    """An output a call allocates: memory of the stream that writes it.  With another stream than the current
    one, the current one's later use is waited for as well before the memory is given out again."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=cache.device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=cache.device)
    t.record_stream(torch.cuda.current_stream(cache.device))
    return t


def _check_rows(name, t, cache, heads):
    """A [N, heads, d] input of the cache's row type, d contiguous."""
    if t.dim() != 3 or t.shape[2] != cache.d or (heads is not None and t.shape[1] != heads):
        raise ValueError(f"{name} must be [N, heads, d] with the cache's d" + ("" if heads is None else " and H"))
    if t.dtype is not cache.row_dtype or t.get_device() != cache.index:
        raise ValueError(f"{name} must be {cache.row_dtype} on the cache's device")
    if t.stride(2) != 1:
        raise ValueError(f"{name}'s last axis must be contiguous")


def _row_strides(t):
    """Token and head strides of a [N, heads, d] tensor; an axis of length one has none."""
    n, h, _ = t.stride()
    return (n if t.shape[0] > 1 else 0), (h if t.shape[1] > 1 else 0)


def _check_whole(name, t, shape, dtype, index):
    """A contiguous tensor of a shape and type on CUDA device `index`; returns its address."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on the cache's device")
    return t.data_ptr()


def fem_cache_write(cache: PagedCache, k, v, slots, stream=None):
    """Put N tokens' keys and values [N, H, d] into the cache at slots (int64 [N]: page *
    page_size + row; negative: left out).  k and v may be strided views; a float8_e4m3fn
    cache quantises each (token, head) row as it is written."""
    _check_device(cache)
    N = k.shape[0]
    _check_rows("k", k, cache, cache.H)
    _check_rows("v", v, cache, cache.H)
    if v.shape[0] != N:
        raise ValueError("k and v must have as many tokens")
    rc = load().fem_cache_write(cache._ref, k.data_ptr(), v.data_ptr(), *_row_strides(k), *_row_strides(v),
                                _check_whole("slots", slots, (N,), torch.int64, cache.index), N,
                                _raw_stream(stream, cache))
    if rc != 0:
        raise FemError("fem_cache_write", rc)


def fem_cache_gather(cache: PagedCache, block_table, starts, offsets, total: int, k_out=None, v_out=None, stream=None):
    """Read stretches of cached sequences back as contiguous (k, v) [total, H, d].

    block_table: int32 [S, max_pages]; starts: int32 [S], each stretch's first position;
    offsets: int32 [S + 1], its rows of the output; total = offsets[S]."""
    _check_device(cache)
    if block_table.dim() != 2:
        raise ValueError("block_table must be [S, max_pages]")
    (S, max_pages), shape, index = block_table.shape, (total, cache.H, cache.d), cache.index
    if k_out is None:
        k_out = _output(shape, cache.row_dtype, cache, stream)
    if v_out is None:
        v_out = _output(shape, cache.row_dtype, cache, stream)
    rc = load().fem_cache_gather(cache._ref, _check_whole("block_table", block_table, (S, max_pages), torch.int32, index),
                                 max_pages, _check_whole("starts", starts, (S,), torch.int32, index),
                                 _check_whole("offsets", offsets, (S + 1,), torch.int32, index), S,
                                 _check_whole("k_out", k_out, shape, cache.row_dtype, index),
                                 _check_whole("v_out", v_out, shape, cache.row_dtype, index), total,
                                 _raw_stream(stream, cache))
    if rc != 0:
        raise FemError("fem_cache_gather", rc)
    return k_out, v_out


def fem_paged_read(q, cache: PagedCache, beta, q_offsets, ctx_lens, block_table, max_q: int, causal: bool = True,
                   out=None, lse=None, stream=None):
    """The read of new tokens q [N, Hq, d] over a paged cache that holds their own keys and values.

    Sequence s has the rows q_offsets[s] .. q_offsets[s+1] - 1 (int32 [S + 1]) and ctx_lens[s]
    (int32 [S]) cached positions; block_table is int32 [S, max_pages]; beta is float32 [H, d] of
    the cache's heads or None (the prior mean, plain softmax attention); max_q bounds the rows
    of a sequence.  Returns (out [N, Hq, d] of q's type, lse [N, Hq] float32); ``lse=False``
    skips the log-normaliser."""
    _check_device(cache)
    _check_rows("q", q, cache, None)
    N, Hq, d = q.shape
    if Hq % cache.H:
        raise ValueError("q's heads must be a multiple of the cache's")
    if block_table.dim() != 2:
        raise ValueError("block_table must be [S, max_pages]")
    (S, max_pages), index = block_table.shape, cache.index
    out_ptr = lse_ptr = beta_ptr = None
    if out is None:
        out = _output((N, Hq, d), cache.row_dtype, cache, stream)
        out_ptr = out.data_ptr()
    else:
        out_ptr = _check_whole("out", out, (N, Hq, d), q.dtype, index)
    if lse is None:
        lse = _output((N, Hq), torch.float32, cache, stream)
        lse_ptr = lse.data_ptr()
    elif lse is not False:
        lse_ptr = _check_whole("lse", lse, (N, Hq), torch.float32, index)
    if beta is not None:
        beta_ptr = _check_whole("beta", beta, (cache.H, d), torch.float32, index)
    rc = load().fem_paged_read(cache._ref, q.data_ptr(), *_row_strides(q), beta_ptr,
                               _check_whole("q_offsets", q_offsets, (S + 1,), torch.int32, index),
                               _check_whole("ctx_lens", ctx_lens, (S,), torch.int32, index),
                               _check_whole("block_table", block_table, (S, max_pages), torch.int32, index),
                               max_pages, S, N, Hq, int(max_q), int(bool(causal)), out_ptr, lse_ptr,
                               _raw_stream(stream, cache))
    if rc != 0:
        raise FemError("fem_paged_read", rc)
    return out, (None if lse is False else lse)


_TYPES = {torch.bfloat16: 0, torch.float32: 2}  # fem_type
_heads_bytes = struct.Struct("@Pqqq").pack  # fem_heads of include/fem.h: address, strides over b, t and h


def _current(index):
    """The library launches on the current device, where its error word and workspaces are."""
    if index < 0 or torch._C._cuda_getDevice() != index:
        raise ValueError("the tensors' device must be a CUDA device and the current one")


_UNSUPPORTED = 2  # of STATUS


def _sizes(entry, *sizes):
    """The entries take sizes of 32 bits, and ctypes would pass on the low ones of a larger number."""
    if max(sizes) > 0x7fffffff:
        raise FemError(entry, _UNSUPPORTED)


def _stream_number(stream, index):
    return torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream


def _new(like, shape, dtype, stream):
    """An output a call allocates, on `like`'s device (_output)."""
    return torch.empty(shape, dtype=dtype, device=like.device) if stream is None else _output(shape, dtype, like, stream)


def _optional(name, t, shape, dtype, index):
    """Address of a contiguous tensor that may be absent."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on the other tensors' device")
    return t.data_ptr()


def _heads(name, t, shape, dtype, index):
    """[N, H, d] or [B, H, T, d] as fem_heads."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        raise ValueError(f"{name} must be {dtype} {tuple(shape)} on the other tensors' device")
    st = t.stride()
    if st[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}'s last axis must be contiguous")
    if len(st) == 3:
        return _heads_bytes(t.data_ptr(), 0, st[0], st[1])
    return _heads_bytes(t.data_ptr(), st[0], st[2], st[1])


def _fresh_heads(t, shape):
    """A contiguous tensor's fem_heads."""
    if len(shape) == 3:
        return _heads_bytes(t.data_ptr(), 0, shape[1] * shape[2], shape[2])
    return _heads_bytes(t.data_ptr(), shape[1] * shape[2] * shape[3], shape[3], shape[2] * shape[3])


class _Settled:
    """Its attributes stay as the constructor leaves them, which ends with `_settle`: the calls take what it made of them."""

    def _settle(self):
        self.__dict__["_settled"] = True

    def __setattr__(self, name, value):
        if "_settled" in self.__dict__:
            raise AttributeError(f"a {type(self).__name__}'s {name} cannot be changed: make another one")
        object.__setattr__(self, name, value)


class Rope(_Settled):
    """The rates of rotary positions, for ``fem_rope``: of every head the first ``rotary_dim`` elements turn in pairs,
    elements i and i + rotary_dim/2, or 2 i and 2 i + 1 where ``interleaved``, by pos * base^(-2 i / rotary_dim).

    ``scaling`` stretches the rates for contexts ``factor`` times as long: "linear" all of them, "base" by a larger
    base, "parts" those that turn less than ``low`` times over ``context`` positions, those that turn more than
    ``high`` times not, and those between in part.  ``amplitude`` multiplies the rotated part.  The table lives on
    ``device``; the attributes cannot be assigned to."""

    SCALINGS = {None: 0, "linear": 1, "base": 2, "parts": 3}

    def __init__(self, rotary_dim: int, base: float = 10000.0, interleaved: bool = False, scaling=None, factor: float = 1.0,
                 context: float = 4096.0, low: float = 1.0, high: float = 32.0, amplitude: float = 1.0, device="cuda"):
        if scaling not in self.SCALINGS:
            raise ValueError(f"scaling must be one of {list(self.SCALINGS)}")
        _sizes("fem_rope_turns", rotary_dim)
        table = (ctypes.c_uint64 * max(1, min(rotary_dim, 1024) // 2))()  # longer ones are refused
        rc = load().fem_rope_turns(rotary_dim, base, self.SCALINGS[scaling], factor, context, low, high, table)
        if rc != 0:
            raise FemError("fem_rope_turns", rc)
        signed = [v - (1 << 64) if v >> 63 else v for v in table]
        self.turns = torch.tensor(signed, dtype=torch.int64).to(device)
        self.index = self.turns.get_device()
        self.rotary_dim, self.interleaved, self.amplitude = rotary_dim, int(bool(interleaved)), float(amplitude)
        self._settle()


def fem_rope(rope: Rope, q, k=None, positions=None, inverse: bool = False, out=None, stream=None):
    """Rotary positions of queries and keys, [N, heads, d] or [B, heads, T, d] of bf16 or float32 (k may be None).

    positions: int32 [N] or [B, T]; None counts from 0 along N or T.  ``inverse`` turns back, which takes the outputs'
    gradients to the inputs'.  Strided views are taken as they are.  ``out``: the pair of output tensors, which may be
    (q, k) themselves.  Returns (q, k)."""
    shape, dtype, index = q.shape, q.dtype, q.get_device()
    if len(shape) == 3:
        (T, Hq, d), B = shape, 1
    elif len(shape) == 4:
        B, Hq, T, d = shape
    else:
        raise ValueError("q must be [N, heads, d] or [B, heads, T, d]")
    if dtype not in _TYPES:
        raise ValueError(f"q has dtype {dtype}")
    _current(index)
    _sizes("fem_rope", B, T, Hq, d, *(() if k is None else k.shape))
    if rope.index != index:
        raise ValueError("the rope's table must be on q's device")
    q_out, k_out = out if out is not None else (None, None)
    qv = _heads("q", q, shape, dtype, index)
    if q_out is None:
        q_out = _new(q, shape, dtype, stream)
        qo = _fresh_heads(q_out, shape)
    else:
        qo = _heads("out", q_out, shape, dtype, index)
    kv = ko = None
    Hk = 0
    if k is not None:
        k_shape = k.shape
        if len(k_shape) != len(shape) or k_shape[-1] != d or (k_shape[0] != T if B == 1 and len(shape) == 3 else
                                                              (k_shape[0], k_shape[2]) != (B, T)):
            raise ValueError("q and k must have the same tokens and d")
        Hk = k_shape[1]
        kv = _heads("k", k, k_shape, dtype, index)
        if k_out is None:
            k_out = _new(k, k_shape, dtype, stream)
            ko = _fresh_heads(k_out, k_shape)
        else:
            ko = _heads("out", k_out, k_shape, dtype, index)
    elif k_out is not None:
        raise ValueError("out has keys and the call none")
    pos = None
    if positions is not None:
        pos = _optional("positions", positions, (T,) if len(shape) == 3 else (B, T), torch.int32, index)
    rc = load().fem_rope(qv, qo, Hq, kv, ko, Hk, B, T, d, _TYPES[dtype], rope.turns.data_ptr(), rope.rotary_dim, rope.interleaved,
                         rope.amplitude, pos, 1 if inverse else 0, _stream_number(stream, index))
    if rc != 0:
        raise FemError("fem_rope", rc)
    return q_out, k_out


def _recur_rows(name, t, shape, dtype, index):
    """Address and row stride of a [N, C] or [B, T, C] tensor."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        raise ValueError(f"{name} must have s's shape, type and device")
    if t.is_contiguous():
        return t.data_ptr(), shape[-1]
    st = t.stride()
    if st[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}'s last axis must be contiguous")
    if len(shape) == 2:
        return t.data_ptr(), (st[0] if shape[0] > 1 else shape[1])
    B, T, C = shape
    row = st[1] if T > 1 else st[0] if B > 1 else C
    if B > 1 and T > 1 and st[0] != T * row:
        raise ValueError(f"{name}'s rows must be evenly spaced over batch and time")
    return t.data_ptr(), row


def _recur_sizes(entry, s, offsets, max_len):
    """(shape, dtype, device, address of the offsets, S, T, N, C) of a call; checks s and the offsets."""
    shape, dtype, index = s.shape, s.dtype, s.get_device()
    if dtype not in _TYPES:
        raise ValueError(f"s has dtype {dtype}")
    _current(index)
    if len(shape) != (3 if offsets is None else 2):
        raise ValueError("s must be [B, T, C], or [N, C] with offsets")
    if offsets is None:
        B, T, C = shape
        _sizes(entry, B, T, B * T, C)
        return shape, dtype, index, None, B, T, B * T, C
    if offsets.dim() != 1 or offsets.shape[0] < 1:
        raise ValueError("offsets must be int32 [S + 1]")
    S, (N, C) = offsets.shape[0] - 1, shape
    _sizes(entry, S, N, C)
    off = _optional("offsets", offsets, (S + 1,), torch.int32, index)
    return shape, dtype, index, off, S, N if max_len is None else min(int(max_len), 0x7fffffff), N, C


def fem_recur_fwd(s, u, offsets=None, max_len=None, h0=None, state_rows=None, mean: bool = False, out=None,
                  state_out=None, stream=None):
    """The gated linear recurrence h_t = exp(-s_t) h_{t-1} + w(s_t) u_t of every channel, w = 1, or 1 - exp(-s_t)
    where ``mean``, on bf16 or float32 CUDA tensors.

    s, u: [B, T, C], or packed [N, C] with offsets int32 [S + 1] (``max_len`` bounds their lengths); s >= 0.
    h0: float32 states before the first step, [S, C], or [num_states, C] with state_rows int32 [S] (negative: none).
    state_out: where the states after the last step go, shaped like h0: None allocates [S, C], or with state_rows
    updates h0 in place; False skips them.  Returns (h, states)."""
    shape, dtype, index, off, S, T, N, C = _recur_sizes("fem_recur_fwd", s, offsets, max_len)
    if state_out is None and state_rows is not None and h0 is not None:
        state_out = h0
    kept = state_out is not None and state_out is not False
    if h0 is None and not kept:
        if state_rows is not None:
            raise ValueError("state_rows goes with h0 or state_out")
        num = S
    else:
        num = (state_out if h0 is None else h0).shape[0]
        _sizes("fem_recur_fwd", num)
        if state_rows is None and num != S:
            raise ValueError("h0 and state_out must have a row for each sequence, or state_rows")
    h0_ptr = _optional("h0", h0, (num, C), torch.float32, index)
    rows_ptr = _optional("state_rows", state_rows, (S,), torch.int32, index)
    s_ptr, s_st = _recur_rows("s", s, shape, dtype, index)
    u_ptr, u_st = _recur_rows("u", u, shape, dtype, index)
    if out is None:
        out = _new(s, shape, dtype, stream)
        h_ptr, h_st = out.data_ptr(), C
    else:
        h_ptr, h_st = _recur_rows("out", out, shape, dtype, index)
    if state_out is False:
        last_ptr = state_out = None
    elif state_out is None:
        num = max(num, S)
        state_out = _new(s, (S, C), torch.float32, stream)
        last_ptr = state_out.data_ptr()
    else:
        last_ptr = _optional("state_out", state_out, (num, C), torch.float32, index)
    rc = load().fem_recur_fwd(s_ptr, u_ptr, s_st, u_st, off, S, T, N, C, _TYPES[dtype], 1 if mean else 0, h0_ptr, last_ptr,
                              rows_ptr, num, h_ptr, h_st, _stream_number(stream, index))
    if rc != 0:
        raise FemError("fem_recur_fwd", rc)
    return out, state_out


def fem_recur_bwd(s, u, h, dh, offsets=None, max_len=None, h0=None, dstate=None, mean: bool = False, stream=None):
    """Gradients of ``fem_recur_fwd`` from its outputs h and their cotangents dh, and the last states' dstate
    (float32 [S, C] or None).  h0: float32 [S, C] or None, as the forward had it.  u is read where ``mean`` only, and
    may be None elsewhere.

    Returns (ds, du, dh0), dh0 None where h0 is."""
    shape, dtype, index, off, S, T, N, C = _recur_sizes("fem_recur_bwd", s, offsets, max_len)
    (s_ptr, s_st), (h_ptr, h_st), (g_ptr, g_st) = (
        _recur_rows(name, t, shape, dtype, index) for name, t in (("s", s), ("h", h), ("dh", dh)))
    if u is None and mean:
        raise ValueError("the mean's gradients need u")
    u_ptr, u_st = _recur_rows("u", u, shape, dtype, index) if u is not None else (None, 0)
    ds, du = _new(s, shape, dtype, stream), _new(s, shape, dtype, stream)
    dh0 = None if h0 is None else _new(s, (S, C), torch.float32, stream)
    rc = load().fem_recur_bwd(s_ptr, u_ptr, h_ptr, g_ptr, s_st, u_st, h_st, g_st, off, S, T, N, C, _TYPES[dtype], 1 if mean else 0,
                              _optional("h0", h0, (S, C), torch.float32, index),
                              _optional("dstate", dstate, (S, C), torch.float32, index), ds.data_ptr(), du.data_ptr(), C, C,
                              None if dh0 is None else dh0.data_ptr(), _stream_number(stream, index))
    if rc != 0:
        raise FemError("fem_recur_bwd", rc)
    return ds, du, dh0


_norm_bytes = struct.Struct("@9i2f4P").pack  # fem_norm of include/fem.h


class BlockNorm(_Settled):
    """A block's end and the next one's start, for ``fem_norm_fwd`` and ``fem_norm_bwd``:

        r = x + scale act(gate) (w_post P(y) + b_post),    z = w_pre Q(r) + b_pre

    ``post`` and ``pre`` name P and Q: "none", "rms" or "layer" (``pre`` "none": there is no z); ``gate`` the gate's act:
    "none" (no gate), "identity", "sigmoid" or "silu".  The weights are float32 [width] CUDA tensors or None (1 and 0); the object
    keeps them, and looks at and reads them at each call.  Its attributes cannot be assigned to."""

    KINDS = {"none": 0, "rms": 1, "layer": 2}
    ACTS = {"none": 0, "identity": 0, "sigmoid": 1, "silu": 2}

    def __init__(self, width: int, post: str = "rms", pre: str = "rms", gate: str = "none", w_post=None, b_post=None,
                 w_pre=None, b_pre=None, scale: float = 1.0, eps: float = 1e-6):
        if width < 1:
            raise ValueError("width must be positive")
        if post not in self.KINDS or pre not in self.KINDS or gate not in self.ACTS:
            raise ValueError(f"post and pre are one of {list(self.KINDS)}, gate one of {list(self.ACTS)}")
        self.width, self.post, self.pre, self.gate, self.scale, self.eps = width, post, pre, gate, float(scale), float(eps)
        self._weights = {"w_post": w_post, "b_post": b_post, "w_pre": w_pre, "b_pre": b_pre}
        self.index = None  # of the weights' device
        for name, t in self._weights.items():
            if t is None:
                continue
            if t.device.type != "cuda":
                raise ValueError(f"{name} must be a contiguous float32 CUDA tensor of shape ({width},)")
            if self.index not in (None, t.get_device()):
                raise ValueError("the weights must be on one device")
            self.index = t.get_device()
        self._fixed = (self.KINDS[post], self.KINDS[pre], self.ACTS[gate], self.scale, self.eps)
        self._vector = torch.Size((width,))
        self._settle()
        self._addresses()

    @property
    def weights(self):
        """The weights by name, to be read: what they hold may change, which there are may not."""
        return types.MappingProxyType(self._weights)

    def _addresses(self):
        """The weights' addresses for a call, each looked at again: a module that changes its type or device replaces
        what is behind a parameter."""
        got = []
        for name, t in self._weights.items():
            if t is None:
                got.append(0)
                continue
            if t.dtype is not torch.float32 or t.shape != self._vector or t.get_device() != self.index or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous float32 CUDA tensor of shape ({self.width},) on the device it came from")
            got.append(t.data_ptr())
        return got

    def _call(self, entry, name, x, y, gate):
        """((B, T, H, d), x's shape, x's and the branch's type, device) of a call; checks x, y and the gate."""
        shape, dtype, index = x.shape, x.dtype, x.get_device()
        if dtype not in _TYPES or not shape or shape[-1] != self.width or not x.is_contiguous():
            raise ValueError(f"{name} must be a contiguous bf16 or float32 tensor [..., {self.width}]")
        _current(index)
        if self.index is not None and self.index != index:
            raise ValueError(f"{name} must be on the weights' device")
        if (gate is not None) != (y is not None and self.gate != "none"):
            raise ValueError("gate goes with y and with a norm that has one")
        rows = x.numel() // self.width
        if y is None or y.shape == shape:
            B, T, H, d = 1, rows, 1, self.width
        else:
            y_shape = y.shape
            if len(y_shape) == 3:
                (T, H, d), B = y_shape, 1
            elif len(y_shape) == 4:
                B, H, T, d = y_shape
            else:
                raise ValueError("y must have x's shape or be [N, H, d] or [B, H, T, d]")
            if B * T != rows or H * d != self.width or (len(shape) == 3 and len(y_shape) == 4 and (B, T) != shape[:2]):
                raise ValueError("y must have x's rows, and heads of its width together")
        _sizes(entry, B, T, H, d)
        y_type = dtype if y is None else y.dtype
        if y_type not in _TYPES:
            raise ValueError(f"y has dtype {y_type}")
        return (B, T, H, d), shape, dtype, y_type, index

    def _describe(self, sizes, x_type, y_type):
        return _norm_bytes(*sizes, _TYPES[x_type], _TYPES[y_type], *self._fixed, *self._addresses())


def _branch(name, t, x_shape, shape, dtype, index):
    """A branch tensor (x's shape, [N, H, d] or [B, H, T, d]) as fem_heads."""
    if t.shape != x_shape:
        return _heads(name, t, shape, dtype, index)
    if t.dtype is not dtype or t.get_device() != index or shape != x_shape:
        raise ValueError(f"{name} must be {dtype} {tuple(shape)} on x's device")
    width = x_shape[-1]
    if t.is_contiguous():
        return _heads_bytes(t.data_ptr(), 0, width, 0)
    st = t.stride()
    if st[-1] != 1 and width > 1:
        raise ValueError(f"{name}'s last axis must be contiguous")
    row, span = None, 1  # rows of all leading axes, evenly spaced
    for n, step in zip(reversed(x_shape[:-1]), reversed(st[:-1])):
        if n > 1:
            if row is not None and step != row * span:
                raise ValueError(f"{name}'s rows must be evenly spaced")
            row = step if row is None else row
            span *= n
    return _heads_bytes(t.data_ptr(), 0, 0 if row is None else row, 0)


def _fresh_branch(t, x_shape, shape):
    return _heads_bytes(t.data_ptr(), 0, x_shape[-1], 0) if shape == x_shape else _fresh_heads(t, shape)


def fem_norm_fwd(norm: BlockNorm, x, y=None, gate=None, out=None, z_out=None, stream=None):
    """The residual stream after a block and what the next block reads (``BlockNorm``), in one pass.

    x: contiguous [..., width], bf16 or float32; y and gate: x's shape, or heads [N, H, d] or [B, H, T, d] (the read's
    outputs as they are), bf16, or float32 with a float32 x; without y there is no block before and r is x.  ``out`` may
    be x itself.  Returns (r, z), z of y's type (without y of z_out's, or x's)."""
    sizes, shape, dtype, y_type, index = norm._call("fem_norm_fwd", "x", x, y, gate)
    yv = gv = r_ptr = z_ptr = None
    if y is not None:
        y_shape = y.shape
        yv = _branch("y", y, shape, y_shape, y_type, index)
        if gate is not None:
            gv = _branch("gate", gate, shape, y_shape, y_type, index)
        if out is None:
            out = _new(x, shape, dtype, stream)
            r_ptr = out.data_ptr()
        else:
            r_ptr = _optional("out", out, shape, dtype, index)
    elif out is not None:
        raise ValueError("out goes with y")
    else:
        out = x
        if z_out is not None:
            y_type = z_out.dtype
            if y_type not in _TYPES:
                raise ValueError(f"z_out has dtype {y_type}")
    if norm.pre != "none":
        if z_out is None:
            z_out = _new(x, shape, y_type, stream)
            z_ptr = z_out.data_ptr()
        else:
            z_ptr = _optional("z_out", z_out, shape, y_type, index)
    elif z_out is not None:
        raise ValueError("z_out goes with a pre norm")
    rc = load().fem_norm_fwd(norm._describe(sizes, dtype, y_type), x.data_ptr(), yv, gv, r_ptr, z_ptr, _stream_number(stream, index))
    if rc != 0:
        raise FemError("fem_norm_fwd", rc)
    return out, z_out


def fem_norm_bwd(norm: BlockNorm, r, y=None, gate=None, dr=None, dz=None, stream=None):
    """Gradients of ``fem_norm_fwd`` from its r, y and gate and the cotangents dr (or None) and dz (with a pre norm).

    Returns (dx, dy, dgate, dw_post, db_post, dw_pre, db_pre): dy and dgate of y's shape, contiguous; the weights'
    float32 [width], summed over all rows; None for what is not there (biases' where the norm has none)."""
    sizes, shape, dtype, y_type, index = norm._call("fem_norm_bwd", "r", r, y, gate)
    if (norm.pre != "none") != (dz is not None):
        raise ValueError("dz goes with a pre norm")
    if y is None and dz is not None:
        y_type = dz.dtype
        if y_type not in _TYPES:
            raise ValueError(f"dz has dtype {y_type}")
    dr_ptr = _optional("dr", dr, shape, dtype, index)
    dz_ptr = _optional("dz", dz, shape, y_type, index)
    dx = _new(r, shape, dtype, stream)
    dy = dgate = yv = gv = dyv = dgv = None
    if y is not None:
        y_shape = y.shape
        yv = _branch("y", y, shape, y_shape, y_type, index)
        dy = _new(r, y_shape, y_type, stream)
        dyv = _fresh_branch(dy, shape, y_shape)
        if gate is not None:
            gv = _branch("gate", gate, shape, y_shape, y_type, index)
            dgate = _new(r, y_shape, y_type, stream)
            dgv = _fresh_branch(dgate, shape, y_shape)
    pre, weights = norm.pre != "none", norm._weights
    wanted = (y is not None, y is not None and weights["b_post"] is not None, pre, pre and weights["b_pre"] is not None)
    sums = [_new(r, (norm.width,), torch.float32, stream) if on else None for on in wanted]
    rc = load().fem_norm_bwd(norm._describe(sizes, dtype, y_type), r.data_ptr(), yv, gv, dr_ptr, dz_ptr, dx.data_ptr(), dyv, dgv,
                             *(None if t is None else t.data_ptr() for t in sums), _stream_number(stream, index))
    if rc != 0:
        raise FemError("fem_norm_bwd", rc)
    return dx, dy, dgate, *sums


def probe_wait_timeout(limit_us: int, stream=None, device=None):
    """Enqueue the library's wait probe: a bounded wait on an mbarrier nothing completes,
    which gives up after limit_us microseconds and records a timeout in the error word."""
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    rc = load().fem_probe_wait_timeout(int(limit_us), _stream(stream, dev))
    if rc != 0:
        raise FemError("fem_probe_wait_timeout", rc)


def check_device_error(stream=None, device=None):
    """Synchronise and raise FemError if a kernel gave up on a bounded wait or met an index outside its buffers."""
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    rc = load().fem_check_device_error(_stream(stream, dev))
    if rc != 0:
        raise FemError("fem_check_device_error", rc)


def set_kernel_events(start, stop):
    """Have the next bf16 read of this thread record torch CUDA events around its tensor-core kernel."""
    load().fem_set_kernel_events(ctypes.c_void_p(start.cuda_event), ctypes.c_void_p(stop.cuda_event))


def last_fixup_rows(stream=None, device=None) -> int:
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    return int(load().fem_last_fixup_rows(_stream(stream, dev)))
