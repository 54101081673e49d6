"""Thin ctypes binding of libwf (include/wf.h), same names as the C ABI.

Argument marshalling only: torch tensors are turned into device pointers and
wf_tensor descriptors, the current CUDA stream is passed through, and a
negative status raises WfError.  Every step of the path runs in libwf's CUDA
kernels; if libwf.so is missing this module raises on import of the library
(there is no fallback).

Tensors are [B, H, rows, d] views whose last axis is contiguous (BHSD or
BSHD strides both work); idx, level_sets, tables, lengths and masks are int32.

A short call is bound by the time spent here, so the marshalling avoids what
costs most: addresses and descriptors go to ctypes as they are (the argtypes
convert them), shapes and strides are read once a tensor, and the current
stream's handle is asked for without building a stream object.
"""
from __future__ import annotations

import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libwf.so")

WF_F32, WF_BF16, WF_MXFP8, WF_MXFP4 = 0, 1, 2, 3
_DTYPES = {torch.float32: WF_F32, torch.bfloat16: WF_BF16}


class WfError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_str(status)} ({status})")
        self.status = status


class wf_tensor(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("seq", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64),
                ("stride_s", ctypes.c_int64), ("dtype", ctypes.c_int32)]


class wf_testing_plan(ctypes.Structure):
    _fields_ = [("workspace_used", ctypes.c_longlong)] + [
        (name, ctypes.c_int) for name in ("prompt_parts", "own_parts", "key_tile", "prompt_rows", "joined", "direct",
                                          "join_rows")]


_lib = None

# Every symbol declared in include/wf.h, with its ctypes signature.
_P, _I, _I64, _SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
_T = ctypes.POINTER(wf_tensor)
SIGNATURES = {
    "wf_status_str": (ctypes.c_char_p, [_I]),
    "wf_coeffs_bytes": (_SZ, [_T, _I]),
    "wf_dwt_build": (_I, [_P, _P, _T, _I, _P, _SZ, _P]),
    "wf_default_schedule": (_I, [_I64, _I, _I64, _P]),
    "wf_level0_schedule": (_I, [_I64, _I, _I64, _P]),
    "wf_cache_update": (_I, [_P, _P, _T, _P, _P, _T, _I64, _I, _P, _SZ, _P]),
    "wf_schedule_from_proportions": (_I, [_I64, _I, _P, _P]),
    "wf_filter_workspace_bytes": (_SZ, [_T, _T, _I, _P]),
    "wf_filter": (_I, [_P, _T, _P, _P, _T, _I, _P, _P, _P, _P, _SZ, _P]),
    "wf_wavelet_approx": (_I, [_P, _T, _P, _I, _I, _I, _P, _SZ, _P]),
    "wf_filter_wavelet_workspace_bytes": (_SZ, [_T, _T, _I, _P, _I]),
    "wf_filter_wavelet": (_I, [_P, _T, _P, _P, _T, _I, _P, _I, _P, _P, _P, _SZ, _P]),
    "wf_attn_workspace_bytes": (_SZ, [_T, _I, _I]),
    "wf_sparse_attn": (_I, [_P, _T, _P, _P, _T, _P, _I, _P, _P, _T, _P, _T, ctypes.c_float, _P, _SZ, _P]),
    "wf_step_workspace_bytes": (_SZ, [_T, _T, _I, _P, _I]),
    "wf_sparse_attn_noalloc": (_I, [_P, _T, _P, _P, _T, _P, _I, _P, _P, _T, _P, _T, ctypes.c_float, _P]),
    "wf_noalloc_status": (_I, [_P]),
    "wf_step": (_I, [_P, _T, _P, _P, _T, _P, _P, _T, _P, _SZ, _I, _I, _P, _P, _P, _P, _T, _P, _SZ, _P]),
    "wf_step_wavelet_workspace_bytes": (_SZ, [_T, _T, _I, _P, _I, _I]),
    "wf_step_wavelet": (_I, [_P, _T, _P, _P, _P, _T, _P, _P, _T, _I, _P, _I, _P, _P, _P, _T, _P, _SZ, _P]),
    "wf_scales_bytes": (_SZ, [_T]),
    "wf_cache_quantize": (_I, [_P, _P, _T, _P, _P, _P, _P, _T, _SZ, _I64, _P]),
    "wf_cache_dequantize": (_I, [_P, _P, _P, _P, _T, _SZ, _P, _I64, _P, _P, _T, _P]),
    "wf_prefix_attn_workspace_bytes": (_SZ, [_T, _T, _I, _I]),
    "wf_prefix_attn": (_I, [_P, _T, _P, _P, _T, _P, _P, _P, _I, _P, _P, _P, _T, _P, _P, _T, ctypes.c_float, _P, _SZ,
                            _P]),
    "wf_rotary_plan": (_I, [_P, _P, _I, _P]),
    "wf_rotary_apply": (_I, [_P, _T, _P, _T, _P, _I, _I, _P, _I, _P, _T, _P, _T, _P]),
    "wf_paged_append": (_I, [_P, _P, _T, _P, _I, _P, _P, _P, _I, _I, _P, _I, _P, _P, _P, _P, _T, _SZ, _P, _I, _P]),
    "wf_tree_attn_workspace_bytes": (_SZ, [_T, _T, _I, _I]),
    "wf_tree_attn": (_I, [_P, _T, _P, _P, _T, _P, _P, _P, _I, _I, _P, _P, _P, _T, _P, _P, _P, _T, ctypes.c_float, _P,
                          _SZ, _P]),
    "wf_workspace_status": (_I, [_P, _P]),
    # include/wf_testing.h (test-only)
    "wf_testing_set_wait_failure": (_I, [_I, ctypes.c_longlong]),
    "wf_testing_prefix_plan": (_I, [_T, _T, _I, _I, ctypes.POINTER(wf_testing_plan)]),
}


def lib():
    """Load libwf.so (built by __graft_entry__.build() / build.py)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"libwf.so not built at {LIB_PATH}; run paper_2606_00724_gb300/build.py")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def status_str(status: int) -> str:
    return lib().wf_status_str(status).decode()


def _check(status: int, what: str):
    if status != 0:
        raise WfError(status, what)


# Descriptors by what they describe (never by an address): building one takes longer
# than finding it.  No call writes to a descriptor.
_DESCS: dict = {}


def _desc(shape, stride, dtype, fmt=None) -> wf_tensor:
    key = (shape, stride, dtype, fmt)
    d = _DESCS.get(key)
    if d is None:
        d = _row_desc(shape, stride, dtype) if fmt is None else _code_desc(shape, stride, dtype.itemsize, fmt)
        if len(_DESCS) >= 4096:
            _DESCS.clear()
        _DESCS[key] = d
    return d


def _row_desc(shape, stride, dtype) -> wf_tensor:
    if len(shape) != 4:
        raise ValueError("expected a [B, H, rows, d] tensor")
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError(f"unsupported dtype {dtype}")
    sb, sh, ss, sd = stride
    B, H, S, D = shape
    if D > 1 and sd != 1:
        raise ValueError("head_dim axis must be contiguous")
    return wf_tensor(B, H, S, D, sb, sh, ss, code)


def desc(t: torch.Tensor) -> wf_tensor:
    """wf_tensor for a [B, H, rows, d] tensor with a contiguous last axis."""
    return _row_desc(t.shape, t.stride(), t.dtype)


def _code_desc(shape, stride, size: int, fmt: int) -> wf_tensor:
    if len(shape) != 4 or size != 1:
        raise ValueError("expected a [B, H, rows, bytes] tensor of 8-bit codes")
    if fmt == WF_MXFP4:
        per = 2
    elif fmt == WF_MXFP8:
        per = 1
    else:
        raise ValueError(f"unknown format {fmt}")
    B, H, S, W = shape
    sb, sh, ss, sd = stride
    if W > 1 and sd != 1:
        raise ValueError("head_dim axis must be contiguous")
    return wf_tensor(B, H, S, W * per, sb * per, sh * per, ss * per, fmt)


def code_desc(codes: torch.Tensor, fmt: int) -> wf_tensor:
    """wf_tensor for the codes of a quantised cache: [B, H, rows, d] bytes
    (WF_MXFP8) or [B, H, rows, d / 2] (WF_MXFP4), last axis contiguous."""
    return _code_desc(codes.shape, codes.stride(), codes.element_size(), fmt)


def _scales(K_scales, V_scales):
    """Size of the smaller scale tensor (contiguous bytes; 0 if there is none)."""
    size = 0
    for s in (K_scales, V_scales):
        if s is not None:
            n = s.nbytes
            if n != s.numel() or not s.is_contiguous():
                raise ValueError("scales must be contiguous bytes")
            size = n if size == 0 or n < size else size
    return size


def _on_gpu(*tensors):
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise ValueError("expected tensors on the GPU")


def _pair_desc(K, V, what: str, fmt=None) -> wf_tensor:
    """Descriptor of K (codes of the format fmt where that is given); V, where
    there is one, lies as K does."""
    shape, stride, dtype = K.shape, K.stride(), K.dtype
    if V is not None and (V.stride() != stride or V.shape != shape or V.dtype != dtype):
        raise ValueError(f"{what} must share dtype, shape and strides")
    return _desc(shape, stride, dtype, fmt)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _ints(t):
    """Address of a contiguous int32 tensor, or None."""
    if t is None:
        return None
    if t.dtype is not torch.int32 or not t.is_contiguous():
        raise ValueError("indices and lengths must be contiguous int32 tensors")
    return t.data_ptr()


def _same_layout(a, b) -> bool:
    return a.shape == b.shape and a.stride() == b.stride()


# The handle without a stream object, where this torch has the calls for it
# (they are not part of torch's public interface; the public one takes 2.9 us, these 0.2).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


_KEEP_TYPES: dict = {}


def _keep_arr(keep):
    n = len(keep)
    t = _KEEP_TYPES.get(n)
    if t is None:
        t = _KEEP_TYPES[n] = ctypes.c_int32 * n
    return t(*map(int, keep))


def wf_coeffs_bytes(K: torch.Tensor, levels: int) -> int:
    d = desc(K)
    return int(lib().wf_coeffs_bytes(d, levels))


def wf_dwt_build(K: torch.Tensor, levels: int, coeffs: torch.Tensor, stream=None):
    d = desc(K)
    _check(lib().wf_dwt_build(_ptr(K), None, d, levels, _ptr(coeffs),
                              coeffs.nbytes, _stream(stream)), "wf_dwt_build")


def wf_cache_update(Knew: torch.Tensor, Vnew, K: torch.Tensor, V, pos: int, levels: int, coeffs: torch.Tensor,
                    stream=None) -> None:
    """Write Knew (and Vnew) into the caches at [pos, pos + count) and refresh
    the touched pyramid blocks (see the C header)."""
    dn, dk = desc(Knew), desc(K)
    _check(lib().wf_cache_update(_ptr(Knew), _ptr(Vnew) if Vnew is not None else None, dn, _ptr(K),
                                 _ptr(V) if V is not None else None, dk, pos, levels, _ptr(coeffs),
                                 coeffs.nbytes, _stream(stream)), "wf_cache_update")


def wf_default_schedule(n: int, levels: int, k: int) -> list[int]:
    keep = (ctypes.c_int32 * (levels + 1))()
    _check(lib().wf_default_schedule(n, levels, k, keep), "wf_default_schedule")
    return list(keep)


def wf_level0_schedule(n: int, levels: int, k: int) -> list[int]:
    keep = (ctypes.c_int32 * (levels + 1))()
    _check(lib().wf_level0_schedule(n, levels, k, keep), "wf_level0_schedule")
    return list(keep)


def wf_schedule_from_proportions(n: int, levels: int, m) -> list[int]:
    arr = (ctypes.c_double * (levels + 1))(*[float(x) for x in m])
    keep = (ctypes.c_int32 * (levels + 1))()
    _check(lib().wf_schedule_from_proportions(n, levels, arr, keep), "wf_schedule_from_proportions")
    return list(keep)


def wf_filter_workspace_bytes(Q: torch.Tensor, K: torch.Tensor, levels: int, keep) -> int:
    dq, dk = desc(Q), desc(K)
    return int(lib().wf_filter_workspace_bytes(dq, dk, levels, _keep_arr(keep)))


def wf_filter(Q: torch.Tensor, coeffs: torch.Tensor, K: torch.Tensor, levels: int, keep, idx: torch.Tensor,
              ws: torch.Tensor, level_sets: torch.Tensor | None = None, stream=None):
    dq, dk = desc(Q), desc(K)
    _check(lib().wf_filter(_ptr(Q), dq, _ptr(coeffs), _ptr(K), dk, levels,
                           _keep_arr(keep), _ptr(idx), _ptr(level_sets), _ptr(ws), ws.nbytes,
                           _stream(stream)), "wf_filter")


WF_WAVELET_HAAR, WF_WAVELET_DB2 = 0, 1


def wf_wavelet_approx(K: torch.Tensor, level: int, wavelet: int, out: torch.Tensor, cand=None, m=None,
                      stream=None):
    """Level-`level` approximation rows of the gathered blocks of `cand`
    ([B*H][m] int32, or None for the whole prompt) into out ([B, H, m, d])."""
    dk = desc(K)
    if m is None:
        m = cand.shape[1] if cand is not None else K.shape[2] >> level
    _check(lib().wf_wavelet_approx(_ptr(K), dk, _ptr(cand), int(m), level, wavelet, _ptr(out),
                                   out.nbytes, _stream(stream)), "wf_wavelet_approx")


def wf_filter_wavelet_workspace_bytes(Q: torch.Tensor, K: torch.Tensor, levels: int, keep, wavelet: int) -> int:
    dq, dk = desc(Q), desc(K)
    return int(lib().wf_filter_wavelet_workspace_bytes(dq, dk, levels, _keep_arr(keep),
                                                       wavelet))


def wf_filter_wavelet(Q: torch.Tensor, top: torch.Tensor, K: torch.Tensor, levels: int, keep, wavelet: int,
                      idx: torch.Tensor, ws: torch.Tensor, level_sets: torch.Tensor | None = None, stream=None):
    dq, dk = desc(Q), desc(K)
    _check(lib().wf_filter_wavelet(_ptr(Q), dq, _ptr(top), _ptr(K), dk, levels,
                                   _keep_arr(keep), wavelet, _ptr(idx), _ptr(level_sets), _ptr(ws),
                                   ws.nbytes, _stream(stream)), "wf_filter_wavelet")


def wf_attn_workspace_bytes(Q: torch.Tensor, k: int, n_g: int) -> int:
    dq = desc(Q)
    return int(lib().wf_attn_workspace_bytes(dq, k, n_g))


def wf_sparse_attn(Q, K, V, idx, k: int, Kg, Vg, O, ws, scale: float = 0.0, stream=None):
    dq, dk, do = desc(Q), desc(K), desc(O)
    dg = desc(Kg) if Kg is not None else None
    if Vg is not None and Kg is not None and not _same_layout(Vg, Kg):
        raise ValueError("Kg and Vg must share shape and strides")
    if not _same_layout(V, K):
        raise ValueError("K and V must share shape and strides")
    _check(lib().wf_sparse_attn(_ptr(Q), dq, _ptr(K), _ptr(V), dk, _ptr(idx), k,
                                _ptr(Kg), _ptr(Vg), dg, _ptr(O),
                                do, float(scale), _ptr(ws), ws.nbytes,
                                _stream(stream)), "wf_sparse_attn")


def wf_sparse_attn_noalloc(Q, K, V, idx, k: int, Kg, Vg, O, scale: float = 0.0, stream=None):
    """wf_sparse_attn for callers that cannot allocate device memory: the
    scratch comes from libwf's fixed static device array
    (WF_NOALLOC_SCRATCH_BYTES = 16 MiB), shared by every call in a CUDA
    context."""
    dq, dk, do = desc(Q), desc(K), desc(O)
    dg = desc(Kg) if Kg is not None else None
    if Vg is not None and Kg is not None and not _same_layout(Vg, Kg):
        raise ValueError("Kg and Vg must share shape and strides")
    if not _same_layout(V, K):
        raise ValueError("K and V must share shape and strides")
    _check(lib().wf_sparse_attn_noalloc(_ptr(Q), dq, _ptr(K), _ptr(V), dk, _ptr(idx),
                                        k, _ptr(Kg), _ptr(Vg), dg,
                                        _ptr(O), do, float(scale), _stream(stream)),
           "wf_sparse_attn_noalloc")


def wf_noalloc_status(stream=None):
    """Raise WfError(WF_ERR_TIMEOUT) if a bounded device wait of the
    allocation-free attention gave up since the last check (synchronising)."""
    _check(lib().wf_noalloc_status(_stream(stream)), "wf_noalloc_status")


def wf_step_workspace_bytes(Q: torch.Tensor, K: torch.Tensor, levels: int, keep, n_g: int) -> int:
    dq, dk = desc(Q), desc(K)
    return int(lib().wf_step_workspace_bytes(dq, dk, levels, _keep_arr(keep), n_g))


def wf_step(Q, K, V, Kg, Vg, coeffs, refresh: bool, levels: int, keep, idx, O, ws, stream=None,
            level_sets=None):
    dq, dk, do = desc(Q), desc(K), desc(O)
    dg = desc(Kg) if Kg is not None else None
    if not _same_layout(V, K):
        raise ValueError("K and V must share shape and strides")
    _check(lib().wf_step(_ptr(Q), dq, _ptr(K), _ptr(V), dk, _ptr(Kg), _ptr(Vg),
                         dg, _ptr(coeffs),
                         coeffs.nbytes, int(bool(refresh)), levels, _keep_arr(keep),
                         _ptr(idx), _ptr(level_sets), _ptr(O), do, _ptr(ws),
                         ws.nbytes, _stream(stream)), "wf_step")


def wf_step_wavelet_workspace_bytes(Q: torch.Tensor, K: torch.Tensor, levels: int, keep, wavelet: int,
                                    n_g: int) -> int:
    dq, dk = desc(Q), desc(K)
    return int(lib().wf_step_wavelet_workspace_bytes(dq, dk, levels, _keep_arr(keep),
                                                     wavelet, n_g))


def wf_step_wavelet(Q, top, K, V, Kg, Vg, levels: int, keep, wavelet: int, idx, O, ws, stream=None,
                    level_sets=None):
    dq, dk, do = desc(Q), desc(K), desc(O)
    dg = desc(Kg) if Kg is not None else None
    if not _same_layout(V, K):
        raise ValueError("K and V must share shape and strides")
    _check(lib().wf_step_wavelet(_ptr(Q), dq, _ptr(top), _ptr(K), _ptr(V), dk,
                                 _ptr(Kg), _ptr(Vg), dg, levels,
                                 _keep_arr(keep), wavelet, _ptr(idx), _ptr(level_sets), _ptr(O), do,
                                 _ptr(ws), ws.nbytes, _stream(stream)), "wf_step_wavelet")


def wf_scales_bytes(codes: torch.Tensor, fmt: int) -> int:
    return int(lib().wf_scales_bytes(code_desc(codes, fmt)))


def wf_cache_quantize(Knew, Vnew, Kc, Ks, Vc, Vs, fmt: int, pos: int, stream=None) -> None:
    """Quantise Knew (and Vnew) into the caches' codes and scales at
    [pos, pos + count) (see the C header; Vnew, Vc, Vs all None: keys alone)."""
    _on_gpu(Knew, Vnew, Kc, Ks, Vc, Vs)
    dn, dk = _pair_desc(Knew, Vnew, "Knew and Vnew"), _pair_desc(Kc, Vc, "Kc and Vc", fmt)
    _check(lib().wf_cache_quantize(_ptr(Knew), _ptr(Vnew), dn, _ptr(Kc), _ptr(Ks), _ptr(Vc), _ptr(Vs), dk,
                                   _scales(Ks, Vs), pos, _stream(stream)), "wf_cache_quantize")


def wf_cache_dequantize(Kc, Ks, Vc, Vs, fmt: int, Kout, Vout, pos: int = 0, idx=None, stream=None) -> None:
    """Rows [pos, pos + m), or the rows idx ([B*H][m] int32), of the caches
    into Kout (and Vout) ([B, H, m, d]) (see the C header)."""
    _on_gpu(Kc, Ks, Vc, Vs, Kout, Vout, idx)
    do, dk = _pair_desc(Kout, Vout, "Kout and Vout"), _pair_desc(Kc, Vc, "Kc and Vc", fmt)
    if idx is not None and tuple(idx.shape) != (Kout.shape[0] * Kout.shape[1], Kout.shape[2]):
        raise ValueError("idx must be [B*H, m]")
    _check(lib().wf_cache_dequantize(_ptr(Kc), _ptr(Ks), _ptr(Vc), _ptr(Vs), dk, _scales(Ks, Vs), _ints(idx), pos,
                                     _ptr(Kout), _ptr(Vout), do, _stream(stream)), "wf_cache_dequantize")


def wf_prefix_attn_workspace_bytes(Q: torch.Tensor, K: torch.Tensor, k: int, n_g: int, fmt=None) -> int:
    return int(lib().wf_prefix_attn_workspace_bytes(desc(Q), _pair_desc(K, None, "", fmt), k, n_g))


def wf_prefix_attn(Q, K, V, k: int, Kg, Vg, O, ws, idx=None, prefix_len=None, gen_len=None, Ks=None, Vs=None,
                   fmt=None, scale: float = 0.0, stream=None) -> None:
    """Attention of Q [B, Hq, q, d] over P cached prompts K, V [P, H, n, d], the
    first k rows or the rows idx [P*H, k] of each, and each sequence's own rows
    Kg, Vg [B, H, n_g, d] (see the C header).  fmt (WF_MXFP8, WF_MXFP4): K and V
    are codes, with scales Ks and Vs."""
    _on_gpu(Q, K, V, Kg, Vg, O, ws, idx, prefix_len, gen_len, Ks, Vs)
    dq = desc(Q)
    do = dq if O.stride() == Q.stride() and O.shape == Q.shape and O.dtype == Q.dtype else desc(O)
    dk = _pair_desc(K, V, "K and V", fmt)
    dg = _pair_desc(Kg, Vg, "Kg and Vg") if Kg is not None else None
    if fmt is not None:
        if Ks is None or Vs is None or _scales(Ks, Vs) < dk.batch * dk.heads * dk.seq * (dk.head_dim // 32):
            raise ValueError("a quantised prompt needs the scales of its K and V")
    if idx is not None and tuple(idx.shape) != (dk.batch * dk.heads, k):
        raise ValueError("idx must be [P*H, k]")
    if prefix_len is not None and prefix_len.numel() != dk.batch:
        raise ValueError("prefix_len must have an entry a prompt")
    if gen_len is not None and gen_len.numel() != dq.batch:
        raise ValueError("gen_len must have an entry a sequence")
    _check(lib().wf_prefix_attn(_ptr(Q), dq, _ptr(K), _ptr(V), dk, _ptr(Ks), _ptr(Vs), _ints(idx), k,
                                _ints(prefix_len), _ptr(Kg), _ptr(Vg), dg, _ints(gen_len), _ptr(O), do, float(scale),
                                _ptr(ws), ws.nbytes, _stream(stream)), "wf_prefix_attn")


def wf_rotary_plan(freq: torch.Tensor, axis: torch.Tensor | None = None) -> torch.Tensor:
    """The plan of a rotation, [pairs, 2] int64 on the host, from the radians a
    position of each pair (float64) and its axis (int32, None: all 0); both are
    tensors on the host (see the C header).  Copy it to the GPU once."""
    if freq.dtype != torch.float64 or freq.dim() != 1 or not freq.is_contiguous() or freq.is_cuda:
        raise ValueError("frequencies must be a contiguous float64 vector on the host")
    if axis is not None and (axis.is_cuda or axis.shape != freq.shape):
        raise ValueError("axes must be a vector on the host, one a pair")
    plan = torch.empty(freq.shape[0], 2, dtype=torch.int64)
    _check(lib().wf_rotary_plan(_ptr(freq), _ints(axis), freq.shape[0], _ptr(plan)), "wf_rotary_plan")
    return plan


def _plan(plan):
    """Address and pairs of a plan on the GPU (None and 0 where there is none)."""
    if plan is None:
        return None, 0
    shape = plan.shape
    if len(shape) != 2 or shape[1] != 2 or plan.dtype != torch.int64 or not plan.is_contiguous():
        raise ValueError("expected a plan of wf_rotary_plan")
    return plan.data_ptr(), shape[0]


def _positions(pos, batch: int, rows: int):
    """Address and axes of positions [axes, B, rows] (None and 0 where there are none)."""
    if pos is None:
        return None, 0
    shape = pos.shape
    if len(shape) != 3 or shape[1] != batch or shape[2] != rows:
        raise ValueError("positions must be [axes, B, rows]")
    return _ints(pos), shape[0]


def wf_rotary_apply(Q, K, plan, pos, Qout, Kout, adjacent: bool = False, stream=None) -> None:
    """Q [B, Hq, rows, d] and K [B, Hk, rows, d] (None: Q alone) rotated by pos
    [axes, B, rows] into Qout and Kout, which may be Q and K (see the C header)."""
    _on_gpu(Q, K, plan, pos, Qout, Kout)
    shape, dtype = Q.shape, Q.dtype
    dq, do = _desc(shape, Q.stride(), dtype), _desc(Qout.shape, Qout.stride(), Qout.dtype)
    dk = dl = k = l = None
    if K is not None and Kout is not None:
        dk, dl = _desc(K.shape, K.stride(), K.dtype), _desc(Kout.shape, Kout.stride(), Kout.dtype)
        k, l = K.data_ptr(), Kout.data_ptr()
    elif K is not Kout:
        raise ValueError("keys and their outputs are given together")
    at, pairs = _plan(plan)
    where, axes = _positions(pos, shape[0], shape[2])
    _check(lib().wf_rotary_apply(Q.data_ptr(), dq, k, dk, at, pairs, adjacent, where, axes, Qout.data_ptr(), do, l, dl,
                                 _stream(stream)), "wf_rotary_apply")


def _table(pages, batch: int):
    """Address and entries a sequence of a page table [B, entries]."""
    shape = pages.shape
    if len(shape) != 2 or shape[0] != batch:
        raise ValueError("a page table has a row a sequence")
    return _ints(pages), shape[1]


def wf_paged_append(Knew, Vnew, K, V, pages, start, Ks=None, Vs=None, fmt=None, rows=None, count=None, plan=None,
                    pos=None, adjacent: bool = False, stream=None) -> None:
    """Knew (and Vnew) [B, H, rows, d] into the pages of K (and V) [pages, H,
    page rows, d] from place start [B] on by the table pages [B, entries] (see
    the C header).  fmt: K and V are codes with scales Ks, Vs.  rows [B, m]: those
    new rows; count [B]: how many of them.  plan: the keys are rotated by pos
    [axes, B, rows], or by their place."""
    _on_gpu(Knew, Vnew, K, V, pages, start, Ks, Vs, rows, count, plan, pos)
    dn, dk = _pair_desc(Knew, Vnew, "Knew and Vnew"), _pair_desc(K, V, "K and V", fmt)
    B, n = dn.batch, dn.seq
    m = n
    if rows is not None:
        if rows.dim() != 2 or rows.shape[0] != B:
            raise ValueError("rows must be [B, m]")
        m = rows.shape[1]
    if start.numel() != B or (count is not None and count.numel() != B):
        raise ValueError("start and count must have an entry a sequence")
    at, pairs = _plan(plan)
    where, axes = _positions(pos, B, n)
    table, entries = _table(pages, B)
    _check(lib().wf_paged_append(Knew.data_ptr(), _ptr(Vnew), dn, _ints(rows), m, _ints(start), _ints(count), at, pairs,
                                 adjacent, where, axes, K.data_ptr(), _ptr(V), _ptr(Ks), _ptr(Vs), dk,
                                 0 if Ks is None else _scales(Ks, Vs), table, entries, _stream(stream)),
           "wf_paged_append")


def wf_tree_attn_workspace_bytes(Q: torch.Tensor, K: torch.Tensor, n: int, n_t: int, fmt=None) -> int:
    return int(lib().wf_tree_attn_workspace_bytes(desc(Q), _pair_desc(K, None, "", fmt), n, n_t))


def wf_tree_attn(Q, K, V, pages, n: int, Kt, Vt, O, ws, cache_len=None, tree_len=None, mask=None, Ks=None, Vs=None,
                 fmt=None, scale: float = 0.0, stream=None) -> None:
    """Attention of Q [B, Hq, q, d] over the first n rows, or cache_len [B] of
    them, that the table pages [B, entries] finds in the pool K, V [pages, H, page
    rows, d], and over the drafted rows Kt, Vt [B, H, n_t, d] (None: none), the first
    tree_len [B] of them, that mask [B, q, words] lets each query row see (see the C
    header).  fmt: K and V are codes, with scales Ks and Vs."""
    _on_gpu(Q, K, V, pages, Kt, Vt, O, ws, cache_len, tree_len, mask, Ks, Vs)
    dq, do = _desc(Q.shape, Q.stride(), Q.dtype), _desc(O.shape, O.stride(), O.dtype)
    dk = _pair_desc(K, V, "K and V", fmt)
    dt, n_t = None, 0
    if (Kt is None) != (Vt is None):
        raise ValueError("drafted keys and values are given together")
    if Kt is not None:
        dt = _pair_desc(Kt, Vt, "Kt and Vt")
        n_t = dt.seq
    B = dq.batch
    if fmt is not None:
        if Ks is None or Vs is None or _scales(Ks, Vs) < dk.batch * dk.heads * dk.seq * (dk.head_dim // 32):
            raise ValueError("a quantised cache needs the scales of its K and V")
    if (cache_len is not None and cache_len.numel() != B) or (tree_len is not None and tree_len.numel() != B):
        raise ValueError("lengths must have an entry a sequence")
    if mask is not None and tuple(mask.shape) != (B, dq.seq, (n_t + 31) // 32):
        raise ValueError("the mask must be [B, q, words of 32 drafted rows]")
    table, entries = _table(pages, B)
    _check(lib().wf_tree_attn(Q.data_ptr(), dq, K.data_ptr(), V.data_ptr(), dk, _ptr(Ks), _ptr(Vs), table, entries, n,
                              _ints(cache_len), _ptr(Kt), _ptr(Vt), dt, _ints(tree_len), _ints(mask), O.data_ptr(), do,
                              scale, ws.data_ptr(), ws.nbytes, _stream(stream)), "wf_tree_attn")


def wf_workspace_status(ws: torch.Tensor, stream=None):
    """Raise WfError(WF_ERR_TIMEOUT) if a bounded device wait of the fused
    step kernel gave up since the last check (synchronising)."""
    _check(lib().wf_workspace_status(_ptr(ws), _stream(stream)), "wf_workspace_status")


def wf_testing_set_wait_failure(stall: bool, wait_limit_cycles: int = 0):
    """Test-only (include/wf_testing.h): make the tensor-core kernels' first
    wait stall (a barrier nothing completes) and bound the waits that can give
    up by wait_limit_cycles (0: the default bound).  Reset with (False, 0)."""
    _check(lib().wf_testing_set_wait_failure(int(bool(stall)), int(wait_limit_cycles)),
           "wf_testing_set_wait_failure")


def wf_testing_prefix_plan(q: wf_tensor, kv: wf_tensor, k: int, n_g: int) -> wf_testing_plan:
    """Test-only (include/wf_testing.h): how a wf_prefix_attn call of these
    shapes would be run."""
    plan = wf_testing_plan()
    _check(lib().wf_testing_prefix_plan(q, kv, k, n_g, plan), "wf_testing_prefix_plan")
    return plan
