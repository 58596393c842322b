"""ctypes binding of libe0m4: argument marshalling only.

Every function has the name of the C entry point it calls (see
``include/e0m4.h``) and does nothing but turn torch tensors into device
pointers and sizes; all arithmetic happens in the HIP kernels.  torch is used
for device memory and streams.  There is no CPU fallback: if the shared
library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libe0m4.so")

_lib = None


class E0M4KV4Shape(NamedTuple):
    """Sizes of a key/value cache in E0M4 codes (see include/e0m4.h)."""
    batch: int
    kv_heads: int
    capacity: int
    dim: int
    group: int


class _KV4Shape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("kv_heads", ctypes.c_int64), ("capacity", ctypes.c_int64), ("dim", ctypes.c_int),
                ("group", ctypes.c_int)]


class _KV4Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_ld", ctypes.c_int64), ("row_ld", ctypes.c_int64), ("head_ld", ctypes.c_int64)]


class _KV4Mask(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_ld", ctypes.c_int64), ("row_ld", ctypes.c_int64), ("rows", ctypes.c_int64)]


class E0M4Error(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().e0m4_strerror(code).decode()
        if code == -6:
            msg += ": " + lib().e0m4_last_hip_error().decode()
        super().__init__("%s failed (%d): %s" % (where, code, msg))


def lib() -> ctypes.CDLL:
    """Load libe0m4.so (built in-tree by ``paper_2403_20041_amd.build``); fails loudly if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            "libe0m4.so is not built: run `python -m paper_2403_20041_amd.build` (needs hipcc); "
            "there is no fallback path")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, ci, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
    L.e0m4_abi_version.restype = ci
    L.e0m4_abi_version.argtypes = []
    L.e0m4_strerror.restype = ctypes.c_char_p
    L.e0m4_strerror.argtypes = [ci]
    L.e0m4_last_hip_error.restype = ctypes.c_char_p
    L.e0m4_last_hip_error.argtypes = []
    L.e0m4_codes_bytes.restype = sz
    L.e0m4_codes_bytes.argtypes = [i64, i64, ci]
    L.e0m4_params_elems.restype = sz
    L.e0m4_params_elems.argtypes = [i64, i64, ci]
    L.e0m4_workspace_bytes.restype = sz
    L.e0m4_workspace_bytes.argtypes = [i64, i64, i64, ci]
    L.e0m4_quantize.restype = ci
    L.e0m4_quantize.argtypes = [vp, i64, i64, ci, vp, vp, vp, vp]
    L.e0m4_encode.restype = ci
    L.e0m4_encode.argtypes = [vp, i64, i64, ci, vp, vp, vp, vp]
    L.e0m4_dequant.restype = ci
    L.e0m4_dequant.argtypes = [vp, vp, vp, i64, i64, ci, vp, vp]
    L.e0m4_unpack_codes.restype = ci
    L.e0m4_unpack_codes.argtypes = [vp, i64, i64, ci, vp, vp]
    L.e0m4_matmul.restype = ci
    L.e0m4_matmul.argtypes = [vp, i64, vp, vp, vp, i64, i64, ci, vp, vp, sz, vp]
    L.e0m4_matmul_static.restype = ci
    L.e0m4_matmul_static.argtypes = [vp, i64, vp, i64, i64, ci, vp, vp]
    L.e0m4_fused_workspace_bytes.restype = sz
    L.e0m4_fused_workspace_bytes.argtypes = [i64, i64, i64, ci, ci, ci]
    L.e0m4_fused_workspace_best_bytes.restype = sz
    L.e0m4_fused_workspace_best_bytes.argtypes = [i64, i64, i64, ci, ci, ci]
    for name in ("e0m4_matmul_fused", "e0m4_matmul_fused_best"):
        getattr(L, name).restype = ci
        getattr(L, name).argtypes = [vp, i64, vp, ctypes.c_float, vp, i64, i64, ci, ci, vp, vp, vp, sz, vp]
    L.e0m8_codes_bytes.restype = sz
    L.e0m8_codes_bytes.argtypes = [i64, i64, ci]
    L.e0m8_quantize.restype = ci
    L.e0m8_quantize.argtypes = [vp, i64, i64, ci, vp, vp, vp, vp]
    L.e0m8_dequant.restype = ci
    L.e0m8_dequant.argtypes = [vp, i64, i64, ci, vp, vp]
    L.e0m8_unpack_codes.restype = ci
    L.e0m8_unpack_codes.argtypes = [vp, i64, i64, ci, vp, vp]
    L.e0m8_matmul.restype = ci
    L.e0m8_matmul.argtypes = [vp, i64, vp, i64, i64, ci, vp, vp, sz, vp]
    L.e0m8_fused_workspace_bytes.restype = sz
    L.e0m8_fused_workspace_bytes.argtypes = [i64, i64, i64, ci, ci, ci]
    L.e0m8_matmul_fused.restype = ci
    L.e0m8_matmul_fused.argtypes = [vp, i64, vp, ctypes.c_float, vp, i64, i64, ci, ci, vp, vp, vp, sz, vp]
    L.e0m8_workspace_bytes.restype = sz
    L.e0m8_workspace_bytes.argtypes = [i64, i64, i64, ci]
    L.e0m4_kv_append.restype = ci
    L.e0m4_kv_append.argtypes = [vp, i64, i64, vp, i64, i64, vp, vp]
    shp, rws, msk = ctypes.POINTER(_KV4Shape), ctypes.POINTER(_KV4Rows), ctypes.POINTER(_KV4Mask)
    L.e0m4_kv4_bytes.restype = sz
    L.e0m4_kv4_bytes.argtypes = [shp]
    L.e0m4_kv4_append.restype = ci
    L.e0m4_kv4_append.argtypes = [vp, shp, rws, rws, ci, i64, vp, vp, vp]
    L.e0m4_kv4_read.restype = ci
    L.e0m4_kv4_read.argtypes = [vp, shp, vp, vp, i64, vp, vp, vp]
    L.e0m4_kv4_attention_workspace_bytes.restype = sz
    L.e0m4_kv4_attention_workspace_bytes.argtypes = [shp, i64, i64, ci]
    L.e0m4_kv4_attention.restype = ci
    L.e0m4_kv4_attention.argtypes = [rws, ci, i64, i64, vp, shp, vp, vp, ci, i64, msk, vp, vp, vp, sz, vp]
    L.e0m4_kv4_evict.restype = ci
    L.e0m4_kv4_evict.argtypes = [vp, shp, vp, vp, i64, i64, vp, shp, vp, vp, vp, vp]
    L.e0m4_int4_quantize.restype = ci
    L.e0m4_int4_quantize.argtypes = [vp, i64, i64, ci, vp, vp, vp, vp]
    L.e0m4_int4_dequant.restype = ci
    L.e0m4_int4_dequant.argtypes = [vp, i64, i64, ci, vp, vp]
    L.e0m4_int4_gemv.restype = ci
    L.e0m4_int4_gemv.argtypes = [vp, vp, i64, i64, ci, vp, vp]
    for name in ("e0m3_quantize", "e0m4_bf16_quantize", "e0m4_bf16_encode"):
        getattr(L, name).restype = ci
        getattr(L, name).argtypes = [vp, i64, i64, ci, vp, vp, vp, vp]
    L.e0m3_unpack_codes.restype = ci
    L.e0m3_unpack_codes.argtypes = [vp, i64, i64, ci, vp, vp]
    L.e0m4_bf16_dequant.restype = ci
    L.e0m4_bf16_dequant.argtypes = [vp, i64, i64, ci, vp, vp]
    L.e0m4_bf16_matmul.restype = ci
    L.e0m4_bf16_matmul.argtypes = [vp, i64, vp, i64, i64, ci, vp, vp]
    L.e0m4_set_knob.restype = ci
    L.e0m4_set_knob.argtypes = [ctypes.c_char_p, ci]
    if L.e0m4_abi_version() != 4:
        raise RuntimeError("libe0m4 ABI version mismatch")
    _lib = L
    return L


# The handle of the current device's current stream, without the Stream object that torch.cuda.current_stream() makes.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None and _current_device is not None:
            return _raw_stream(_current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _can_allocate(device, stream) -> bool:
    """Whether _empty can make a buffer for `stream`."""
    return stream is None or hasattr(stream, "cuda_stream") or int(stream) == torch.cuda.current_stream(device).cuda_stream


def _empty(shape, dtype, device, stream, what: str):
    """torch.empty for a buffer that the kernels enqueued on `stream` will use.  The caching allocator ties a
    block to the stream that was current when it was allocated, so the buffer is allocated with `stream`
    current; a raw stream handle that is not the current stream cannot be made current here, and the caller
    must then own the buffer."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not _can_allocate(device, stream):
        raise ValueError("%s: pass a caller-owned tensor when `stream` is a raw handle other than torch's current stream"
                         % what)
    if hasattr(stream, "cuda_stream"):
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=device)
    return torch.empty(shape, dtype=dtype, device=device)


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _check(rc: int, where: str):
    if rc != 0:
        raise E0M4Error(rc, where)


def _need(t: torch.Tensor, dtype, shape, name: str):
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or not t.is_cuda:
        raise ValueError("%s must be a contiguous cuda %s tensor of shape %s, got %s %s on %s"
                         % (name, dtype, tuple(shape), t.dtype, tuple(t.shape), t.device))


def e0m4_codes_bytes(N: int, K: int, group: int) -> int:
    return lib().e0m4_codes_bytes(N, K, group)


def e0m4_params_elems(N: int, K: int, group: int) -> int:
    return lib().e0m4_params_elems(N, K, group)


def e0m4_workspace_bytes(M: int, N: int, K: int, group: int) -> int:
    return lib().e0m4_workspace_bytes(M, N, K, group)


def e0m4_set_knob(name: str, value: int) -> None:
    _check(lib().e0m4_set_knob(name.encode(), int(value)), "e0m4_set_knob")


def alloc_packed(N: int, K: int, group: int, device):
    """Uninitialised output buffers for e0m4_quantize: (codes u8, scales f16 [N,K/G], bias f16 [N,K/G])."""
    codes = torch.empty(max(e0m4_codes_bytes(N, K, group), 16), dtype=torch.uint8, device=device)
    scales = torch.empty((N, K // group), dtype=torch.float16, device=device)
    bias = torch.empty((N, K // group), dtype=torch.float16, device=device)
    return codes, scales, bias


def e0m4_quantize(W: torch.Tensor, group: int, out=None, stream=None):
    """W [N,K] fp16 -> (codes, scales, bias); see include/e0m4.h."""
    N, K = W.shape
    _need(W, torch.float16, (N, K), "W")
    codes, scales, bias = out if out is not None else alloc_packed(N, K, group, W.device)
    _check(lib().e0m4_quantize(_ptr(W), N, K, group, _ptr(codes), _ptr(scales), _ptr(bias), _stream(stream)),
           "e0m4_quantize")
    return codes, scales, bias


def e0m4_encode(W: torch.Tensor, scales: torch.Tensor, bias: torch.Tensor, group: int, codes=None, stream=None):
    N, K = W.shape
    _need(W, torch.float16, (N, K), "W")
    _need(scales, torch.float16, (N, K // group), "scales")
    _need(bias, torch.float16, (N, K // group), "bias")
    if codes is None:
        codes = torch.empty(max(e0m4_codes_bytes(N, K, group), 16), dtype=torch.uint8, device=W.device)
    _check(lib().e0m4_encode(_ptr(W), N, K, group, _ptr(scales), _ptr(bias), _ptr(codes), _stream(stream)),
           "e0m4_encode")
    return codes


def e0m4_dequant(codes, scales, bias, N: int, K: int, group: int, out=None, stream=None) -> torch.Tensor:
    if out is None:
        out = torch.empty((N, K), dtype=torch.float16, device=codes.device)
    _need(out, torch.float16, (N, K), "out")
    _check(lib().e0m4_dequant(_ptr(codes), _ptr(scales), _ptr(bias), N, K, group, _ptr(out), _stream(stream)),
           "e0m4_dequant")
    return out


def e0m4_unpack_codes(codes, N: int, K: int, group: int, out=None, stream=None) -> torch.Tensor:
    if out is None:
        out = torch.empty((N, K), dtype=torch.uint8, device=codes.device)
    _need(out, torch.uint8, (N, K), "out")
    _check(lib().e0m4_unpack_codes(_ptr(codes), N, K, group, _ptr(out), _stream(stream)), "e0m4_unpack_codes")
    return out


def e0m4_matmul(X, codes, scales, bias, N: int, K: int, group: int, out=None, workspace=None, stream=None):
    """Y [M,N] fp16 = X [M,K] fp16 times the dequantised weights, transposed."""
    M = X.shape[0]
    _need(X, torch.float16, (M, K), "X")
    if out is None:
        out = _empty((M, N), torch.float16, X.device, stream, "out")
    else:
        _need(out, torch.float16, (M, N), "out")
    # (one row never needs a workspace; two or more may)
    if workspace is None and M > 1:
        need = e0m4_workspace_bytes(M, N, K, group)
        if need > 0:
            workspace = _empty(need, torch.uint8, X.device, stream, "workspace")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().e0m4_matmul(_ptr(X), M, _ptr(codes), _ptr(scales), _ptr(bias), N, K, group, _ptr(out),
                             _ptr(workspace), ws_bytes, _stream(stream)), "e0m4_matmul")
    return out


E0M4_STATIC_SCRATCH_BYTES = 128 << 20


def e0m4_matmul_static(X, codes, N: int, K: int, group: int, out, stream=None):
    """e0m4_matmul without a workspace argument: the library's own fixed scratch array serves the split along
    K.  `out` is required, so that the call itself allocates nothing."""
    M = X.shape[0]
    _need(X, torch.float16, (M, K), "X")
    _need(out, torch.float16, (M, N), "out")
    _check(lib().e0m4_matmul_static(_ptr(X), M, _ptr(codes), N, K, group, _ptr(out), _stream(stream)),
           "e0m4_matmul_static")
    return out


E0M4_EPILOGUE_NONE = 0
E0M4_EPILOGUE_SWIGLU = 1


def e0m4_fused_workspace_bytes(M: int, N: int, K: int, group: int, with_rmsnorm: bool, epilogue: int) -> int:
    return lib().e0m4_fused_workspace_bytes(M, N, K, group, 1 if with_rmsnorm else 0, epilogue)


def _capturing(stream) -> bool:
    if stream is None or not hasattr(stream, "cuda_stream"):
        return torch.cuda.is_current_stream_capturing()
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


def _chunks_are_shorter(M: int, n_out: int, K: int) -> bool:
    """Of a call of 17 to 64 rows with an rms-norm that is issued by itself and may do without a workspace: with one it is shorter on the GPU, and
    by a launch and an allocation 3 - 4 us longer on the host.  In row chunks it takes 8 - 10 us where these (one for 16 rows and
    16 columns) are no more than the compute units and rows of X not long, less than the host does then (M = 20, 2048 x 2048 8.3
    and 10.1 - 12.8 us, replayed in a graph 8.5 and 7.1); else 12 - 35 (M = 45, 4608 x 4096 19.7 and 11.9; M = 18, gated 2304 x 6272
    15.7 and 12.5)."""
    return -(-M // 16) * -(-n_out // 16) <= 256 and K <= 4608


def e0m4_matmul_fused(X, codes, N: int, K: int, group: int, rms_gamma=None, rms_eps: float = 0.0,
                      epilogue: int = E0M4_EPILOGUE_NONE, residual=None, out=None, workspace=None, stream=None):
    """The matmul with rms-norm on X, the SiLU-gated product of the two output halves and a residual add
    folded in (each optional; see include/e0m4.h).  Y is [M, N/2] with the gated epilogue, else [M, N]."""
    M = X.shape[0]
    _need(X, torch.float16, (M, K), "X")
    n_out = N // 2 if epilogue == E0M4_EPILOGUE_SWIGLU else N
    if rms_gamma is not None:
        _need(rms_gamma, torch.float16, (K,), "rms_gamma")
    if residual is not None:
        _need(residual, torch.float16, (M, n_out), "residual")
    if out is None:
        out = _empty((M, n_out), torch.float16, X.device, stream, "out")
    else:
        _need(out, torch.float16, (M, n_out), "out")
    L = lib()
    normed = 0 if rms_gamma is None else 1
    call = L.e0m4_matmul_fused                          # (which writes to a caller's workspace only where one is needed)
    if workspace is None:
        if not _can_allocate(X.device, stream) or (normed and 17 <= M <= 64 and _chunks_are_shorter(M, n_out, K) and not _capturing(stream)):
            need = L.e0m4_fused_workspace_bytes(M, N, K, group, normed, epilogue)     # (0 if it can do without)
        else:
            need = L.e0m4_fused_workspace_best_bytes(M, N, K, group, normed, epilogue)
            call = L.e0m4_matmul_fused_best
        if need > 0:
            workspace = _empty(need, torch.uint8, X.device, stream, "workspace")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(call(_ptr(X), M, _ptr(rms_gamma), float(rms_eps), _ptr(codes), N, K, group, epilogue, _ptr(residual), _ptr(out),
                _ptr(workspace), ws_bytes, _stream(stream)), "e0m4_matmul_fused")
    return out


def e0m4_kv_append(cache, new_rows, position_ids, stream=None):
    """cache [max_seq, row] fp16 is updated in place: cache[position_ids[i]] = new_rows[i].  new_rows may be a
    column slice of a wider matrix (last dimension contiguous); position_ids is an int64 device tensor."""
    max_seq, row = cache.shape
    n_new = new_rows.shape[0]
    if cache.dtype != torch.float16 or new_rows.dtype != torch.float16 or position_ids.dtype != torch.int64:
        raise TypeError("e0m4_kv_append: cache and new_rows must be float16, position_ids int64")
    if not cache.is_contiguous() or new_rows.shape[1] != row or new_rows.stride(1) != 1 or \
            not position_ids.is_contiguous() or position_ids.numel() != n_new:
        raise ValueError("e0m4_kv_append: bad shapes or strides")
    _check(lib().e0m4_kv_append(_ptr(cache), max_seq, row, _ptr(new_rows), n_new, new_rows.stride(0),
                                _ptr(position_ids), _stream(stream)), "e0m4_kv_append")
    return cache


# ---- key/value cache in E0M4 codes (see include/e0m4.h) ----------------------------------------------

_KV4_DTYPES = {torch.float16: 0, torch.bfloat16: 1}


@functools.lru_cache(maxsize=256)
def _kv4_shape(shape):
    """(the C struct, bytes of a cache) of a shape: both are its alone, and a call asks for them each time."""
    c = _KV4Shape(*shape)
    return c, lib().e0m4_kv4_bytes(c)


def _kv4_per_sequence(t, shape, name: str, where: str):
    """Device int32 [batch], or None."""
    if t is None:
        return 0
    if t.dtype is not torch.int32 or t.shape != (shape[0],) or not t.is_contiguous() or not t.is_cuda:
        raise ValueError("%s: %s must be a contiguous cuda int32 tensor of shape (%d,), got %s %s on %s"
                         % (where, name, shape[0], t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


def _kv4_rows(t, n: int, heads: int, shape, name: str, where: str):
    """A [batch, n, heads, dim] tensor of any strides but the last."""
    if t.dtype not in _KV4_DTYPES:
        raise TypeError("%s: %s must be float16 or bfloat16" % (where, name))
    batch, dim = shape[0], shape[3]
    ld = t.stride()
    if t.shape != (batch, n, heads, dim) or not t.is_cuda or (ld[3] != 1 and t.numel()):
        raise ValueError("%s: %s must be a cuda tensor of shape %s whose last dimension is contiguous, got %s with strides %s on %s"
                         % (where, name, (batch, n, heads, dim), tuple(t.shape), ld, t.device))
    # (the stride of a dimension of one is never walked, whatever it says)
    return _KV4Rows(t.data_ptr(), ld[0] if batch > 1 else 0, ld[1] if n > 1 else 0, ld[2] if heads > 1 else 0)


def _kv4_cache(cache, shape, name: str, where: str):
    c, need = _kv4_shape(shape)
    if cache.dtype is not torch.uint8 or not cache.is_contiguous() or not cache.is_cuda or cache.numel() < need:
        raise ValueError("%s: %s must be a contiguous cuda uint8 tensor of at least %d bytes" % (where, name, need))
    return c


def e0m4_kv4_bytes(shape: E0M4KV4Shape) -> int:
    return _kv4_shape(shape)[1]


def e0m4_kv4_attention_workspace_bytes(shape: E0M4KV4Shape, heads: int, n_new: int, with_weights: bool = False) -> int:
    return lib().e0m4_kv4_attention_workspace_bytes(_kv4_shape(shape)[0], heads, n_new, 1 if with_weights else 0)


def e0m4_kv4_alloc(shape: E0M4KV4Shape, device) -> torch.Tensor:
    """Memory for a cache (uninitialised: rows count once they are appended)."""
    need = e0m4_kv4_bytes(shape)
    if need == 0 and shape.batch * shape.kv_heads * shape.capacity != 0:
        raise ValueError("e0m4_kv4_alloc: unsupported shape %s" % (shape,))
    return torch.empty(max(need, 16), dtype=torch.uint8, device=device)


def e0m4_kv4_append(cache, shape: E0M4KV4Shape, keys, values, starts, counts=None, stream=None):
    """Rows of keys and values [batch, n, kv_heads, dim] (fp16 or bf16, any strides but the last) are quantised into the
    cache from row starts[b] on, the first counts[b] of them (None: all)."""
    where = "e0m4_kv4_append"
    n = keys.shape[1]
    k = _kv4_rows(keys, n, shape[1], shape, "keys", where)
    v = _kv4_rows(values, n, shape[1], shape, "values", where)
    if keys.dtype != values.dtype:
        raise TypeError("e0m4_kv4_append: keys and values must be of one type")
    _check(lib().e0m4_kv4_append(_ptr(cache), _kv4_cache(cache, shape, "cache", where), k, v, _KV4_DTYPES[keys.dtype], n,
                                 _kv4_per_sequence(starts, shape, "starts", where), _kv4_per_sequence(counts, shape, "counts", where),
                                 _stream(stream)), where)
    return cache


def e0m4_kv4_read(cache, shape: E0M4KV4Shape, lengths, rows: int, first=None, stream=None):
    """(keys, values) fp16 [batch, rows, kv_heads, dim]: what the codes of rows first[b] + i stand for, zeros from lengths[b] on."""
    where = "e0m4_kv4_read"
    s = _kv4_cache(cache, shape, "cache", where)
    size = (shape.batch, max(rows, 0), shape.kv_heads, shape.dim)
    device = cache.device
    keys = _empty(size, torch.float16, device, stream, "keys")
    values = _empty(size, torch.float16, device, stream, "values")
    _check(lib().e0m4_kv4_read(_ptr(cache), s, _kv4_per_sequence(lengths, shape, "lengths", where),
                               _kv4_per_sequence(first, shape, "first", where), rows, _ptr(keys), _ptr(values), _stream(stream)), where)
    return keys, values


def e0m4_kv4_attention(queries, cache, shape: E0M4KV4Shape, lengths, counts=None, causal: bool = True, window: int = 0, mask=None,
                       weights=None, out=None, workspace=None, stream=None):
    """Attention of the newest tokens' queries [batch, n, heads, dim] over the cache; see include/e0m4.h.  mask: bool
    [batch, n, rows] (dimensions of one are shared), weights: fp32 [batch, kv_heads, capacity], added to in place."""
    where = "e0m4_kv4_attention"
    batch, n, heads, dim = queries.shape
    q = _kv4_rows(queries, n, heads, shape, "queries", where)
    s = _kv4_cache(cache, shape, "cache", where)
    m = None
    if mask is not None:
        if mask.dtype != torch.bool or mask.dim() != 3 or mask.shape[0] not in (1, batch) or mask.shape[1] not in (1, n) or \
                (mask.numel() and mask.stride(2) != 1 and mask.shape[2] != 1) or not mask.is_cuda:
            raise ValueError("e0m4_kv4_attention: mask must be a cuda bool tensor [batch, n, rows] with its rows side by side")
        m = _KV4Mask(_ptr(mask), *(mask.stride(i) if mask.shape[i] > 1 else 0 for i in range(2)), mask.shape[2])
    if weights is not None:
        _need(weights, torch.float32, (shape.batch, shape.kv_heads, shape.capacity), "weights")
    if out is None:
        out = _empty((batch, n, heads, dim), queries.dtype, queries.device, stream, "out")
    else:
        _need(out, queries.dtype, (batch, n, heads, dim), "out")
    if workspace is None:
        need = lib().e0m4_kv4_attention_workspace_bytes(s, heads, n, 0 if weights is None else 1)
        if need > 0:
            workspace = _empty(need, torch.uint8, queries.device, stream, "workspace")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().e0m4_kv4_attention(q, _KV4_DTYPES[queries.dtype], heads, n, _ptr(cache), s,
                                    _kv4_per_sequence(lengths, shape, "lengths", where), _kv4_per_sequence(counts, shape, "counts", where),
                                    1 if causal else 0, window, m, _ptr(weights), _ptr(out), _ptr(workspace), ws_bytes, _stream(stream)),
           where)
    return out


def e0m4_kv4_evict(cache, shape: E0M4KV4Shape, received, lengths, budget: int, recent: int, small, small_shape: E0M4KV4Shape,
                   stream=None):
    """The rows that received most attention, and the newest `recent`, move to the cache `small`.  Returns (kept int32
    [batch, kv_heads, budget], lengths int32 [batch], received fp32 [batch, kv_heads, budget]); see include/e0m4.h."""
    where = "e0m4_kv4_evict"
    s, o = _kv4_cache(cache, shape, "cache", where), _kv4_cache(small, small_shape, "small", where)
    _need(received, torch.float32, (shape.batch, shape.kv_heads, shape.capacity), "received")
    size = (shape.batch, shape.kv_heads, max(budget, 0))
    kept = _empty(size, torch.int32, cache.device, stream, "kept")
    lengths_out = _empty((shape.batch,), torch.int32, cache.device, stream, "lengths")
    received_out = _empty(size, torch.float32, cache.device, stream, "received")
    _check(lib().e0m4_kv4_evict(_ptr(cache), s, _ptr(received), _kv4_per_sequence(lengths, shape, "lengths", where), budget, recent,
                                _ptr(small), o, _ptr(kept), _ptr(lengths_out), _ptr(received_out), _stream(stream)), where)
    return kept, lengths_out, received_out


# ---- E0M8, the 8-bit member of the family (see include/e0m4.h) ---------------------------------------

def e0m8_codes_bytes(N: int, K: int, group: int) -> int:
    return lib().e0m8_codes_bytes(N, K, group)


def e0m8_quantize(W: torch.Tensor, group: int, stream=None):
    """W [N,K] fp16 -> (codes packed uint8, scales [N,K/group] fp16, bias [N,K/group] fp16)."""
    N, K = W.shape
    _need(W, torch.float16, (N, K), "W")
    nbytes = e0m8_codes_bytes(N, K, group)
    if nbytes == 0 and N * K > 0:
        raise ValueError("e0m8_quantize: unsupported shape or group")
    codes = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=W.device)
    scales = torch.empty((N, max(K // group, 1)), dtype=torch.float16, device=W.device)
    bias = torch.empty_like(scales)
    _check(lib().e0m8_quantize(_ptr(W), N, K, group, _ptr(codes), _ptr(scales), _ptr(bias), _stream(stream)),
           "e0m8_quantize")
    return codes, scales, bias


def e0m8_dequant(codes, N: int, K: int, group: int, out=None, stream=None) -> torch.Tensor:
    if out is None:
        out = torch.empty((N, K), dtype=torch.float16, device=codes.device)
    _need(out, torch.float16, (N, K), "out")
    _check(lib().e0m8_dequant(_ptr(codes), N, K, group, _ptr(out), _stream(stream)), "e0m8_dequant")
    return out


def e0m8_unpack_codes(codes, N: int, K: int, group: int, stream=None) -> torch.Tensor:
    out = torch.empty((N, K), dtype=torch.uint8, device=codes.device)
    _check(lib().e0m8_unpack_codes(_ptr(codes), N, K, group, _ptr(out), _stream(stream)), "e0m8_unpack_codes")
    return out


def e0m8_workspace_bytes(M: int, N: int, K: int, group: int) -> int:
    return lib().e0m8_workspace_bytes(M, N, K, group)


def e0m8_matmul(X, codes, N: int, K: int, group: int, out=None, workspace=None, stream=None) -> torch.Tensor:
    """Y [M,N] fp16 = X [M,K] fp16 times the dequantised 8-bit weights, transposed."""
    M = X.shape[0]
    _need(X, torch.float16, (M, K), "X")
    if out is None:
        out = _empty((M, N), torch.float16, X.device, stream, "out")
    else:
        _need(out, torch.float16, (M, N), "out")
    need = e0m8_workspace_bytes(M, N, K, group)
    if workspace is None and need > 0:
        workspace = _empty(need, torch.uint8, X.device, stream, "workspace")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().e0m8_matmul(_ptr(X), M, _ptr(codes), N, K, group, _ptr(out), _ptr(workspace), ws_bytes,
                             _stream(stream)), "e0m8_matmul")
    return out


def e0m8_matmul_fused(X, codes, N: int, K: int, group: int, rms_gamma=None, rms_eps: float = 0.0,
                      epilogue: int = E0M4_EPILOGUE_NONE, residual=None, out=None, workspace=None, stream=None):
    """e0m4_matmul_fused on 8-bit codes."""
    M = X.shape[0]
    _need(X, torch.float16, (M, K), "X")
    n_out = N // 2 if epilogue == E0M4_EPILOGUE_SWIGLU else N
    if rms_gamma is not None:
        _need(rms_gamma, torch.float16, (K,), "rms_gamma")
    if residual is not None:
        _need(residual, torch.float16, (M, n_out), "residual")
    if out is None:
        out = _empty((M, n_out), torch.float16, X.device, stream, "out")
    else:
        _need(out, torch.float16, (M, n_out), "out")
    need = lib().e0m8_fused_workspace_bytes(M, N, K, group, 1 if rms_gamma is not None else 0, epilogue)
    if workspace is None and need > 0:
        workspace = _empty(need, torch.uint8, X.device, stream, "workspace")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().e0m8_matmul_fused(_ptr(X), M, _ptr(rms_gamma), float(rms_eps), _ptr(codes), N, K, group, epilogue,
                                   _ptr(residual), _ptr(out), _ptr(workspace), ws_bytes, _stream(stream)),
           "e0m8_matmul_fused")
    return out


# ---- INT4 twin (see include/e0m4.h) ------------------------------------------------------------

def e0m4_int4_quantize(W: torch.Tensor, group: int, out=None, stream=None):
    """W [N,K] fp16 -> (codes, scales, zeros) in the INT4 comparison format."""
    N, K = W.shape
    _need(W, torch.float16, (N, K), "W")
    codes, scales, zeros = out if out is not None else alloc_packed(N, K, group, W.device)
    _check(lib().e0m4_int4_quantize(_ptr(W), N, K, group, _ptr(codes), _ptr(scales), _ptr(zeros), _stream(stream)),
           "e0m4_int4_quantize")
    return codes, scales, zeros


def e0m4_int4_dequant(codes, N: int, K: int, group: int, out=None, stream=None) -> torch.Tensor:
    if out is None:
        out = torch.empty((N, K), dtype=torch.float16, device=codes.device)
    _need(out, torch.float16, (N, K), "out")
    _check(lib().e0m4_int4_dequant(_ptr(codes), N, K, group, _ptr(out), _stream(stream)), "e0m4_int4_dequant")
    return out


def e0m4_int4_gemv(X, codes, N: int, K: int, group: int, out=None, stream=None) -> torch.Tensor:
    """Y [1,N] fp16 = X [1,K] fp16 times the dequantised INT4 weights, transposed."""
    _need(X, torch.float16, (1, K), "X")
    if out is None:
        out = torch.empty((1, N), dtype=torch.float16, device=X.device)
    _need(out, torch.float16, (1, N), "out")
    _check(lib().e0m4_int4_gemv(_ptr(X), _ptr(codes), N, K, group, _ptr(out), _stream(stream)), "e0m4_int4_gemv")
    return out


# ---- E0M3 (3-bit codes in 4-bit slots) and E0M4 on bfloat16 (see include/e0m4.h) -----------------

def e0m3_quantize(W: torch.Tensor, group: int, stream=None):
    """W [N,K] fp16 -> (codes, scales, bias); the buffer is read by e0m4_dequant / e0m4_matmul unchanged."""
    N, K = W.shape
    _need(W, torch.float16, (N, K), "W")
    codes, scales, bias = alloc_packed(N, K, group, W.device)
    _check(lib().e0m3_quantize(_ptr(W), N, K, group, _ptr(codes), _ptr(scales), _ptr(bias), _stream(stream)),
           "e0m3_quantize")
    return codes, scales, bias


def e0m3_unpack_codes(codes, N: int, K: int, group: int, stream=None) -> torch.Tensor:
    out = torch.empty((N, K), dtype=torch.uint8, device=codes.device)
    _check(lib().e0m3_unpack_codes(_ptr(codes), N, K, group, _ptr(out), _stream(stream)), "e0m3_unpack_codes")
    return out


def e0m4_bf16_quantize(W: torch.Tensor, group: int, stream=None):
    """W [N,K] bfloat16 -> (codes, scales bf16 [N,K/G], bias bf16 [N,K/G])."""
    N, K = W.shape
    _need(W, torch.bfloat16, (N, K), "W")
    codes = torch.empty(max(e0m4_codes_bytes(N, K, group), 16), dtype=torch.uint8, device=W.device)
    scales = torch.empty((N, K // group), dtype=torch.bfloat16, device=W.device)
    bias = torch.empty((N, K // group), dtype=torch.bfloat16, device=W.device)
    _check(lib().e0m4_bf16_quantize(_ptr(W), N, K, group, _ptr(codes), _ptr(scales), _ptr(bias), _stream(stream)),
           "e0m4_bf16_quantize")
    return codes, scales, bias


def e0m4_bf16_encode(W: torch.Tensor, scales: torch.Tensor, bias: torch.Tensor, group: int, stream=None):
    N, K = W.shape
    _need(W, torch.bfloat16, (N, K), "W")
    _need(scales, torch.bfloat16, (N, K // group), "scales")
    _need(bias, torch.bfloat16, (N, K // group), "bias")
    codes = torch.empty(max(e0m4_codes_bytes(N, K, group), 16), dtype=torch.uint8, device=W.device)
    _check(lib().e0m4_bf16_encode(_ptr(W), N, K, group, _ptr(scales), _ptr(bias), _ptr(codes), _stream(stream)),
           "e0m4_bf16_encode")
    return codes


def e0m4_bf16_dequant(codes, N: int, K: int, group: int, out=None, stream=None) -> torch.Tensor:
    if out is None:
        out = torch.empty((N, K), dtype=torch.bfloat16, device=codes.device)
    _need(out, torch.bfloat16, (N, K), "out")
    _check(lib().e0m4_bf16_dequant(_ptr(codes), N, K, group, _ptr(out), _stream(stream)), "e0m4_bf16_dequant")
    return out


def e0m4_bf16_matmul(X, codes, N: int, K: int, group: int, out=None, stream=None) -> torch.Tensor:
    """Y [M,N] bfloat16 = X [M,K] bfloat16 times the dequantised weights, transposed."""
    M = X.shape[0]
    _need(X, torch.bfloat16, (M, K), "X")
    if out is None:
        out = _empty((M, N), torch.bfloat16, X.device, stream, "out")
    else:
        _need(out, torch.bfloat16, (M, N), "out")
    _check(lib().e0m4_bf16_matmul(_ptr(X), M, _ptr(codes), N, K, group, _ptr(out), _stream(stream)), "e0m4_bf16_matmul")
    return out
