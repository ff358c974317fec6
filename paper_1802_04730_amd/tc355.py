"""Thin binding of libtc355.so: argument marshalling only, in native code (csrc/fast_call.cpp) for the arguments that calls are
made with in earnest and through ctypes for the rest, errors among them.

Every function has the name and argument order of the C entry point in
include/tc355.h.  Tensors are torch CUDA tensors (device memory owned by the
caller); extents are read from their shapes; work is enqueued on torch's
current stream unless ``stream`` (a raw hipStream_t value) is given.  A non-zero
status raises ``TcError``.  There is no CPU fallback: if the library cannot be
loaded the import of this module's functions fails loudly.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import shutil
import struct
import warnings

import torch

from . import build as _build

_LIB = None
_FAST = None  # csrc/fast_call.cpp, from the moment the library is loaded; None where it cannot be built or loaded
_AT = {}  # addresses of the entry points

TC_OK = 0
STATUS_NAMES = {0: "TC_OK", 1: "TC_ERR_NULL", 2: "TC_ERR_SHAPE", 3: "TC_ERR_ALIAS", 4: "TC_ERR_ALIGN",
                5: "TC_ERR_WORKSPACE", 6: "TC_ERR_LAUNCH", 7: "TC_ERR_UNSUPPORTED", 8: "TC_ERR_SCRATCH_LIMIT"}
TC_MLP_STATIC_SCRATCH_BYTES = 8 << 20
# tc355_set_option keys and values (include/tc355.h)
TC_OPT_INT8, TC_OPT_MLP_KERNEL, TC_OPT_MLP_SPIN_LIMIT = 0, 1, 2
TC_INT8_AUTO, TC_INT8_OFF, TC_INT8_TEN, TC_INT8_THIRTEEN = 0, 1, 2, 3
TC_MLP_AUTO, TC_MLP_ROWS, TC_MLP_TILES, TC_MLP_PER_LAYER = 0, 1, 2, 3
# storage types of the operators around experts (tc_type)
TC_F32, TC_BF16, TC_F16 = 0, 1, 2
_TYPES = {torch.float32: TC_F32, torch.bfloat16: TC_BF16, torch.float16: TC_F16}
TC_Q8_BLOCK = 128  # elements of a scale of 8-bit operands

EXPORTS = ["tc_status_string", "tc355_version", "tc355_set_option", "tc355_get_option", "tc355_last_path", "tc_tbmm", "tc_tbmm_ws", "tc_tbmm_workspace_bytes", "tc_mlp_fcrelu", "tc_mlp_fcrelu_workspace_bytes",
           "tc_mlp_fcrelu_static",
           "tc_group_conv", "tc_group_conv_infer", "tc_kron", "tc_sconv2d", "tc_sconv2d_infer", "tc_lut",
           "tc_embed", "tc_embed_grad", "tc_embed_grad_workspace_bytes", "tc_route", "tc_route_workspace_bytes", "tc_route_grad",
           "tc_expert_mm", "tc_expert_mm_grad_x", "tc_expert_mm_grad_w", "tc_expert_mm_grad_w_workspace_bytes", "tc_expert_sum",
           "tc_expert_sum_grad",
           "tc_layer_norm", "tc_layer_norm_grad", "tc_layer_norm_grad_workspace_bytes", "tc_route_balanced", "tc_route_balanced_workspace_bytes",
           "tc_route_balanced_grad", "tc_quantize_rows", "tc_quantize_weights", "tc_expert_mm_q8", "tc_expert_mm_q8_workspace_bytes"]


_RAW_STREAM = getattr(torch._C, "_cuda_getCurrentRawStream", None)


class TcError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s" % (where, status_string(status)))


def lib() -> ctypes.CDLL:
    """Load libtc355.so, building it first if it is missing or older than its sources (and hipcc is there)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = _build.LIB
    if not os.path.exists(path) or (_build.is_stale() and _build.have_hipcc()):
        _build.build(force=True)
    L = ctypes.CDLL(path)
    i64, i32, vp = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p  # (vp also for host arrays: bytes and ctypes arrays pass)
    L.tc_status_string.argtypes = [ctypes.c_int]
    L.tc_status_string.restype = ctypes.c_char_p
    L.tc355_version.restype = ctypes.c_int
    L.tc355_set_option.argtypes = [ctypes.c_int, i64]
    L.tc355_set_option.restype = ctypes.c_int
    L.tc355_get_option.argtypes = [ctypes.c_int]
    L.tc355_get_option.restype = i64
    L.tc355_last_path.restype = ctypes.c_char_p
    L.tc_tbmm.argtypes = [vp, vp, vp, i64, i64, i64, i64, vp]
    L.tc_tbmm.restype = ctypes.c_int
    L.tc_tbmm_ws.argtypes = [vp, vp, vp, i64, i64, i64, i64, vp, ctypes.c_size_t, vp]
    L.tc_tbmm_ws.restype = ctypes.c_int
    L.tc_tbmm_workspace_bytes.argtypes = [i64, i64, i64, i64]
    L.tc_tbmm_workspace_bytes.restype = ctypes.c_size_t
    L.tc_mlp_fcrelu.argtypes = [vp, i64, i32, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    L.tc_mlp_fcrelu.restype = ctypes.c_int
    L.tc_mlp_fcrelu_static.argtypes = [vp, i64, i32, vp, vp, vp, vp, vp]
    L.tc_mlp_fcrelu_static.restype = ctypes.c_int
    L.tc_mlp_fcrelu_workspace_bytes.argtypes = [i64, i32, ctypes.POINTER(i64)]
    L.tc_mlp_fcrelu_workspace_bytes.restype = ctypes.c_size_t
    L.tc_group_conv.argtypes = [vp, vp, vp, vp] + [i64] * 8 + [vp]
    L.tc_group_conv.restype = ctypes.c_int
    L.tc_group_conv_infer.argtypes = [i64, i64, i64, i64, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    L.tc_group_conv_infer.restype = ctypes.c_int
    L.tc_kron.argtypes = [vp, vp, vp, vp] + [i64] * 5 + [vp]
    L.tc_kron.restype = ctypes.c_int
    L.tc_sconv2d.argtypes = [vp, vp, vp, vp] + [i64] * 9 + [vp]
    L.tc_sconv2d.restype = ctypes.c_int
    L.tc_sconv2d_infer.argtypes = [i64] * 6 + [ctypes.POINTER(i64), ctypes.POINTER(i64)]
    L.tc_sconv2d_infer.restype = ctypes.c_int
    L.tc_lut.argtypes = [i32, vp, vp, vp, vp, vp, i64, i64, vp]
    L.tc_lut.restype = ctypes.c_int
    size, f32, kind = ctypes.c_size_t, ctypes.c_float, ctypes.c_int
    for name, args in {"tc_embed": [vp, vp, vp, i64, i64, i64, f32, kind, vp],
                       "tc_embed_grad": [vp, vp, vp, i64, i64, i64, f32, i64, i32, kind, kind, vp, size, vp],
                       "tc_route": [vp] * 6 + [i64, i64, i64, i32, kind, vp, size, vp],
                       "tc_route_grad": [vp] * 4 + [i64, i64, i64, i32, kind, vp],
                       "tc_expert_mm": [vp] * 5 + [i64] * 5 + [i32, kind, vp],
                       "tc_expert_mm_grad_x": [vp] * 5 + [i64] * 4 + [kind, vp],
                       "tc_expert_mm_grad_w": [vp] * 5 + [i64] * 5 + [i32, kind, kind, vp, size, vp],
                       "tc_expert_sum": [vp] * 4 + [i64] * 4 + [kind, vp],
                       "tc_expert_sum_grad": [vp] * 6 + [i64] * 4 + [kind, vp],
                       "tc_layer_norm": [vp] * 4 + [i64, i64, f32, kind, kind, vp],
                       "tc_layer_norm_grad": [vp] * 6 + [i64, i64, f32, i32, kind, kind, vp, size, vp],
                       "tc_route_balanced": [vp] * 7 + [i64] * 5 + [i32, i32, f32, kind, vp, size, vp],
                       "tc_route_balanced_grad": [vp] * 4 + [i64, i64, i64, i32, i32, f32, kind, vp],
                       "tc_quantize_rows": [vp] * 3 + [i64, i64, kind, vp],
                       "tc_quantize_weights": [vp] * 5 + [i64, i64, i64, kind, vp],
                       "tc_expert_mm_q8": [vp] * 8 + [i64] * 5 + [i32, kind, vp, size, vp]}.items():
        getattr(L, name).argtypes = args
        getattr(L, name).restype = ctypes.c_int
    for name, n in (("tc_embed_grad_workspace_bytes", 3), ("tc_route_workspace_bytes", 3), ("tc_expert_mm_grad_w_workspace_bytes", 4),
                    ("tc_layer_norm_grad_workspace_bytes", 2), ("tc_route_balanced_workspace_bytes", 3), ("tc_expert_mm_q8_workspace_bytes", 5)):
        getattr(L, name).argtypes = [i64] * n
        getattr(L, name).restype = size
    _load_fast(L)
    _LIB = L
    return L


def _load_fast(L) -> None:
    """The native calls, built first if they are missing or older than their source (and a compiler is there).  The general path
    does all that they do: what keeps them from being built or loaded here costs host time and nothing else."""
    global _FAST
    try:
        if _build.fast_is_stale():
            if shutil.which(os.environ.get("CXX", "g++")) is None:
                return
            _build.build_fast()
        spec = importlib.util.spec_from_file_location("_fast", _build.FAST)
        fast = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(fast)
    except (RuntimeError, OSError, ImportError) as e:
        warnings.warn("the binding's native calls are not available: calls go through ctypes, some microseconds slower (%s)" % e,
                      RuntimeWarning, stacklevel=3)
        return
    for name in ("tc_tbmm", "tc_tbmm_ws", "tc_mlp_fcrelu", "tc_group_conv", "tc_kron", "tc_sconv2d", "tc_lut", "tc_embed", "tc_embed_grad", "tc_route",
                 "tc_route_grad", "tc_expert_mm", "tc_expert_mm_grad_x", "tc_expert_mm_grad_w", "tc_expert_sum", "tc_expert_sum_grad",
                 "tc_layer_norm", "tc_layer_norm_grad", "tc_route_balanced", "tc_route_balanced_grad", "tc_quantize_rows", "tc_quantize_weights", "tc_expert_mm_q8"):
        _AT[name] = ctypes.cast(getattr(L, name), ctypes.c_void_p).value
    _FAST = fast


def status_string(status: int) -> str:
    return lib().tc_status_string(int(status)).decode()


def tc355_version() -> int:
    return int(lib().tc355_version())


def set_option(key: int, value: int) -> int:
    """Set an option of the calling host thread (tc355_set_option); returns the previous value."""
    old = int(lib().tc355_get_option(int(key)))
    _check(lib().tc355_set_option(int(key), int(value)), "tc355_set_option")
    return old


def get_option(key: int) -> int:
    return int(lib().tc355_get_option(int(key)))


def last_path() -> str:
    """Kernel family chosen by this thread's most recent entry-point call, e.g. "tbmm:lds" (tc355_last_path)."""
    return lib().tc355_last_path().decode()


class option:
    """Context manager: an option of the calling thread for the duration of a block."""

    def __init__(self, key: int, value: int):
        self.key, self.value = key, value

    def __enter__(self):
        self.old = set_option(self.key, self.value)
        return self

    def __exit__(self, *exc):
        set_option(self.key, self.old)
        return False


def _ptr(t, name: str, index=None) -> int:
    if t is None:
        return None
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is torch.float32 and t.is_contiguous():
        return t.data_ptr()
    if index is not None:
        name = name % index  # (formatted for the message only)
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a torch CUDA tensor" % name)
    if t.dtype != torch.float32:
        raise TypeError("%s must be float32, got %s" % (name, t.dtype))
    raise ValueError("%s must be dense row-major (contiguous)" % name)


def _stream(stream) -> int:
    if stream is None:
        # torch.cuda.current_stream().cuda_stream without the Stream object (2.6 us, a third of a small call's host time);
        # not a public name, so not relied on
        if _RAW_STREAM is None:
            return torch.cuda.current_stream().cuda_stream
        return _RAW_STREAM(torch.cuda.current_device())
    return int(stream)


def _array(values, n: int) -> bytes:
    """A host array of n 64-bit words (pointers or extents) for the duration of a call."""
    if len(values) != n:
        raise IndexError("%d values for %d entries" % (len(values), n))
    return struct.pack("%dq" % n, *values)


def _check(status: int, where: str) -> None:
    if status != TC_OK:
        raise TcError(status, where)


def tc_tbmm(X, Y, Z, stream=None) -> None:
    """Z[B,N,M] = sum_k X[B,N,K] * Y[B,M,K]; Z is written in place."""
    if _FAST is not None:
        status = _FAST.tbmm(_AT["tc_tbmm"], X, Y, Z, stream)
        if status >= 0:
            return _check(status, "tc_tbmm")
    B, N, K = X.shape
    B2, M, K2 = Y.shape
    if (B, K) != (B2, K2) or tuple(Z.shape) != (B, N, M):
        raise ValueError("tc_tbmm: shapes X %s Y %s Z %s do not fit" % (tuple(X.shape), tuple(Y.shape), tuple(Z.shape)))
    _check(lib().tc_tbmm(_ptr(X, "X"), _ptr(Y, "Y"), _ptr(Z, "Z"), B, N, M, K, _stream(stream)), "tc_tbmm")


def tc_tbmm_workspace_bytes(B: int, N: int, M: int, K: int) -> int:
    return int(lib().tc_tbmm_workspace_bytes(int(B), int(N), int(M), int(K)))


def tc_tbmm_ws(X, Y, Z, workspace, stream=None) -> None:
    """tc_tbmm with a workspace (a uint8 tensor of at least tc_tbmm_workspace_bytes bytes, or None)."""
    if _FAST is not None:
        status = _FAST.tbmm_ws(_AT["tc_tbmm_ws"], X, Y, Z, workspace, stream)
        if status >= 0:
            return _check(status, "tc_tbmm_ws")
    B, N, K = X.shape
    B2, M, K2 = Y.shape
    if (B, K) != (B2, K2) or tuple(Z.shape) != (B, N, M):
        raise ValueError("tc_tbmm_ws: shapes X %s Y %s Z %s do not fit" % (tuple(X.shape), tuple(Y.shape), tuple(Z.shape)))
    wp = ctypes.c_void_p(workspace.data_ptr()) if workspace is not None else None
    wn = int(workspace.numel() * workspace.element_size()) if workspace is not None else 0
    _check(lib().tc_tbmm_ws(_ptr(X, "X"), _ptr(Y, "Y"), _ptr(Z, "Z"), B, N, M, K, wp, ctypes.c_size_t(wn), _stream(stream)),
           "tc_tbmm_ws")


def tc_mlp_fcrelu_workspace_bytes(batch: int, dims) -> int:
    n = len(dims) - 1
    arr = (ctypes.c_int64 * (n + 1))(*[int(d) for d in dims])
    return int(lib().tc_mlp_fcrelu_workspace_bytes(int(batch), n, arr))


def _mlp_args(I, W, bias, O, where):
    n = len(W)
    batch, d0 = I.shape
    dims = [d0] + [int(w.shape[0]) for w in W]
    for l in range(n):
        if tuple(W[l].shape) != (dims[l + 1], dims[l]) or tuple(bias[l].shape) != (dims[l + 1],):
            raise ValueError("%s: layer %d shapes do not chain" % (where, l))
        if O[l] is not None and tuple(O[l].shape) != (batch, dims[l + 1]):
            raise ValueError("%s: O[%d] has the wrong shape" % (where, l))
    Wp = _array([_ptr(w, "W[%d]", l) for l, w in enumerate(W)], n)
    bp = _array([_ptr(b, "bias[%d]", l) for l, b in enumerate(bias)], n)
    Op = _array([_ptr(o, "O[%d]", l) or 0 for l, o in enumerate(O)], n)
    dm = _array(dims, n + 1)
    return batch, n, dm, Wp, bp, Op


def tc_mlp_fcrelu(I, W, bias, O, workspace=None, stream=None) -> None:
    """Chained fcrelu layers.  W, bias, O are lists (O[l] may be None for l < last).

    ``workspace`` is a torch CUDA uint8 tensor of at least
    tc_mlp_fcrelu_workspace_bytes(batch, dims) bytes (None only when that is 0).
    """
    if _FAST is not None:
        status = _FAST.mlp(_AT["tc_mlp_fcrelu"], I, W, bias, O, workspace, stream)
        if status >= 0:
            return _check(status, "tc_mlp_fcrelu")
    batch, n, dm, Wp, bp, Op = _mlp_args(I, W, bias, O, "tc_mlp_fcrelu")
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise TypeError("workspace must be a contiguous CUDA tensor")
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(lib().tc_mlp_fcrelu(_ptr(I, "I"), batch, n, dm, Wp, bp, Op, ws_ptr, ws_bytes, _stream(stream)),
           "tc_mlp_fcrelu")


def tc_mlp_fcrelu_static(I, W, bias, O, stream=None) -> None:
    """tc_mlp_fcrelu on the library's static scratch array: no workspace argument, no allocation."""
    batch, n, dm, Wp, bp, Op = _mlp_args(I, W, bias, O, "tc_mlp_fcrelu_static")
    _check(lib().tc_mlp_fcrelu_static(_ptr(I, "I"), batch, n, dm, Wp, bp, Op, _stream(stream)),
           "tc_mlp_fcrelu_static")


def tc_group_conv_infer(H: int, W: int, KH: int, KW: int):
    oh, ow = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().tc_group_conv_infer(H, W, KH, KW, ctypes.byref(oh), ctypes.byref(ow)), "tc_group_conv_infer")
    return int(oh.value), int(ow.value)


def tc_group_conv(I, W1, bias, O, stream=None) -> None:
    """O[N,G,F,OH,OW] = grouped conv of I[N,G,C,H,W] with W1[G,F,C,KH,KW] plus bias[G*F] (or None)."""
    if _FAST is not None:
        status = _FAST.gconv(_AT["tc_group_conv"], I, W1, bias, O, stream)
        if status >= 0:
            return _check(status, "tc_group_conv")
    N, G, C, H, W = I.shape
    G2, F, C2, KH, KW = W1.shape
    if (G, C) != (G2, C2):
        raise ValueError("tc_group_conv: I and W1 disagree on G or C")
    if bias is not None and tuple(bias.shape) != (G * F,):
        raise ValueError("tc_group_conv: bias must be [G*F]")
    if tuple(O.shape) != (N, G, F, H - KH + 1, W - KW + 1):
        raise ValueError("tc_group_conv: O has the wrong shape")
    _check(lib().tc_group_conv(_ptr(I, "I"), _ptr(W1, "W1"), _ptr(bias, "bias"), _ptr(O, "O"),
                               N, G, C, F, H, W, KH, KW, _stream(stream)), "tc_group_conv")


def tc_kron(W1, W2, X, Y, stream=None) -> None:
    """Y[B,I,J] = sum_{k,l} W1[I,K] * W2[J,L] * X[B,K,L]."""
    if _FAST is not None:
        status = _FAST.kron(_AT["tc_kron"], W1, W2, X, Y, stream)
        if status >= 0:
            return _check(status, "tc_kron")
    I, K = W1.shape
    J, L = W2.shape
    B, K2, L2 = X.shape
    if (K, L) != (K2, L2) or tuple(Y.shape) != (B, I, J):
        raise ValueError("tc_kron: shapes do not fit")
    _check(lib().tc_kron(_ptr(W1, "W1"), _ptr(W2, "W2"), _ptr(X, "X"), _ptr(Y, "Y"), B, I, K, J, L,
                         _stream(stream)), "tc_kron")


def tc_sconv2d_infer(H: int, W: int, KH: int, KW: int, sh: int, sw: int):
    oh, ow = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().tc_sconv2d_infer(H, W, KH, KW, sh, sw, ctypes.byref(oh), ctypes.byref(ow)), "tc_sconv2d_infer")
    return int(oh.value), int(ow.value)


def tc_sconv2d(I, Wt, bias, O, sh: int, sw: int, stream=None) -> None:
    """O[N,F,OH,OW] = bias[F] + convolution of I[N,C,H,W] with Wt[F,C,KH,KW], strides (sh, sw), no padding."""
    if _FAST is not None:
        status = _FAST.sconv(_AT["tc_sconv2d"], I, Wt, bias, O, sh, sw, stream)
        if status >= 0:
            return _check(status, "tc_sconv2d")
    N, C, H, W = I.shape
    F, C2, KH, KW = Wt.shape
    if C != C2:
        raise ValueError("tc_sconv2d: I and Wt disagree on C")
    if bias is not None and tuple(bias.shape) != (F,):
        raise ValueError("tc_sconv2d: bias must be [F]")
    # (the library's rule for the extents; what it refuses, it is asked about)
    fits = sh > 0 and sw > 0 and 0 < KH <= H and 0 < KW <= W
    OH, OW = ((H - KH) // sh + 1, (W - KW) // sw + 1) if fits else tc_sconv2d_infer(H, W, KH, KW, sh, sw)
    if tuple(O.shape) != (N, F, OH, OW):
        raise ValueError("tc_sconv2d: O has the wrong shape")
    _check(lib().tc_sconv2d(_ptr(I, "I"), _ptr(Wt, "Wt"), _ptr(bias, "bias"), _ptr(O, "O"),
                            N, C, F, H, W, KH, KW, sh, sw, _stream(stream)), "tc_sconv2d")


def tc_lut(LUT, Idx, O, stream=None) -> None:
    """O[t][B,D] = sum_k LUT[t][Idx[t][B,k], :] for every table t; LUT, Idx, O are lists of equal length."""
    if _FAST is not None:
        status = _FAST.lut(_AT["tc_lut"], LUT, Idx, O, stream)
        if status >= 0:
            return _check(status, "tc_lut")
    n = len(LUT)
    if n == 0 or len(Idx) != n or len(O) != n:
        raise ValueError("tc_lut: LUT, Idx and O must be lists of the same, non-zero length")
    B, D = O[0].shape
    for t in range(n):
        if Idx[t].dtype != torch.int32 or not Idx[t].is_cuda or not Idx[t].is_contiguous():
            raise TypeError("tc_lut: Idx[%d] must be a contiguous int32 CUDA tensor" % t)
        if LUT[t].shape[1] != D or Idx[t].shape[0] != B or tuple(O[t].shape) != (B, D):
            raise ValueError("tc_lut: table %d shapes do not fit" % t)
    Lp = _array([_ptr(x, "LUT[%d]", t) for t, x in enumerate(LUT)], n)
    Ip = _array([x.data_ptr() for x in Idx], n)
    Op = _array([_ptr(x, "O[%d]", t) for t, x in enumerate(O)], n)
    Ev = _array([x.shape[0] for x in LUT], n)
    Lv = _array([x.shape[1] for x in Idx], n)
    _check(lib().tc_lut(n, Lp, Ip, Op, Ev, Lv, D, B, _stream(stream)), "tc_lut")


# ---- operators around experts --------------------------------------------------------------------------------------------------


def _typed(t, name: str, dims: int, dtype=None):
    """Address of a dense CUDA tensor of `dims` dimensions, of one of the storage types or of `dtype`."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a torch CUDA tensor" % name)
    if (t.dtype is not dtype) if dtype is not None else (t.dtype not in _TYPES):
        raise TypeError("%s must be %s, got %s" % (name, dtype or "float32, bfloat16 or float16", t.dtype))
    if t.dim() != dims:
        raise ValueError("%s must have %d dimensions" % (name, dims))
    if not t.is_contiguous():
        raise ValueError("%s must be dense row-major (contiguous)" % name)
    return t.data_ptr()


def _grad_of(t, name: str, dims: int, dtype):
    """The same for a gradient, which may be kept in float32 whatever the type of what it is taken from."""
    return _typed(t, name, dims, None if getattr(t, "dtype", None) is torch.float32 else dtype)


def _fit(ok: bool, where: str) -> None:
    if not ok:
        raise ValueError("%s: shapes do not fit" % where)


def _workspace(ws):
    if ws is None:
        return None, 0
    if not isinstance(ws, torch.Tensor) or not ws.is_cuda or not ws.is_contiguous():
        raise TypeError("workspace must be a contiguous CUDA tensor")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def tc_embed(LUT, Idx, O, scale: float = 1.0, stream=None) -> None:
    """O[T,D] = scale * LUT[Idx[T], :] (int32 numbers; one outside [0, E) gives a row of NaN)."""
    if _FAST is not None:
        status = _FAST.embed(_AT["tc_embed"], LUT, Idx, O, scale, stream)
        if status >= 0:
            return _check(status, "tc_embed")
    l, i, o = _typed(LUT, "LUT", 2), _typed(Idx, "Idx", 1, torch.int32), _typed(O, "O", 2, LUT.dtype)
    (E, D), T = LUT.shape, Idx.shape[0]
    _fit(tuple(O.shape) == (T, D), "tc_embed")
    _check(lib().tc_embed(l, i, o, E, D, T, scale, _TYPES[LUT.dtype], _stream(stream)), "tc_embed")


def tc_embed_grad_workspace_bytes(E: int, D: int, T: int) -> int:
    return int(lib().tc_embed_grad_workspace_bytes(int(E), int(D), int(T)))


def tc_embed_grad(dO, Idx, dLUT, workspace, scale: float = 1.0, pad: int = -1, add: bool = False, stream=None) -> None:
    """dLUT[E,D] (+)= scale * the sum of the rows of dO[T,D] whose number Idx[T] is the row's; `pad` and numbers outside [0, E) take no part.

    dLUT is of dO's type or float32.  ``workspace``: a uint8 tensor of at least tc_embed_grad_workspace_bytes(E, D, T) bytes."""
    if _FAST is not None:
        status = _FAST.embed_grad(_AT["tc_embed_grad"], dO, Idx, dLUT, workspace, scale, pad, add, stream)
        if status >= 0:
            return _check(status, "tc_embed_grad")
    d, i, g = _typed(dO, "dO", 2), _typed(Idx, "Idx", 1, torch.int32), _grad_of(dLUT, "dLUT", 2, dO.dtype)
    (T, D), E = dO.shape, dLUT.shape[0]
    _fit(dLUT.shape[1] == D and Idx.shape[0] == T, "tc_embed_grad")
    wp, wn = _workspace(workspace)
    _check(lib().tc_embed_grad(d, i, g, E, D, T, scale, pad, int(add), _TYPES[dO.dtype], _TYPES[dLUT.dtype], wp, wn, _stream(stream)), "tc_embed_grad")


def tc_route_workspace_bytes(T: int, E: int, k: int) -> int:
    return int(lib().tc_route_workspace_bytes(int(T), int(E), int(k)))


def tc_route(L, Wt, Id, Off, Row, Place, workspace=None, norm: bool = False, stream=None) -> None:
    """Weights Wt[T,k] and numbers Id[T,k] of the k largest of L[T,E], and the slots by expert: Off[E+1], Row[T*k], Place[T,k].

    ``workspace``: a uint8 tensor of at least tc_route_workspace_bytes(T, E, k) bytes (None when that is 0; up to 64 tokens less only costs time)."""
    if _FAST is not None:
        status = _FAST.route(_AT["tc_route"], L, Wt, Id, Off, Row, Place, workspace, norm, stream)
        if status >= 0:
            return _check(status, "tc_route")
    i32 = torch.int32
    args = (_typed(L, "L", 2), _typed(Wt, "Wt", 2, torch.float32), _typed(Id, "Id", 2, i32), _typed(Off, "Off", 1, i32), _typed(Row, "Row", 1, i32),
            _typed(Place, "Place", 2, i32))
    (T, E), k = L.shape, Id.shape[1]
    _fit(tuple(Id.shape) == tuple(Wt.shape) == tuple(Place.shape) == (T, k) and Off.shape[0] == E + 1 and Row.shape[0] == T * k, "tc_route")
    wp, wn = _workspace(workspace)
    _check(lib().tc_route(*args, T, E, k, int(norm), _TYPES[L.dtype], wp, wn, _stream(stream)), "tc_route")


def tc_route_grad(L, Id, dWt, dL, norm: bool = False, stream=None) -> None:
    """dL[T,E]: the gradient of tc_route's weights, from L[T,E], Id[T,k] and dWt[T,k]."""
    if _FAST is not None:
        status = _FAST.route_grad(_AT["tc_route_grad"], L, Id, dWt, dL, norm, stream)
        if status >= 0:
            return _check(status, "tc_route_grad")
    args = (_typed(L, "L", 2), _typed(Id, "Id", 2, torch.int32), _typed(dWt, "dWt", 2, torch.float32), _typed(dL, "dL", 2, L.dtype))
    (T, E), k = L.shape, Id.shape[1]
    _fit(tuple(Id.shape) == tuple(dWt.shape) == (T, k) and dL.shape == L.shape, "tc_route_grad")
    _check(lib().tc_route_grad(*args, T, E, k, int(norm), _TYPES[L.dtype], _stream(stream)), "tc_route_grad")


def tc_expert_mm(X, W, Off, Row, Y, relu: bool = False, stream=None) -> None:
    """Y[R,N]: rows Off[e] .. Off[e+1] are those of X times W[e] ([N,K]), clamped at 0 if relu; row r of X[T,K] is Row[r], or r where Row is None."""
    if _FAST is not None:
        status = _FAST.expert_mm(_AT["tc_expert_mm"], X, W, Off, Row, Y, relu, stream)
        if status >= 0:
            return _check(status, "tc_expert_mm")
    i32 = torch.int32
    args = (_typed(X, "X", 2), _typed(W, "W", 3, X.dtype), _typed(Off, "Off", 1, i32), None if Row is None else _typed(Row, "Row", 1, i32),
            _typed(Y, "Y", 2, X.dtype))
    (T, K), (E, N), R = X.shape, W.shape[:2], Y.shape[0]
    _fit(W.shape[2] == K and Off.shape[0] == E + 1 and Y.shape[1] == N and (T if Row is None else Row.shape[0]) == R, "tc_expert_mm")
    _check(lib().tc_expert_mm(*args, T, R, E, N, K, int(relu), _TYPES[X.dtype], _stream(stream)), "tc_expert_mm")


def tc_expert_mm_grad_x(dY, W, Off, gate, dX, stream=None) -> None:
    """dX[R,K]: the rows of each expert of dY[R,N] times W[e] ([N,K]); 0 where gate[R,K] (or None) is not above 0."""
    if _FAST is not None:
        status = _FAST.expert_mm_grad_x(_AT["tc_expert_mm_grad_x"], dY, W, Off, gate, dX, stream)
        if status >= 0:
            return _check(status, "tc_expert_mm_grad_x")
    args = (_typed(dY, "dY", 2), _typed(W, "W", 3, dY.dtype), _typed(Off, "Off", 1, torch.int32), None if gate is None else _typed(gate, "gate", 2, dY.dtype),
            _typed(dX, "dX", 2, dY.dtype))
    (R, N), (E, N2, K) = dY.shape, W.shape
    _fit(N == N2 and Off.shape[0] == E + 1 and tuple(dX.shape) == (R, K) and (gate is None or tuple(gate.shape) == (R, K)), "tc_expert_mm_grad_x")
    _check(lib().tc_expert_mm_grad_x(*args, R, E, N, K, _TYPES[dY.dtype], _stream(stream)), "tc_expert_mm_grad_x")


def tc_expert_mm_grad_w_workspace_bytes(R: int, E: int, N: int, K: int) -> int:
    return int(lib().tc_expert_mm_grad_w_workspace_bytes(int(R), int(E), int(N), int(K)))


def tc_expert_mm_grad_w(dY, X, Off, Row, dW, workspace=None, add: bool = False, stream=None) -> None:
    """dW[E,N,K] (+)= for each expert the products of its rows of dY[R,N] with those of X (taken through Row as in tc_expert_mm).

    dW is of dY's type or float32.  ``workspace``: as tc_tbmm_ws; less than tc_expert_mm_grad_w_workspace_bytes(R, E, N, K) bytes
    only cost time."""
    if _FAST is not None:
        status = _FAST.expert_mm_grad_w(_AT["tc_expert_mm_grad_w"], dY, X, Off, Row, dW, workspace, add, stream)
        if status >= 0:
            return _check(status, "tc_expert_mm_grad_w")
    i32 = torch.int32
    args = (_typed(dY, "dY", 2), _typed(X, "X", 2, dY.dtype), _typed(Off, "Off", 1, i32), None if Row is None else _typed(Row, "Row", 1, i32),
            _grad_of(dW, "dW", 3, dY.dtype))
    (R, N), (T, K), E = dY.shape, X.shape, dW.shape[0]
    _fit(tuple(dW.shape) == (E, N, K) and Off.shape[0] == E + 1 and (T if Row is None else Row.shape[0]) == R, "tc_expert_mm_grad_w")
    wp, wn = _workspace(workspace)
    _check(lib().tc_expert_mm_grad_w(*args, T, R, E, N, K, int(add), _TYPES[dY.dtype], _TYPES[dW.dtype], wp, wn, _stream(stream)), "tc_expert_mm_grad_w")


def tc_expert_sum(Y, Wt, Place, O, stream=None) -> None:
    """O[T,N] = the sum over i of Wt[T,k] (None: ones) times the rows Place[T,k] of Y[R,N]; a place outside [0, R) takes no part."""
    if _FAST is not None:
        status = _FAST.expert_sum(_AT["tc_expert_sum"], Y, Wt, Place, O, stream)
        if status >= 0:
            return _check(status, "tc_expert_sum")
    args = (_typed(Y, "Y", 2), None if Wt is None else _typed(Wt, "Wt", 2, torch.float32), _typed(Place, "Place", 2, torch.int32), _typed(O, "O", 2, Y.dtype))
    (R, N), (T, k) = Y.shape, Place.shape
    _fit(tuple(O.shape) == (T, N) and (Wt is None or tuple(Wt.shape) == (T, k)), "tc_expert_sum")
    _check(lib().tc_expert_sum(*args, T, R, k, N, _TYPES[Y.dtype], _stream(stream)), "tc_expert_sum")


def tc_expert_sum_grad(dO, Y, Wt, Place, dY, dWt, stream=None) -> None:
    """dY[R,N] (rows of the places that occur) and dWt[T,k]: the gradients of tc_expert_sum, from dO[T,N]."""
    if _FAST is not None:
        status = _FAST.expert_sum_grad(_AT["tc_expert_sum_grad"], dO, Y, Wt, Place, dY, dWt, stream)
        if status >= 0:
            return _check(status, "tc_expert_sum_grad")
    args = (_typed(dO, "dO", 2), _typed(Y, "Y", 2, dO.dtype), _typed(Wt, "Wt", 2, torch.float32), _typed(Place, "Place", 2, torch.int32),
            _typed(dY, "dY", 2, dO.dtype), _typed(dWt, "dWt", 2, torch.float32))
    (R, N), (T, k) = Y.shape, Place.shape
    _fit(tuple(dO.shape) == (T, N) and tuple(Wt.shape) == tuple(dWt.shape) == (T, k) and dY.shape == Y.shape, "tc_expert_sum_grad")
    _check(lib().tc_expert_sum_grad(*args, T, R, k, N, _TYPES[dO.dtype], _stream(stream)), "tc_expert_sum_grad")


# ---- operators around experts of even load, with weights in 8 bits ------------------------------------------------------------------


def tc_layer_norm(X, W, B, O, eps: float = 1e-5, stream=None) -> None:
    """O[T,N] = (X[T,N] - mean) / sqrt(variance + eps) * W[N] + B[N] (None: zeros), row by row; W and B of X's type or float32."""
    if _FAST is not None:
        status = _FAST.layer_norm(_AT["tc_layer_norm"], X, W, B, O, eps, stream)
        if status >= 0:
            return _check(status, "tc_layer_norm")
    x, o = _typed(X, "X", 2), _typed(O, "O", 2, X.dtype)
    w = _grad_of(W, "W", 1, X.dtype)
    b = None if B is None else _typed(B, "B", 1, W.dtype)
    T, N = X.shape
    _fit(O.shape == X.shape and W.shape[0] == N and (B is None or B.shape[0] == N), "tc_layer_norm")
    _check(lib().tc_layer_norm(x, w, b, o, T, N, eps, _TYPES[X.dtype], _TYPES[W.dtype], _stream(stream)), "tc_layer_norm")


def tc_layer_norm_grad_workspace_bytes(T: int, N: int) -> int:
    return int(lib().tc_layer_norm_grad_workspace_bytes(int(T), int(N)))


def tc_layer_norm_grad(dO, X, W, dX, dW, dB, workspace=None, eps: float = 1e-5, add: bool = False, stream=None) -> None:
    """dX[T,N] and, (+)=, dW[N] and dB[N] (None: not asked for; dB only beside dW): the gradients of tc_layer_norm, from dO[T,N].

    ``workspace``: a uint8 tensor of at least tc_layer_norm_grad_workspace_bytes(T, N) bytes (None without dW)."""
    if _FAST is not None:
        status = _FAST.layer_norm_grad(_AT["tc_layer_norm_grad"], dO, X, W, dX, dW, dB, workspace, eps, add, stream)
        if status >= 0:
            return _check(status, "tc_layer_norm_grad")
    x, d, g = _typed(X, "X", 2), _typed(dO, "dO", 2, X.dtype), _typed(dX, "dX", 2, X.dtype)
    w = _grad_of(W, "W", 1, X.dtype)
    gw, gb = (None if t is None else _typed(t, n, 1, W.dtype) for t, n in ((dW, "dW"), (dB, "dB")))
    T, N = X.shape
    _fit(dO.shape == dX.shape == X.shape and W.shape[0] == N and all(t is None or t.shape[0] == N for t in (dW, dB)), "tc_layer_norm_grad")
    wp, wn = _workspace(workspace)
    _check(lib().tc_layer_norm_grad(d, x, w, g, gw, gb, T, N, eps, int(add), _TYPES[X.dtype], _TYPES[W.dtype], wp, wn, _stream(stream)), "tc_layer_norm_grad")


def tc_route_balanced_workspace_bytes(T: int, E: int, k: int) -> int:
    return int(lib().tc_route_balanced_workspace_bytes(int(T), int(E), int(k)))


def tc_route_balanced(L, Bias, Wt, Id, Off, Row, Place, workspace=None, groups: int = 1, keep: int = 1, sigmoid: bool = False, norm: bool = False,
                      scale: float = 1.0, stream=None) -> None:
    """tc_route by scores of sigmoid or softmax: the k largest of score + Bias[E] (None: zeros) in the `keep` best of `groups` groups, weights of
    scale times the scores (norm: over their sum).

    ``workspace``: a uint8 tensor of at least tc_route_balanced_workspace_bytes(T, E, k) bytes, as for tc_route."""
    if _FAST is not None:
        status = _FAST.route_balanced(_AT["tc_route_balanced"], L, Bias, Wt, Id, Off, Row, Place, workspace, groups, keep, sigmoid, norm, scale, stream)
        if status >= 0:
            return _check(status, "tc_route_balanced")
    i32 = torch.int32
    args = (_typed(L, "L", 2), None if Bias is None else _typed(Bias, "Bias", 1, torch.float32), _typed(Wt, "Wt", 2, torch.float32), _typed(Id, "Id", 2, i32),
            _typed(Off, "Off", 1, i32), _typed(Row, "Row", 1, i32), _typed(Place, "Place", 2, i32))
    (T, E), k = L.shape, Id.shape[1]
    _fit(tuple(Id.shape) == tuple(Wt.shape) == tuple(Place.shape) == (T, k) and Off.shape[0] == E + 1 and Row.shape[0] == T * k and
         (Bias is None or Bias.shape[0] == E), "tc_route_balanced")
    wp, wn = _workspace(workspace)
    _check(lib().tc_route_balanced(*args, T, E, k, groups, keep, int(sigmoid), int(norm), scale, _TYPES[L.dtype], wp, wn, _stream(stream)), "tc_route_balanced")


def tc_route_balanced_grad(L, Id, dWt, dL, sigmoid: bool = False, norm: bool = False, scale: float = 1.0, stream=None) -> None:
    """dL[T,E]: the gradient of tc_route_balanced's weights, from L[T,E], Id[T,k] and dWt[T,k]."""
    if _FAST is not None:
        status = _FAST.route_balanced_grad(_AT["tc_route_balanced_grad"], L, Id, dWt, dL, sigmoid, norm, scale, stream)
        if status >= 0:
            return _check(status, "tc_route_balanced_grad")
    args = (_typed(L, "L", 2), _typed(Id, "Id", 2, torch.int32), _typed(dWt, "dWt", 2, torch.float32), _typed(dL, "dL", 2, L.dtype))
    (T, E), k = L.shape, Id.shape[1]
    _fit(tuple(Id.shape) == tuple(dWt.shape) == (T, k) and dL.shape == L.shape, "tc_route_balanced_grad")
    _check(lib().tc_route_balanced_grad(*args, T, E, k, int(sigmoid), int(norm), scale, _TYPES[L.dtype], _stream(stream)), "tc_route_balanced_grad")


def _blocks(n: int) -> int:
    return -(-n // TC_Q8_BLOCK)


def tc_quantize_rows(X, Q, S, stream=None) -> None:
    """Q[R,K'] (float8_e4m3fn) and S[R,K'/128] (float8_e8m0fnu): the rows of X[R,K] in 8 bits, a scale for each 128 elements; K': K rounded up to 128s."""
    if _FAST is not None:
        status = _FAST.quantize_rows(_AT["tc_quantize_rows"], X, Q, S, stream)
        if status >= 0:
            return _check(status, "tc_quantize_rows")
    args = (_typed(X, "X", 2), _typed(Q, "Q", 2, torch.float8_e4m3fn), _typed(S, "S", 2, torch.float8_e8m0fnu))
    R, K = X.shape
    _fit(tuple(S.shape) == (R, _blocks(K)) and tuple(Q.shape) == (R, TC_Q8_BLOCK * _blocks(K)), "tc_quantize_rows")
    _check(lib().tc_quantize_rows(*args, R, K, _TYPES[X.dtype], _stream(stream)), "tc_quantize_rows")


def tc_quantize_weights(W, Q, S, Qt=None, St=None, stream=None) -> None:
    """Q[E,N,K'], S[E,N'/128,K'/128]: the weights W[E,N,K] in 8 bits, a scale for each 128 x 128 elements; Qt[E,K,N'], St[E,K'/128,N'/128] (both or
    neither): the same transposed."""
    if _FAST is not None:
        status = _FAST.quantize_weights(_AT["tc_quantize_weights"], W, Q, S, Qt, St, stream)
        if status >= 0:
            return _check(status, "tc_quantize_weights")
    e4, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    args = (_typed(W, "W", 3), _typed(Q, "Q", 3, e4), _typed(S, "S", 3, e8), None if Qt is None else _typed(Qt, "Qt", 3, e4), None if St is None else _typed(St, "St", 3, e8))
    E, N, K = W.shape
    n, k = _blocks(N), _blocks(K)
    _fit(tuple(Q.shape) == (E, N, TC_Q8_BLOCK * k) and tuple(S.shape) == (E, n, k) and (Qt is None or tuple(Qt.shape) == (E, K, TC_Q8_BLOCK * n)) and
         (St is None or tuple(St.shape) == (E, k, n)), "tc_quantize_weights")
    _check(lib().tc_quantize_weights(*args, E, N, K, _TYPES[W.dtype], _stream(stream)), "tc_quantize_weights")


def tc_expert_mm_q8_workspace_bytes(T: int, R: int, E: int, N: int, K: int) -> int:
    return int(lib().tc_expert_mm_q8_workspace_bytes(int(T), int(R), int(E), int(N), int(K)))


def tc_expert_mm_q8(X, SX, W, SW, Off, Row, gate, Y, workspace=None, relu: bool = False, stream=None) -> None:
    """tc_expert_mm with weights W[E,N,K'], SW[E,N'/128,K'/128] in 8 bits (tc_quantize_weights) and rows X[T,K] put in 8 bits on the way, or X[T,K'], SX[T,K'/128]
    that are already; 0 where gate[R,N] (or None) is not above 0.  Off None: one expert (E = 1) has all rows.

    With dY for X and the transposed weights for W: the gradient of the rows.  ``workspace``: a uint8 tensor of at least
    tc_expert_mm_q8_workspace_bytes(T, R, E, N, K) bytes (None where X is in 8 bits)."""
    if _FAST is not None:
        status = _FAST.expert_mm_q8(_AT["tc_expert_mm_q8"], X, SX, W, SW, Off, Row, gate, Y, workspace, relu, stream)
        if status >= 0:
            return _check(status, "tc_expert_mm_q8")
    i32, e4, e8 = torch.int32, torch.float8_e4m3fn, torch.float8_e8m0fnu
    y = _typed(Y, "Y", 2)
    args = (_typed(X, "X", 2, Y.dtype if SX is None else e4), None if SX is None else _typed(SX, "SX", 2, e8), _typed(W, "W", 3, e4), _typed(SW, "SW", 3, e8),
            None if Off is None else _typed(Off, "Off", 1, i32), None if Row is None else _typed(Row, "Row", 1, i32),
            None if gate is None else _typed(gate, "gate", 2, Y.dtype), y)
    (T, K), (E, N, K8), R = X.shape, W.shape, Y.shape[0]
    k = _blocks(K)
    _fit(K8 == TC_Q8_BLOCK * k and (SX is None or (K == K8 and tuple(SX.shape) == (T, k))) and tuple(SW.shape) == (E, _blocks(N), k) and Y.shape[1] == N and
         (E == 1 if Off is None else Off.shape[0] == E + 1) and (T if Row is None else Row.shape[0]) == R and (gate is None or gate.shape == Y.shape), "tc_expert_mm_q8")
    wp, wn = _workspace(workspace)
    _check(lib().tc_expert_mm_q8(*args, T, R, E, N, K, int(relu), _TYPES[Y.dtype], wp, wn, _stream(stream)), "tc_expert_mm_q8")
