"""ctypes binding of libclearmoe.so, one Python function per C entry point (same names).

Argument marshalling only: tensors become device pointers, torch's current stream becomes the
cudaStream_t, non-zero status codes become ClearMoEError. Every step of the layer runs in the
library's CUDA kernels; there is no Python or CPU fallback. The C declarations, with argument
meaning, layout, ownership and errors, are in include/clearmoe.h.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import pathlib

_LIB_PATH = pathlib.Path(__file__).resolve().parent / "libclearmoe.so"
_lib = None

OK, EINVAL, EUNSUPPORTED, ECUDA, ENOMEM, ETIMEOUT = 0, -1, -2, -3, -4, -5
F32, BF16, FP8 = 0, 1, 2


class ClearMoEError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {clearmoe_strerror(code)} ({code})")
        self.code = code


class clearmoe_layer_desc(ctypes.Structure):
    _fields_ = [("max_tokens", ctypes.c_int64), ("d", ctypes.c_int32), ("hidden", ctypes.c_int32),
                ("max_E", ctypes.c_int32), ("max_r", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class clearmoe_router(ctypes.Structure):
    _fields_ = [("W", ctypes.c_void_p), ("b", ctypes.c_void_p)]


class clearmoe_mlp_router(ctypes.Structure):
    _fields_ = [("W_in", ctypes.c_void_p), ("b_in", ctypes.c_void_p), ("W_out", ctypes.c_void_p),
                ("b_out", ctypes.c_void_p), ("hidden", ctypes.c_int32), ("act", ctypes.c_int32)]


class clearmoe_ffn_options(ctypes.Structure):
    _fields_ = [("b2", ctypes.c_void_p), ("cls_stride", ctypes.c_int64), ("W2", ctypes.c_void_p),
                ("mlp_router", ctypes.POINTER(clearmoe_mlp_router)), ("input_layernorm", ctypes.c_int32),
                ("router_in_fc1", ctypes.c_int32)]


class clearmoe_fp8(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


class clearmoe_fp4(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


class _PlacedFp8(clearmoe_fp8):  # and the GPU it lies on (-1: not known), for the calls that look
    _fields_ = [("device", ctypes.c_int32)]


class _PlacedFp4(clearmoe_fp4):
    _fields_ = [("device", ctypes.c_int32)]


class clearmoe_norm(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("residual", ctypes.c_void_p), ("sum", ctypes.c_void_p), ("weight", ctypes.c_void_p),
                ("ldx", ctypes.c_int64), ("ldr", ctypes.c_int64), ("lds", ctypes.c_int64), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("dtype", ctypes.c_int32), ("weight_dtype", ctypes.c_int32), ("eps", ctypes.c_float)]


class clearmoe_fp8_epilogue(ctypes.Structure):
    _fields_ = [("bias", ctypes.c_void_p), ("bias_dtype", ctypes.c_int32), ("act", ctypes.c_int32),
                ("status", ctypes.c_void_p)]


class clearmoe_ffn_weights(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("E", ctypes.c_int32), ("W1", clearmoe_fp8), ("W2", clearmoe_fp8),
                ("W_comb", clearmoe_fp8 * 16), ("b1", ctypes.c_void_p), ("b2", ctypes.c_void_p),
                ("router", clearmoe_router), ("cls_stride", ctypes.c_int64), ("input_layernorm", ctypes.c_int32)]


ACT_NONE, ACT_RELU, ACT_GELU = -1, 0, 1
FEW_MAX = 64
NORM_MAX = 32768  # columns of clearmoe_rms_norm


def mlp_router(W_in, b_in, W_out, b_out, act: str = "relu") -> clearmoe_mlp_router:
    """The MLP router's weights as the C struct (act: "relu" or "gelu")."""
    return clearmoe_mlp_router(_ptr(W_in), _ptr(b_in), _ptr(W_out), _ptr(b_out), W_in.shape[0],
                               {"relu": ACT_RELU, "gelu": ACT_GELU}[act])


_P, _I64, _I32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
_SIGS = {
    "clearmoe_layer_create": [ctypes.POINTER(clearmoe_layer_desc), ctypes.POINTER(ctypes.c_void_p)],
    "clearmoe_layer_destroy": [_P],
    "clearmoe_route": [_P, _P, _I64, ctypes.POINTER(clearmoe_router), _I32, _P],
    "clearmoe_route_mlp": [_P, _P, _I64, ctypes.POINTER(clearmoe_mlp_router), _I32, _P],
    "clearmoe_ffn_forward": [_P, _P, _I64, _P, _P, _P, _P, _P, ctypes.POINTER(ctypes.c_void_p),
                             ctypes.POINTER(clearmoe_router), _I32, _I32, _P, _P],
    "clearmoe_ffn_forward_ex": [_P, _P, _I64, _P, _P, _P, _P, _P, ctypes.POINTER(ctypes.c_void_p),
                                ctypes.POINTER(clearmoe_router), _I32, _I32,
                                ctypes.POINTER(clearmoe_ffn_options), _P, _P],
    "clearmoe_materialize_basis": [_P, _P, _P, _P, _I32, _P, _P],
    "clearmoe_ffn_forward_folded_ex": [_P, _P, _I64, _P, _P, ctypes.POINTER(ctypes.c_void_p),
                                       ctypes.POINTER(clearmoe_router), _I32,
                                       ctypes.POINTER(clearmoe_ffn_options), _P, _P],
    "clearmoe_ffn_forward_materialized_ex": [_P, _P, _I64, _P, _P, _P, ctypes.POINTER(ctypes.c_void_p),
                                             ctypes.POINTER(clearmoe_router), _I32,
                                             ctypes.POINTER(clearmoe_ffn_options), _P, _P],
    "clearmoe_ffn_forward_materialized": [_P, _P, _I64, _P, _P, _P, ctypes.POINTER(ctypes.c_void_p),
                                          ctypes.POINTER(clearmoe_router), _I32, _P, _P],
    "clearmoe_ffn_forward_scaled": [_P, _P, _I64, _P, _P, _P, _P, _P, _P, _P,
                                    ctypes.POINTER(clearmoe_router), _I32, _I32, _P, _P],
    "clearmoe_dense_ffn_forward": [_P, _P, _I64, _P, _P, _P, _P, _P],
    "clearmoe_dense_ffn_forward_ex": [_P, _P, _I64, _P, _P, _P, _P, _P, _P],
    "clearmoe_dense_ffn_forward_opt": [_P, _P, _I64, _P, _P, _P, ctypes.POINTER(clearmoe_ffn_options), _P, _P],
    "clearmoe_layer_norm": [_P, _P, _I64, _P, _P],
    "clearmoe_get_routing": [_P, _P, _P, _P, _P, _P],
    "clearmoe_layer_status": [_P],
    "clearmoe_debug_set_wait": [_P, _I64, _I32],
    "clearmoe_set_profile_events": [_P, ctypes.POINTER(ctypes.c_void_p), _I32],
    "clearmoe_fold_basis": [_P, _P, _P, _P, ctypes.POINTER(ctypes.c_void_p), _I32, _I32,
                            ctypes.POINTER(ctypes.c_void_p), _P],
    "clearmoe_ffn_forward_folded": [_P, _P, _I64, _P, _P, ctypes.POINTER(ctypes.c_void_p),
                                    ctypes.POINTER(clearmoe_router), _I32, _P, _P],
    "clearmoe_route_noalloc": [_P, _I64, _I32, _I32, ctypes.POINTER(clearmoe_router), _I32, _P, _P,
                               _P, _P, _P, _P],
    "clearmoe_fp8_quantize_rows": [_P, _I32, _I64, _P, ctypes.POINTER(clearmoe_fp8), _P],
    "clearmoe_fp8_quantize_gathered": [_P, _I64, _I32, _I64, _P, ctypes.POINTER(clearmoe_fp8), _P],
    "clearmoe_fp8_quantize_weight": [_P, _I32, _I64, ctypes.POINTER(clearmoe_fp8), _P],
    "clearmoe_fp8_dequantize": [ctypes.POINTER(clearmoe_fp8), _I32, _P, _I32, _I64, _P],
    "clearmoe_fp8_gemm": [ctypes.POINTER(clearmoe_fp8), ctypes.POINTER(clearmoe_fp8),
                          ctypes.POINTER(clearmoe_fp8_epilogue), _P, _I32, _I64, _P],
    "clearmoe_fp8_gemm_fp8": [ctypes.POINTER(clearmoe_fp8), ctypes.POINTER(clearmoe_fp8),
                              ctypes.POINTER(clearmoe_fp8_epilogue), ctypes.POINTER(clearmoe_fp8), _P],
    "clearmoe_fp8_grouped_gemm": [ctypes.POINTER(clearmoe_fp8), ctypes.POINTER(clearmoe_fp8), _I32, _P, _P,
                                  ctypes.POINTER(clearmoe_fp8_epilogue), _P, _I32, _I64, _P],
    "clearmoe_debug_fp8_kernel": [_I32, _I32],
    "clearmoe_ffn_forward_few": [_P, _P, _I64, ctypes.POINTER(clearmoe_ffn_weights), _P, _P],
    "clearmoe_ffn_forward_fp8": [_P, _P, _I64, ctypes.POINTER(clearmoe_ffn_weights), _P, _P],
    "clearmoe_fp4_quantize": [_P, _I64, _I32, _I64, _P, ctypes.POINTER(clearmoe_fp4), _P],
    "clearmoe_fp4_dequantize": [ctypes.POINTER(clearmoe_fp4), _P, _I32, _I64, _P],
    "clearmoe_fp4_gemm": [ctypes.POINTER(clearmoe_fp4), ctypes.POINTER(clearmoe_fp4),
                          ctypes.POINTER(clearmoe_fp8_epilogue), _P, _I32, _I64, _P],
    "clearmoe_fp4_gemm_fp4": [ctypes.POINTER(clearmoe_fp4), ctypes.POINTER(clearmoe_fp4),
                              ctypes.POINTER(clearmoe_fp8_epilogue), ctypes.POINTER(clearmoe_fp4), _P],
    "clearmoe_fp4_grouped_gemm": [ctypes.POINTER(clearmoe_fp4), ctypes.POINTER(clearmoe_fp4), _I32, _P, _P,
                                  ctypes.POINTER(clearmoe_fp8_epilogue), _P, _I32, _I64, _P],
    "clearmoe_debug_fp4_kernel": [_I32, _I32],
    "clearmoe_debug_fp4_wait": [_I64],
    "clearmoe_rms_norm": [ctypes.POINTER(clearmoe_norm), _P, _I32, _I64, _P],
    "clearmoe_rms_norm_fp8": [ctypes.POINTER(clearmoe_norm), ctypes.POINTER(clearmoe_fp8), _P],
    "clearmoe_rms_norm_fp4": [ctypes.POINTER(clearmoe_norm), ctypes.POINTER(clearmoe_fp4), _P],
    "clearmoe_strerror": [ctypes.c_int],
    "clearmoe_version": [],
}


def lib() -> ctypes.CDLL:
    """Loads libclearmoe.so (built in-tree). Raises if it is missing: there is no fallback."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise RuntimeError(f"{_LIB_PATH} is not built; run paper_2606_28516_gb300.build.build()")
        try:
            import torch  # noqa: F401  (loads the CUDA runtime the library links against)
        except ImportError:
            pass
        L = ctypes.CDLL(str(_LIB_PATH))
        for name, args in _SIGS.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = ctypes.c_char_p if name == "clearmoe_strerror" else ctypes.c_int
        _lib = L
    return _lib


_calls = None


def _bind_calls():
    """Loads the compiled part of this binding (built in-tree with the library) and gives it the library's functions."""
    global _calls
    path = _LIB_PATH.with_name("_calls.so")
    if not path.exists():
        raise RuntimeError(f"{path} is not built; run paper_2606_28516_gb300.build.build()")
    loader = importlib.machinery.ExtensionFileLoader("_calls", str(path))
    m = importlib.util.module_from_spec(importlib.util.spec_from_loader("_calls", loader))
    loader.exec_module(m)
    L = lib()
    m.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in
             (L.clearmoe_fp8_quantize_rows, L.clearmoe_fp8_gemm, L.clearmoe_fp8_gemm_fp8, L.clearmoe_ffn_forward_few,
              L.clearmoe_ffn_forward_fp8)))
    m.bind_fp4(*(ctypes.cast(f, ctypes.c_void_p).value for f in
                 (L.clearmoe_fp4_quantize, L.clearmoe_fp4_gemm, L.clearmoe_fp4_gemm_fp4, L.clearmoe_rms_norm, L.clearmoe_rms_norm_fp8,
                  L.clearmoe_rms_norm_fp4)))
    try:
        import torch
        m.bind_torch(torch.bfloat16, torch.float32, torch.int32, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
        m.bind_dlpack(torch._C._to_dlpack)
    except (ImportError, AttributeError):  # a torch without CUDA: every call then goes by integers
        pass
    _calls = m
    return m


def _check(code: int, where: str) -> None:
    if code != OK:
        raise ClearMoEError(code, where)


def _ptr(t) -> int | None:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors passed to libclearmoe must be contiguous CUDA tensors")
    return t.data_ptr()


_torch = None
_raw_stream = None  # device index -> handle of torch's current stream
_device = None      # the current device's index, once CUDA is initialised


def _stream(stream) -> int | None:
    """The given stream's handle, or that of torch's current stream. The handle is asked for directly:
    building torch's Stream object for it costs 3.2 us a call on the GB300's host, this 0.3 us."""
    global _torch, _raw_stream, _device
    if stream is not None:
        return stream.cuda_stream
    if _device is not None:
        return _raw_stream(_device())
    if _torch is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _torch = torch
    if _raw_stream is None or not _torch.cuda.is_initialized():
        return _torch.cuda.current_stream().cuda_stream
    _device = _torch._C._cuda_getDevice
    return _raw_stream(_device())


def _ptrs(tensors, E: int):
    """A C array of the device pointers of E matrices: a sequence of tensors, or one contiguous
    [E x ...] tensor (the first E of it), whose matrices follow one another: then one base address and
    E steps, since slicing a tensor costs 1.5 us a matrix."""
    stride = getattr(tensors, "stride", None)
    if stride is not None and tensors.dim() > 1 and tensors.shape[0] >= E and tensors.is_contiguous():
        base, step = _ptr(tensors), stride(0) * tensors.element_size()
        return (ctypes.c_void_p * E)(*[base + e * step for e in range(E)])
    return (ctypes.c_void_p * E)(*[_ptr(tensors[e]) for e in range(E)])


def clearmoe_strerror(code: int) -> str:
    return lib().clearmoe_strerror(code).decode()


def clearmoe_version() -> int:
    return lib().clearmoe_version()


def clearmoe_layer_create(max_tokens: int, d: int, hidden: int, max_E: int, max_r: int,
                          dtype: int) -> int:
    desc = clearmoe_layer_desc(max_tokens, d, hidden, max_E, max_r, dtype)
    h = ctypes.c_void_p()
    _check(lib().clearmoe_layer_create(ctypes.byref(desc), ctypes.byref(h)), "clearmoe_layer_create")
    return h.value


def clearmoe_layer_destroy(layer: int) -> None:
    _check(lib().clearmoe_layer_destroy(layer), "clearmoe_layer_destroy")


def _router(Wg, bg) -> clearmoe_router:
    return clearmoe_router(_ptr(Wg), _ptr(bg))


def clearmoe_route(layer: int, x, Wg, bg, stream=None) -> None:
    r = _router(Wg, bg)
    _check(lib().clearmoe_route(layer, _ptr(x), x.shape[0], ctypes.byref(r), Wg.shape[0],
                                _stream(stream)), "clearmoe_route")


def clearmoe_route_mlp(layer: int, x, mlp: clearmoe_mlp_router, E: int, stream=None) -> None:
    _check(lib().clearmoe_route_mlp(layer, _ptr(x), x.shape[0], ctypes.byref(mlp), E, _stream(stream)),
           "clearmoe_route_mlp")


def clearmoe_ffn_forward(layer: int, x, W1, b1, U_r, S_r, Vh_r, residual_e, Wg, bg, out,
                         stream=None) -> None:
    """residual_e: a sequence of E [d x H] tensors, or one [E x d x H] tensor."""
    E = Wg.shape[0]
    res = _ptrs(residual_e, E)
    r = _router(Wg, bg)
    _check(lib().clearmoe_ffn_forward(layer, _ptr(x), x.shape[0], _ptr(W1), _ptr(b1), _ptr(U_r),
                                      _ptr(S_r), _ptr(Vh_r), res, ctypes.byref(r), E,
                                      S_r.shape[0], _ptr(out), _stream(stream)),
           "clearmoe_ffn_forward")


def clearmoe_ffn_forward_ex(layer: int, x, W1, b1, U_r, S_r, Vh_r, residual_e, Wg, bg, out,
                            b2=None, W2=None, cls_stride: int = 0, mlp: clearmoe_mlp_router | None = None,
                            E: int | None = None, input_layernorm: bool = False, router_in_fc1: bool = False,
                            stream=None) -> None:
    """clearmoe_ffn_forward with fc2's bias b2, class tokens (every cls_stride-th token from token 0)
    on the dense path W2, the MLP router `mlp` (then Wg, bg may be None and E is given),
    input_layernorm (x is the un-normalised stream y; the layer's input is LN(y)), and
    router_in_fc1 (the linear router's logits computed inside fc1)."""
    E = Wg.shape[0] if E is None else E
    res = _ptrs(residual_e, E)
    r = _router(Wg, bg) if Wg is not None else None
    opt = _options(b2, W2, cls_stride, mlp, input_layernorm, router_in_fc1)
    _check(lib().clearmoe_ffn_forward_ex(layer, _ptr(x), x.shape[0], _ptr(W1), _ptr(b1), _ptr(U_r),
                                         _ptr(S_r), _ptr(Vh_r), res, ctypes.byref(r) if r else None, E,
                                         S_r.shape[0], ctypes.byref(opt), _ptr(out),
                                         _stream(stream)), "clearmoe_ffn_forward_ex")


def clearmoe_fold_basis(layer: int, U_r, S_r, Vh_r, residual_e, W_comb, stream=None) -> None:
    """residual_e, W_comb: sequences of E [d x H] tensors, or [E x d x H] tensors."""
    E = len(residual_e)
    res = _ptrs(residual_e, E)
    comb = _ptrs(W_comb, E)
    _check(lib().clearmoe_fold_basis(layer, _ptr(U_r), _ptr(S_r), _ptr(Vh_r), res, E, S_r.shape[0],
                                     comb, _stream(stream)), "clearmoe_fold_basis")


def clearmoe_ffn_forward_folded(layer: int, x, W1, b1, W_comb, Wg, bg, out, stream=None) -> None:
    E = Wg.shape[0]
    comb = _ptrs(W_comb, E)
    r = _router(Wg, bg)
    _check(lib().clearmoe_ffn_forward_folded(layer, _ptr(x), x.shape[0], _ptr(W1), _ptr(b1), comb,
                                             ctypes.byref(r), E, _ptr(out), _stream(stream)),
           "clearmoe_ffn_forward_folded")


def clearmoe_materialize_basis(layer: int, U_r, S_r, Vh_r, W_sh, stream=None) -> None:
    _check(lib().clearmoe_materialize_basis(layer, _ptr(U_r), _ptr(S_r), _ptr(Vh_r), S_r.shape[0],
                                            _ptr(W_sh), _stream(stream)), "clearmoe_materialize_basis")


def clearmoe_ffn_forward_materialized(layer: int, x, W1, b1, W_sh, residual_e, Wg, bg, out,
                                      stream=None) -> None:
    E = Wg.shape[0]
    res = _ptrs(residual_e, E)
    r = _router(Wg, bg)
    _check(lib().clearmoe_ffn_forward_materialized(layer, _ptr(x), x.shape[0], _ptr(W1), _ptr(b1),
                                                   _ptr(W_sh), res, ctypes.byref(r), E, _ptr(out),
                                                   _stream(stream)), "clearmoe_ffn_forward_materialized")


def clearmoe_ffn_forward_scaled(layer: int, x, W1, b1, U_r, S_r, Vh_r, R, s_e, Wg, bg, out,
                                stream=None) -> None:
    r = _router(Wg, bg)
    _check(lib().clearmoe_ffn_forward_scaled(layer, _ptr(x), x.shape[0], _ptr(W1), _ptr(b1), _ptr(U_r),
                                             _ptr(S_r), _ptr(Vh_r), _ptr(R), _ptr(s_e), ctypes.byref(r),
                                             Wg.shape[0], S_r.shape[0], _ptr(out), _stream(stream)),
           "clearmoe_ffn_forward_scaled")


def _options(b2, W2, cls_stride, mlp, input_layernorm=False, router_in_fc1=False):
    return clearmoe_ffn_options(_ptr(b2), int(cls_stride), _ptr(W2),
                                ctypes.pointer(mlp) if mlp is not None else None, int(bool(input_layernorm)),
                                int(bool(router_in_fc1)))


def clearmoe_ffn_forward_folded_ex(layer: int, x, W1, b1, W_comb, Wg, bg, out, b2=None, W2=None,
                                   cls_stride: int = 0, mlp: clearmoe_mlp_router | None = None,
                                   E: int | None = None, input_layernorm: bool = False,
                                   router_in_fc1: bool = False, stream=None) -> None:
    E = Wg.shape[0] if E is None else E
    comb = _ptrs(W_comb, E)
    r = _router(Wg, bg) if Wg is not None else None
    opt = _options(b2, W2, cls_stride, mlp, input_layernorm, router_in_fc1)
    _check(lib().clearmoe_ffn_forward_folded_ex(layer, _ptr(x), x.shape[0], _ptr(W1), _ptr(b1), comb,
                                                ctypes.byref(r) if r else None, E, ctypes.byref(opt),
                                                _ptr(out), _stream(stream)), "clearmoe_ffn_forward_folded_ex")


def clearmoe_ffn_forward_materialized_ex(layer: int, x, W1, b1, W_sh, residual_e, Wg, bg, out, b2=None,
                                         W2=None, cls_stride: int = 0,
                                         mlp: clearmoe_mlp_router | None = None, E: int | None = None,
                                         input_layernorm: bool = False, router_in_fc1: bool = False,
                                         stream=None) -> None:
    E = Wg.shape[0] if E is None else E
    res = _ptrs(residual_e, E)
    r = _router(Wg, bg) if Wg is not None else None
    opt = _options(b2, W2, cls_stride, mlp, input_layernorm, router_in_fc1)
    _check(lib().clearmoe_ffn_forward_materialized_ex(layer, _ptr(x), x.shape[0], _ptr(W1), _ptr(b1),
                                                      _ptr(W_sh), res, ctypes.byref(r) if r else None, E,
                                                      ctypes.byref(opt), _ptr(out), _stream(stream)),
           "clearmoe_ffn_forward_materialized_ex")


def clearmoe_dense_ffn_forward(layer: int, x, W1, b1, W2, out, stream=None) -> None:
    _check(lib().clearmoe_dense_ffn_forward(layer, _ptr(x), x.shape[0], _ptr(W1), _ptr(b1),
                                            _ptr(W2), _ptr(out), _stream(stream)),
           "clearmoe_dense_ffn_forward")


def clearmoe_dense_ffn_forward_ex(layer: int, x, W1, b1, W2, b2, out, stream=None) -> None:
    _check(lib().clearmoe_dense_ffn_forward_ex(layer, _ptr(x), x.shape[0], _ptr(W1), _ptr(b1),
                                               _ptr(W2), _ptr(b2), _ptr(out), _stream(stream)),
           "clearmoe_dense_ffn_forward_ex")


def clearmoe_dense_ffn_forward_opt(layer: int, x, W1, b1, W2, out, b2=None, input_layernorm: bool = False,
                                   stream=None) -> None:
    """The dense FFN with fc2's bias b2 and input_layernorm (x is y; the input is LN(y))."""
    opt = _options(b2, None, 0, None, input_layernorm)
    _check(lib().clearmoe_dense_ffn_forward_opt(layer, _ptr(x), x.shape[0], _ptr(W1), _ptr(b1), _ptr(W2),
                                                ctypes.byref(opt), _ptr(out), _stream(stream)),
           "clearmoe_dense_ffn_forward_opt")


def clearmoe_layer_norm(layer: int, y, x_out, stream=None) -> None:
    _check(lib().clearmoe_layer_norm(layer, _ptr(y), y.shape[0], _ptr(x_out), _stream(stream)),
           "clearmoe_layer_norm")


def clearmoe_get_routing(layer: int, idx=None, counts=None, offsets=None, perm=None,
                         stream=None) -> None:
    _check(lib().clearmoe_get_routing(layer, _ptr(idx), _ptr(counts), _ptr(offsets), _ptr(perm),
                                      _stream(stream)), "clearmoe_get_routing")


def clearmoe_layer_status(layer: int) -> int:
    return lib().clearmoe_layer_status(layer)


def clearmoe_debug_set_wait(layer: int, wait_limit_ns: int, phantom_arrivals: int) -> None:
    _check(lib().clearmoe_debug_set_wait(layer, wait_limit_ns, phantom_arrivals),
           "clearmoe_debug_set_wait")


def clearmoe_set_profile_events(layer: int, events) -> None:
    """events: torch.cuda.Event(enable_timing=True) objects (or none to stop recording). torch
    creates an event's CUDA handle on its first record, so each is recorded once here first; the
    library then re-records it on the forward's stream."""
    for e in events:
        if not e.cuda_event:
            e.record()
    handles = [e.cuda_event for e in events]
    arr = (ctypes.c_void_p * max(1, len(handles)))(*handles)
    _check(lib().clearmoe_set_profile_events(layer, arr, len(handles)),
           "clearmoe_set_profile_events")


def clearmoe_route_noalloc(x, Wg, bg, idx, counts, offsets, perm, status=None,
                           stream=None) -> None:
    """Routing without a handle or any device allocation (see include/clearmoe.h): the outputs
    idx [T], counts [E], offsets [E + 1], perm [T] (int32) and the optional status word are
    caller-owned CUDA tensors."""
    import torch
    dtype = BF16 if x.dtype == torch.bfloat16 else F32
    r = _router(Wg, bg)
    _check(lib().clearmoe_route_noalloc(_ptr(x), x.shape[0], x.shape[1], dtype, ctypes.byref(r),
                                        Wg.shape[0], _ptr(idx), _ptr(counts), _ptr(offsets),
                                        _ptr(perm), _ptr(status), _stream(stream)),
           "clearmoe_route_noalloc")


# ---------------------------------------------------------------- 8-bit blocks with power-of-two scales
def _device_of(q, scale) -> int:
    """The GPU that both parts of a matrix in blocks lie on, -1 where they do not say."""
    at = [t.get_device() if hasattr(t, "get_device") else -1 for t in (q, scale)]
    if at[0] != at[1]:
        raise ValueError(f"q and scale of one matrix lie on GPU {at[0]} and GPU {at[1]}")
    return at[0]


class Fp8Matrix:
    """A matrix [rows x cols] in 8-bit blocks (clearmoe_fp8): q, one byte per element in rows of cols rounded up
    to 128 (float8_e4m3fn or uint8), and its scale bytes, rows of 4 ceil(cols / 512); 128-row blocks for weights,
    1-row blocks otherwise. Keeps the tensors alive."""

    def __init__(self, q, scale, rows: int, cols: int, weight: bool = False):
        n_scale = -(-rows // 128) if weight else rows
        for name, t, shape in (("q", q, (rows, fp8_pitch(cols))), ("scale", scale, (n_scale, fp8_scale_pitch(cols)))):
            if tuple(t.shape) != shape or t.element_size() != 1:
                raise ValueError(f"{name} of a {rows} x {cols} matrix in 8-bit blocks is one byte per element of {shape}, "
                                 f"got {tuple(t.shape)} {t.dtype}")
        self.q, self.scale, self.rows, self.cols, self.weight = q, scale, rows, cols, weight
        self.c = _PlacedFp8(_ptr(q), _ptr(scale), rows, cols, _device_of(q, scale))
        self.ref, self.addr = ctypes.cast(ctypes.pointer(self.c), ctypes.POINTER(clearmoe_fp8)), ctypes.addressof(self.c)

    def get_device(self) -> int:
        return self.c.device


def fp8_pitch(cols: int) -> int:
    """Bytes from one row of q to the next."""
    return -(-cols // 128) * 128


def fp8_scale_pitch(cols: int) -> int:
    """Bytes from one row of scales to the next."""
    return -(-cols // 512) * 4


def _fp8_empty(rows, cols, weight, device):
    import torch
    q = torch.empty(rows, fp8_pitch(cols), dtype=torch.float8_e4m3fn, device=device)
    n = -(-rows // 128) if weight else rows
    return Fp8Matrix(q, torch.empty(n, fp8_scale_pitch(cols), dtype=torch.uint8, device=device), rows, cols, weight)


def fp8_rows(rows: int, cols: int, device="cuda") -> Fp8Matrix:
    """Buffers for activations in 8-bit blocks, to be written by clearmoe_fp8_quantize_rows or a product."""
    return _fp8_empty(rows, cols, False, device)


def fp8_weight(rows: int, cols: int, device="cuda") -> Fp8Matrix:
    """Buffers for a weight matrix in 8-bit blocks, to be written by clearmoe_fp8_quantize_weight."""
    return _fp8_empty(rows, cols, True, device)


def _refuse_kind(what, weight):
    raise ValueError(f"{what} must be a matrix in 8-bit blocks of {'weights (fp8_weight)' if weight else 'rows (fp8_rows)'}: its "
                     f"scales have one row per {'128 rows' if weight else 'row'}")


_DTYPES = {}  # torch dtype -> clearmoe_dtype, filled on first use (torch is imported late)


def _dtype(t) -> int:
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        dt = {"torch.bfloat16": BF16, "torch.float32": F32}.get(str(t.dtype))
        if dt is None:
            raise ValueError(f"matrices must be bfloat16 or float32, got {t.dtype}")
        _DTYPES[t.dtype] = dt
    return dt


def _int32(t, n, what):
    """Pointer of n int32 values (n None: one or more) on the GPU, or None."""
    if t is None:
        return None
    if str(t.dtype) != "torch.int32" or (t.numel() != n if n is not None else t.numel() < 1):
        raise ValueError(f"{what} must be int32 with {n or 'at least one'} entries, got {t.numel()} of {t.dtype}")
    return _ptr(t)


def _matrix(t, rows, cols, what):
    """Pointer, dtype and row pitch of a [rows x cols] CUDA tensor whose rows are dense (any pitch; rows None: any
    number)."""
    shape = t.shape
    if not t.is_cuda or len(shape) != 2:
        raise ValueError("matrices passed to libclearmoe must be 2-D CUDA tensors with dense rows")
    n, k = shape
    if (rows is not None and n != rows) or k != cols:
        raise ValueError(f"{what} must be [{'any' if rows is None else rows} x {cols}], got {tuple(shape)}")
    ld, step = t.stride()
    if k > 1 and step != 1:
        raise ValueError("matrices passed to libclearmoe must be 2-D CUDA tensors with dense rows")
    return t.data_ptr(), _dtype(t), ld if n > 1 else max(ld, k)


def clearmoe_fp8_quantize_rows(x, out: Fp8Matrix, gather=None, stream=None) -> None:
    """x [rows x cols] (bf16 or fp32, any row pitch) to out in 1 x 128 blocks; gather: int32 source rows (one outside x
    gives a row of NaN)."""
    if getattr(out, "weight", False):
        _refuse_kind("out", False)
    calls = _calls or _bind_calls()
    if gather is not None:
        p, dt, ld = _matrix(x, None, out.cols, "x")
        _check(lib().clearmoe_fp8_quantize_gathered(p, x.shape[0], dt, ld, _int32(gather, out.rows, "gather"), out.ref,
                                                    _stream(stream)), "clearmoe_fp8_quantize_gathered")
        return
    code = calls.quantize_rows_t(x, out.rows, out.cols, out.addr, stream)
    if code is None:
        p, dt, ld = _matrix(x, out.rows, out.cols, "x")
        code = calls.quantize_rows(p, dt, ld, None, out.addr, _stream(stream))
    if code:
        raise ClearMoEError(code, "clearmoe_fp8_quantize_rows")


def clearmoe_fp8_quantize_weight(W, out: Fp8Matrix, stream=None) -> None:
    """W [rows x cols] (bf16 or fp32, any row pitch) to out in 128 x 128 blocks."""
    if not getattr(out, "weight", True):
        _refuse_kind("out", True)
    p, dt, ld = _matrix(W, out.rows, out.cols, "W")
    _check(lib().clearmoe_fp8_quantize_weight(p, dt, ld, out.ref, _stream(stream)), "clearmoe_fp8_quantize_weight")


def clearmoe_fp8_dequantize(m: Fp8Matrix, out, stream=None) -> None:
    """The values m stands for, rounded to out's dtype (bf16 or fp32)."""
    p, dt, ld = _matrix(out, m.rows, m.cols, "out")
    _check(lib().clearmoe_fp8_dequantize(m.ref, 128 if m.weight else 1, p, dt, ld, _stream(stream)),
           "clearmoe_fp8_dequantize")


def _epilogue(bias, act, status, N):
    if bias is None and act == ACT_NONE and status is None:
        return None
    if bias is not None and bias.numel() != N:
        raise ValueError(f"bias must have {N} elements, got {bias.numel()}")
    return ctypes.byref(clearmoe_fp8_epilogue(_ptr(bias), F32 if bias is None else _dtype(bias), act,
                                              _int32(status, None, "status")))


def clearmoe_fp8_gemm(A: Fp8Matrix, W: Fp8Matrix, out, bias=None, act: int = ACT_NONE, status=None, stream=None) -> None:
    """out = act(A W^T + bias). out: a [M x N] bf16 or fp32 tensor of any row pitch, or an Fp8Matrix of rows (the
    result quantised, clearmoe_fp8_gemm_fp8)."""
    if getattr(A, "weight", False):
        _refuse_kind("A", False)
    if not getattr(W, "weight", True):
        _refuse_kind("W", True)
    calls = _calls or _bind_calls()
    blocks = isinstance(out, Fp8Matrix)
    if blocks and out.weight:
        _refuse_kind("out", False)
    if not blocks:
        code = calls.gemm_t(A.addr, W.addr, A.rows, W.rows, act, bias, status, out, stream)
        if code is not None:
            if code:
                raise ClearMoEError(code, "clearmoe_fp8_gemm")
            return
    bp, bdt = None, F32
    if bias is not None:
        if bias.numel() != W.rows:
            raise ValueError(f"bias must have {W.rows} elements, got {bias.numel()}")
        bp, bdt = _ptr(bias), _dtype(bias)
    sp = _int32(status, None, "status")
    if blocks:
        code = calls.gemm_fp8(A.addr, W.addr, bp, bdt, act, sp, out.addr, _stream(stream))
        if code:
            raise ClearMoEError(code, "clearmoe_fp8_gemm_fp8")
        return
    p, dt, ld = _matrix(out, A.rows, W.rows, "out")
    code = calls.gemm(A.addr, W.addr, bp, bdt, act, sp, p, dt, ld, _stream(stream))
    if code:
        raise ClearMoEError(code, "clearmoe_fp8_gemm")


def clearmoe_fp8_grouped_gemm(A: Fp8Matrix, W, offsets, out, perm=None, bias=None, act: int = ACT_NONE, status=None,
                              stream=None) -> None:
    """Rows offsets[e] .. offsets[e + 1] of A times W[e]^T (W: a sequence of Fp8Matrix), row i to out[perm[i]]."""
    if getattr(A, "weight", False):
        _refuse_kind("A", False)
    if not all(getattr(m, "weight", True) for m in W):
        _refuse_kind("every W", True)
    if not len(W) or offsets is None:
        raise ValueError("a grouped product needs matrices and the offsets of their rows")
    off, rows = _int32(offsets, len(W) + 1, "offsets"), _int32(perm, A.rows, "perm")
    p, dt, ld = _matrix(out, A.rows, W[0].rows, "out")
    arr = (clearmoe_fp8 * len(W))(*[m.c for m in W])
    _check(lib().clearmoe_fp8_grouped_gemm(A.ref, arr, len(W), off, rows,
                                           _epilogue(bias, act, status, W[0].rows), p, dt, ld, _stream(stream)),
           "clearmoe_fp8_grouped_gemm")


def clearmoe_debug_fp8_kernel(width: int = 0, pair: int = 0) -> None:
    """For tests: fixes the kernel of the calling thread's later products of 8-bit blocks; no arguments: by size again."""
    _check(lib().clearmoe_debug_fp8_kernel(width, pair), "clearmoe_debug_fp8_kernel")


# ---------------------------------------------------------------- 4-bit blocks with power-of-two scales
class Fp4Matrix:
    """A matrix [rows x cols] in 4-bit blocks (clearmoe_fp4), activations or weights: q, two values a byte in rows of cols
    rounded up to 64 values (uint8), and its scale bytes, [ceil(rows / 128) x ceil(cols / 128) x 512] (uint8). Keeps the
    tensors alive."""

    def __init__(self, q, scale, rows: int, cols: int):
        for name, t, shape in (("q", q, (rows, fp4_pitch(cols))), ("scale", scale, (-(-rows // 128), -(-cols // 128), 512))):
            if tuple(t.shape) != shape or t.element_size() != 1:
                raise ValueError(f"{name} of a {rows} x {cols} matrix in 4-bit blocks is bytes of {shape}, got {tuple(t.shape)} "
                                 f"{t.dtype}")
        self.q, self.scale, self.rows, self.cols = q, scale, rows, cols
        self.c = _PlacedFp4(_ptr(q), _ptr(scale), rows, cols, _device_of(q, scale))
        self.ref, self.addr = ctypes.cast(ctypes.pointer(self.c), ctypes.POINTER(clearmoe_fp4)), ctypes.addressof(self.c)

    def get_device(self) -> int:
        return self.c.device

    @property
    def weight(self):
        """What the calls on 8-bit blocks ask of a matrix first: this one is refused there."""
        raise ValueError("a matrix in 8-bit blocks (fp8_rows, fp8_weight) is needed, got one in 4-bit blocks")


def fp4_pitch(cols: int) -> int:
    """Bytes from one row of q to the next."""
    return -(-cols // 64) * 32


def fp4_matrix(rows: int, cols: int, device="cuda") -> Fp4Matrix:
    """Buffers for a matrix in 4-bit blocks, to be written by clearmoe_fp4_quantize, a product or a norm."""
    import torch
    q = torch.empty(rows, fp4_pitch(cols), dtype=torch.uint8, device=device)
    return Fp4Matrix(q, torch.empty(-(-rows // 128), -(-cols // 128), 512, dtype=torch.uint8, device=device), rows, cols)


def _fp4(m, what):
    """The address of a matrix in 4-bit blocks: what the library sees of it does not tell it from one in 8-bit blocks."""
    if not isinstance(m, Fp4Matrix):
        raise ValueError(f"{what} must be a matrix in 4-bit blocks (fp4_matrix), got {type(m).__name__}")
    return m.ref


def _here(stream, *tensors):
    """Tensors on another GPU than the stream's are refused: the kernels would read them across, or fault."""
    if stream is not None:
        here = getattr(stream, "device_index", None)
    else:
        import torch
        here = torch.cuda.current_device() if torch.cuda.is_initialized() else None
    for t in tensors:
        at = t.get_device() if hasattr(t, "get_device") else here
        if here is not None and at >= 0 and at != here:
            raise ValueError(f"a tensor on GPU {at} was passed to a call on a stream of GPU {here}")


def clearmoe_fp4_quantize(x, out: Fp4Matrix, gather=None, stream=None) -> None:
    """x [rows x cols] (bf16 or fp32, any row pitch) to out in 4-bit blocks, weights and activations alike; gather: int32
    source rows (one outside x gives a row of NaN)."""
    o = _fp4(out, "out")
    if gather is None:
        code = (_calls or _bind_calls()).fp4_quantize_t(x, out.addr, stream)
        if code is not None:
            if code:
                raise ClearMoEError(code, "clearmoe_fp4_quantize")
            return
    _here(stream, x, gather, out)
    p, dt, ld = _matrix(x, out.rows if gather is None else None, out.cols, "x")
    _check(lib().clearmoe_fp4_quantize(p, x.shape[0], dt, ld, _int32(gather, out.rows, "gather"), o, _stream(stream)),
           "clearmoe_fp4_quantize")


def clearmoe_fp4_dequantize(m: Fp4Matrix, out, stream=None) -> None:
    """The values m stands for, rounded to out's dtype (bf16 or fp32)."""
    r = _fp4(m, "m")
    _here(stream, m, out)
    p, dt, ld = _matrix(out, m.rows, m.cols, "out")
    _check(lib().clearmoe_fp4_dequantize(r, p, dt, ld, _stream(stream)), "clearmoe_fp4_dequantize")


def clearmoe_fp4_gemm(A: Fp4Matrix, W: Fp4Matrix, out, bias=None, act: int = ACT_NONE, status=None, stream=None) -> None:
    """out = act(A W^T + bias). out: a [M x N] bf16 or fp32 tensor of any row pitch, or an Fp4Matrix (the result
    quantised, clearmoe_fp4_gemm_fp4)."""
    blocks = isinstance(out, Fp4Matrix)
    if isinstance(A, Fp4Matrix) and isinstance(W, Fp4Matrix):
        code = (_calls or _bind_calls()).fp4_gemm_t(A.addr, W.addr, act, bias, status, out.addr if blocks else out, stream)
        if code is not None:
            if code:
                raise ClearMoEError(code, "clearmoe_fp4_gemm_fp4" if blocks else "clearmoe_fp4_gemm")
            return
    a, w = _fp4(A, "A"), _fp4(W, "W")
    _here(stream, A, W, bias, status, out)
    epi = _epilogue(bias, act, status, W.rows)
    if blocks:
        _check(lib().clearmoe_fp4_gemm_fp4(a, w, epi, out.ref, _stream(stream)), "clearmoe_fp4_gemm_fp4")
        return
    p, dt, ld = _matrix(out, A.rows, W.rows, "out")
    _check(lib().clearmoe_fp4_gemm(a, w, epi, p, dt, ld, _stream(stream)), "clearmoe_fp4_gemm")


def clearmoe_fp4_grouped_gemm(A: Fp4Matrix, W, offsets, out, perm=None, bias=None, act: int = ACT_NONE, status=None,
                              stream=None) -> None:
    """Rows offsets[e] .. offsets[e + 1] of A times W[e]^T (W: a sequence of Fp4Matrix), row i to out[perm[i]]."""
    a = _fp4(A, "A")
    if not len(W) or offsets is None:
        raise ValueError("a grouped product needs matrices and the offsets of their rows")
    for m in W:
        _fp4(m, "every W")
    _here(stream, A, *W, offsets, out, perm, bias, status)
    off, rows = _int32(offsets, len(W) + 1, "offsets"), _int32(perm, A.rows, "perm")
    p, dt, ld = _matrix(out, A.rows, W[0].rows, "out")
    arr = (clearmoe_fp4 * len(W))(*[m.c for m in W])
    _check(lib().clearmoe_fp4_grouped_gemm(a, arr, len(W), off, rows, _epilogue(bias, act, status, W[0].rows), p, dt, ld,
                                           _stream(stream)), "clearmoe_fp4_grouped_gemm")


def clearmoe_debug_fp4_kernel(width: int = 0, pair: int = 0) -> None:
    """For tests: fixes the kernel of the calling thread's later products of 4-bit blocks; no arguments: by size again."""
    _check(lib().clearmoe_debug_fp4_kernel(width, pair), "clearmoe_debug_fp4_kernel")


def clearmoe_debug_fp4_wait(wait_limit_ns: int = 0) -> None:
    """For tests: the limit of the waits in the calling thread's later products of 4-bit blocks; no argument: 1 s again."""
    _check(lib().clearmoe_debug_fp4_wait(wait_limit_ns), "clearmoe_debug_fp4_wait")


# ------------------------------------------------------------------- residual addition and RMS norm
def clearmoe_rms_norm(x, out, residual=None, sum_out=None, weight=None, eps: float = 1e-6, stream=None) -> None:
    """s = x + residual, rounded to x's dtype, to sum_out; s weight / sqrt(mean(s^2) + eps) to out: a [rows x cols] bf16
    or fp32 tensor, or an Fp8Matrix of rows or an Fp4Matrix (the norm quantised, clearmoe_rms_norm_fp8, _fp4). x,
    residual and sum_out are of one dtype, of any row pitch; sum_out may be x or residual."""
    bits = 4 if isinstance(out, Fp4Matrix) else 8 if isinstance(out, Fp8Matrix) else 0
    if bits == 8 and out.weight:
        _refuse_kind("out", False)
    code = (_calls or _bind_calls()).rms_norm_t(x, residual, sum_out, weight, eps, bits, out.addr if bits else out, stream)
    if code is not None:
        if code:
            raise ClearMoEError(code, "clearmoe_rms_norm" + ("", "_fp4", "_fp8")[bits // 4])
        return
    _here(stream, x, residual, sum_out, weight, out)
    if len(x.shape) != 2:
        raise ValueError(f"x must be a matrix, got {tuple(x.shape)}")
    rows, cols = x.shape
    n = clearmoe_norm(rows=rows, cols=cols, eps=eps)
    n.x, n.dtype, n.ldx = _matrix(x, rows, cols, "x")
    for name, t in (("residual", residual), ("sum_out", sum_out)):
        if t is not None:
            p, dt, ld = _matrix(t, rows, cols, name)
            if dt != n.dtype:
                raise ValueError(f"{name} must be of x's dtype, got {t.dtype} and {x.dtype}")
            if name == "residual":
                n.residual, n.ldr = p, ld
            else:
                n.sum, n.lds = p, ld
    if weight is not None:
        if weight.numel() != cols:
            raise ValueError(f"weight must have {cols} elements, got {weight.numel()}")
        n.weight, n.weight_dtype = _ptr(weight), _dtype(weight)
    ref = ctypes.byref(n)
    if bits == 4:
        _check(lib().clearmoe_rms_norm_fp4(ref, out.ref, _stream(stream)), "clearmoe_rms_norm_fp4")
    elif bits == 8:
        _check(lib().clearmoe_rms_norm_fp8(ref, out.ref, _stream(stream)), "clearmoe_rms_norm_fp8")
    else:
        p, dt, ld = _matrix(out, rows, cols, "out")
        _check(lib().clearmoe_rms_norm(ref, p, dt, ld, _stream(stream)), "clearmoe_rms_norm")


# ------------------------------------------------------------- a folded layer's weights and its forwards
class FfnWeights:
    """A folded layer's weights bound once (clearmoe_ffn_weights), with the tensors kept alive; d and the layer's dtype, which
    tokens have to be of."""

    def __init__(self, c, keep, d: int, dtype: int):
        self.c, self.keep, self.d, self.dtype = c, keep, d, dtype
        self.ref, self.addr = ctypes.pointer(c), ctypes.addressof(c)


def ffn_weights(W1, b1, W_comb, Wg, bg, b2=None, W2=None, cls_stride: int = 0,
                input_layernorm: bool = False) -> FfnWeights:
    """W1 [H x d], W_comb (E matrices [d x H]) and W2 (class tokens' dense path) as tensors of the layer's dtype, or
    all as Fp8Matrix weights; b1, b2, Wg, bg in the layer's dtype."""
    E, d = Wg.shape
    layer = _dtype(Wg)
    if len(W_comb) != E or E > 16:
        raise ValueError(f"{E} experts (at most 16) need as many matrices, got {len(W_comb)}")
    fp8 = isinstance(W1, Fp8Matrix)
    H = W1.rows if fp8 else W1.shape[0]

    def mat(W, rows, cols):
        if isinstance(W, Fp8Matrix) != fp8 or (fp8 and not W.weight):
            raise ValueError("W1, W_comb and W2 are all tensors or all Fp8Matrix weights")
        shape = (W.rows, W.cols) if fp8 else tuple(W.shape)
        if shape != (rows, cols):
            raise ValueError(f"a weight matrix must be [{rows} x {cols}], got {shape}")
        if fp8:
            return W.c
        if _dtype(W) != layer:
            raise ValueError(f"W1, W_comb and W2 must be of the router's dtype, got {W.dtype} and {Wg.dtype}")
        return clearmoe_fp8(_ptr(W), None, rows, cols)

    for name, t, n in (("b1", b1, H), ("bg", bg, E), ("b2", b2, d)):
        if t is not None and (t.numel() != n or _dtype(t) != layer):
            raise ValueError(f"{name} must have {n} elements of the router's dtype, got {t.numel()} of {t.dtype}")
    if fp8 and layer != BF16:
        raise ValueError(f"8-bit weights are of bf16 layers: b1, b2, Wg and bg must be bfloat16, got {Wg.dtype}")
    c = clearmoe_ffn_weights()
    c.dtype = FP8 if fp8 else layer
    c.E = E
    c.W1 = mat(W1, H, d)
    for e in range(E):
        c.W_comb[e] = mat(W_comb[e], d, H)
    if W2 is not None:
        c.W2 = mat(W2, d, H)
    c.b1, c.b2 = _ptr(b1), _ptr(b2)
    c.router = _router(Wg, bg)
    c.cls_stride, c.input_layernorm = int(cls_stride), int(bool(input_layernorm))
    return FfnWeights(c, (W1, b1, list(W_comb), Wg, bg, b2, W2), d, layer)


def _tokens(x, out, w):
    """Number of tokens and pointers of x and out, both [T x d] in the layer's dtype."""
    for name, t in (("x", x), ("out", out)):
        if len(t.shape) != 2 or t.shape[1] != w.d or t.shape[0] != x.shape[0] or _dtype(t) != w.dtype:
            raise ValueError(f"{name} must be [T x {w.d}] in the layer's dtype, x and out of the same T; got {tuple(t.shape)} {t.dtype}")
    return x.shape[0], _ptr(x), _ptr(out)


def clearmoe_ffn_forward_few(layer: int, x, w: FfnWeights, out, stream=None) -> None:
    """The whole folded layer for 1 to FEW_MAX tokens: x and out [T x d] in the layer's dtype."""
    calls = _calls or _bind_calls()
    code = calls.ffn_few_t(layer, w.addr, x, out, stream)
    if code is None:
        T, xp, op = _tokens(x, out, w)
        code = calls.ffn_few(layer, xp, T, w.addr, op, _stream(stream))
    if code:
        raise ClearMoEError(code, "clearmoe_ffn_forward_few")


def clearmoe_ffn_forward_fp8(layer: int, x, w: FfnWeights, out, stream=None) -> None:
    """The whole folded layer with both products in 8-bit blocks: x and out [T x d] bf16."""
    calls = _calls or _bind_calls()
    code = calls.ffn_fp8_t(layer, w.addr, x, out, stream)
    if code is None:
        T, xp, op = _tokens(x, out, w)
        code = calls.ffn_fp8(layer, xp, T, w.addr, op, _stream(stream))
    if code:
        raise ClearMoEError(code, "clearmoe_ffn_forward_fp8")
