"""Binding of the C ABI in include/svdcache.h (argument marshalling only): ctypes, and for the step calls with ordinary
arguments the compiled module _fast_calls, which makes the same call from the same tensors with less host time."""
from __future__ import annotations

import ctypes as C
import os
import warnings
from typing import Optional

import torch

PKG_DIR = os.path.dirname(os.path.abspath(__file__))

SVDC_F32, SVDC_BF16 = 0, 1
SVDC_PRECISE, SVDC_FAST = 0, 1
_DTYPES = {torch.float32: SVDC_F32, torch.bfloat16: SVDC_BF16}


class SvdcError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {svdcache_strerror(code)} (status {code})")


class Shape(C.Structure):
    """Mirror of svdc_shape."""
    _fields_ = [("B", C.c_int32), ("N", C.c_int32), ("D", C.c_int32), ("k", C.c_int32),
                ("ldf", C.c_int64), ("block_stride", C.c_int64), ("dtype", C.c_int32), ("precision", C.c_int32)]


class FitParams(C.Structure):
    """Mirror of svdc_fit_params."""
    _fields_ = [("oversample_p", C.c_int32), ("power_iters_q", C.c_int32), ("seed", C.c_uint64),
                ("jacobi_max_sweeps", C.c_int32), ("reserved", C.c_int32)]


class Norm8(C.Structure):
    """Mirror of svdc_norm8."""
    _fields_ = [("rows", C.c_int64), ("D", C.c_int32), ("dtype", C.c_int32), ("dtype_f", C.c_int32), ("eps", C.c_float),
                ("ldx", C.c_int64), ("ldf", C.c_int64), ("ldh", C.c_int64), ("ldy", C.c_int64)]


class Quant8(C.Structure):
    """Mirror of svdc_quant8."""
    _fields_ = [("rows", C.c_int64), ("D", C.c_int32), ("dtype", C.c_int32), ("ldx", C.c_int64), ("block_rows", C.c_int32),
                ("reserved", C.c_int32)]


class Matmul8(C.Structure):
    """Mirror of svdc_matmul8."""
    _fields_ = [("M", C.c_int64), ("N", C.c_int32), ("K", C.c_int32), ("dtype", C.c_int32), ("act", C.c_int32), ("ldo", C.c_int64)]


SVDC_MAX_AXES = 4


class Heads(C.Structure):
    """Mirror of svdc_heads."""
    _fields_ = [("seq", C.c_int64), ("row", C.c_int64), ("head", C.c_int64)]


class Rotary(C.Structure):
    """Mirror of svdc_rotary."""
    _fields_ = [("rows", C.c_int64), ("ld", C.c_int64), ("axes", C.c_int32), ("whole", C.c_int32), ("dims", C.c_int32 * SVDC_MAX_AXES),
                ("theta", C.c_double * SVDC_MAX_AXES)]


class NormRotate(C.Structure):
    """Mirror of svdc_norm_rotate."""
    _fields_ = [("batch", C.c_int64), ("rows", C.c_int64), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32), ("dtype_out", C.c_int32), ("norm", C.c_int32), ("pairs", C.c_int32), ("layout", C.c_int32),
                ("eps", C.c_float), ("reserved", C.c_int32), ("table_seq", C.c_int64), ("q", Heads), ("k", Heads), ("v", Heads),
                ("qo", Heads), ("ko", Heads), ("vo", Heads)]


class Attention(C.Structure):
    """Mirror of svdc_attention."""
    _fields_ = [("batch", C.c_int64), ("q_rows", C.c_int64), ("k_rows", C.c_int64), ("q_total", C.c_int64), ("k_total", C.c_int64),
                ("heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float),
                ("reserved", C.c_int32), ("q", Heads), ("k", Heads), ("v", Heads), ("o", Heads)]


EXPORTS = {
    "svdcache_version": (C.c_int32, []),
    "svdcache_strerror": (C.c_char_p, [C.c_int32]),
    "svdcache_fit_workspace_bytes": (C.c_size_t, [C.POINTER(Shape), C.POINTER(FitParams)]),
    "svdcache_workspace_bytes": (C.c_size_t, [C.POINTER(Shape), C.POINTER(FitParams)]),
    "svdcache_fit_status_offset": (C.c_size_t, [C.POINTER(Shape), C.POINTER(FitParams)]),
    "svdcache_packed_basis_bytes": (C.c_size_t, [C.POINTER(Shape)]),
    "svdcache_has_mfma_path": (C.c_int32, [C.POINTER(Shape)]),
    "svdcache_fit_basis": (C.c_int32, [C.POINTER(Shape), C.POINTER(FitParams), C.c_void_p, C.c_void_p, C.c_void_p,
                                       C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "svdcache_fit_basis_static": (C.c_int32, [C.POINTER(Shape), C.POINTER(FitParams), C.c_void_p, C.c_void_p,
                                              C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "svdcache_pack_basis": (C.c_int32, [C.POINTER(Shape), C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "svdcache_full_step": (C.c_int32, [C.POINTER(Shape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                       C.c_void_p, C.c_void_p, C.c_float, C.c_int32, C.c_void_p]),
    "svdcache_full_step_residual_ema": (C.c_int32, [C.POINTER(Shape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_float, C.c_float,
                                                    C.c_int32, C.c_void_p]),
    "svdcache_forecast": (C.c_int32, [C.POINTER(Shape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_void_p]),
    "svdcache_packed_state_bytes": (C.c_size_t, [C.POINTER(Shape)]),
    "svdcache_pack_state": (C.c_int32, [C.POINTER(Shape), C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "svdcache_full_step_packed": (C.c_int32, [C.POINTER(Shape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                              C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_float, C.c_int32,
                                              C.c_void_p]),
    "svdcache_forecast_packed": (C.c_int32, [C.POINTER(Shape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                             C.c_void_p]),
    "svdcache_select_rank": (C.c_int32, [C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_float, C.c_void_p,
                                         C.c_void_p, C.c_void_p]),
    "svdcache_truncate_basis": (C.c_int32, [C.POINTER(Shape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "svdcache_extrapolation_weights": (C.c_int32, [C.c_int32, C.c_double, C.c_double, C.POINTER(C.c_float)]),
    "svdcache_basis_overlap": (C.c_int32, [C.POINTER(Shape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "svdcache_rebase_state": (C.c_int32, [C.POINTER(Shape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "svdcache_basis_similarity": (C.c_int32, [C.POINTER(Shape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                              C.c_void_p, C.c_void_p, C.c_void_p]),
    "svdcache_forecast_combine": (C.c_int32, [C.POINTER(Shape), C.c_int32, C.POINTER(C.c_void_p),
                                              C.POINTER(C.c_float), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                              C.c_void_p, C.c_void_p]),
    "svdcache_q8_bytes": (C.c_size_t, [C.c_int64, C.c_int32]),
    "svdcache_q8_scale_bytes": (C.c_size_t, [C.c_int64, C.c_int32, C.c_int32]),
    "svdcache_rms_norm8": (C.c_int32, [C.POINTER(Norm8)] + [C.c_void_p] * 8),
    "svdcache_quantize8": (C.c_int32, [C.POINTER(Quant8)] + [C.c_void_p] * 4),
    "svdcache_matmul8_workspace_bytes": (C.c_size_t, [C.POINTER(Matmul8)]),
    "svdcache_matmul8": (C.c_int32, [C.POINTER(Matmul8)] + [C.c_void_p] * 8 + [C.c_size_t, C.c_void_p]),
    "svdcache_rotary_table": (C.c_int32, [C.POINTER(Rotary)] + [C.c_void_p] * 3),
    "svdcache_norm_rotate": (C.c_int32, [C.POINTER(NormRotate)] + [C.c_void_p] * 10),
    "svdcache_attention_workspace_bytes": (C.c_size_t, [C.POINTER(Attention)]),
    "svdcache_attention": (C.c_int32, [C.POINTER(Attention)] + [C.c_void_p] * 8 + [C.c_size_t, C.c_void_p]),
}

_lib = None
_fast = None      # the module _fast_calls, bound to the functions of _lib


def lib_path() -> str:
    return os.path.join(PKG_DIR, "libsvdcache.so")


def exported_symbols():
    return sorted(EXPORTS)


def load_library():
    """Load libsvdcache.so from the package directory; raises if it was not built."""
    global _lib, _fast
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2601_07396_amd.build` "
                           "(there is no fallback path)")
    lib = C.CDLL(path)
    for name, (res, args) in EXPORTS.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _fast = _load_fast_calls(lib)
    _lib = lib
    return lib


def _load_fast_calls(lib):
    """The module _fast_calls bound to `lib`, None where it was not built.  It is built against one torch: with another it may
    not load, and then all calls go through ctypes, which needs none of it."""
    path = os.path.join(PKG_DIR, "_fast_calls.so")
    if not os.path.exists(path):
        return None
    try:
        import importlib.util
        spec = importlib.util.spec_from_file_location("_fast_calls", path)
        fast = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(fast)
        fast.bind({name: C.cast(getattr(lib, name), C.c_void_p).value for name in EXPORTS}, Shape, Norm8, Quant8, Matmul8, Rotary,
                  NormRotate, Attention)
    except Exception as e:
        warnings.warn(f"{path} does not load ({e}): step calls take about 4 us more host time each; "
                      "build it again with `python -m paper_2601_07396_amd.build`", RuntimeWarning, stacklevel=3)
        return None
    return fast


def svdcache_version() -> int:
    return load_library().svdcache_version()


def svdcache_strerror(code: int) -> str:
    return load_library().svdcache_strerror(code).decode()


# The current stream's handle without building a torch.cuda.Stream object for every call (2.7 us of the 10 us that a call of
# a tiny problem took on the host).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _need_gpu(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise RuntimeError("svdcache: tensors must live in GPU memory (no CPU path exists)")


def make_shape(F: torch.Tensor, k: int, precision: int = SVDC_PRECISE) -> Shape:
    """Shape descriptor of a feature tensor [B, N, D] (or [N, D]) whose last dim is contiguous."""
    if F.dim() == 2:
        F = F.unsqueeze(0)
    if F.dim() != 3 or F.stride(2) != 1:
        raise ValueError("F must be [B, N, D] with a contiguous last dimension")
    if F.dtype not in _DTYPES:
        raise ValueError("F must be float32 or bfloat16")
    B, N, D = F.shape
    bs = F.stride(0) if B > 1 else max(F.stride(0), (N - 1) * F.stride(1) + D)
    return Shape(B, N, D, k, F.stride(1), bs, _DTYPES[F.dtype], precision)


_TORCH_OF = {SVDC_F32: torch.float32, SVDC_BF16: torch.bfloat16}


def _like_features(shape: Shape, **tensors):
    """The C ABI describes F, R, Fhat, X and R_prev by ONE (ldf, block_stride, dtype): refuse a tensor whose own
    layout differs (e.g. `empty_like` of a row-strided view comes back contiguous), which the kernels would
    otherwise address with the wrong strides, past the end of its allocation."""
    want, dims = _TORCH_OF[shape.dtype], (shape.B, shape.N, shape.D)
    strides = (shape.block_stride, shape.ldf, 1)
    for name, t in tensors.items():
        if t is None or (t.dtype is want and t.shape == dims and t.stride() == strides):   # the ordinary case
            continue
        if t.dtype != want:
            raise ValueError(f"{name}: dtype {t.dtype} differs from the feature dtype {want}")
        u = t.unsqueeze(0) if t.dim() == 2 else t
        if u.dim() != 3 or tuple(u.shape) != (shape.B, shape.N, shape.D):
            raise ValueError(f"{name}: shape {tuple(t.shape)} is not [B={shape.B}, N={shape.N}, D={shape.D}]")
        if u.stride(2) != 1 or u.stride(1) != shape.ldf or (shape.B > 1 and u.stride(0) != shape.block_stride):
            raise ValueError(f"{name}: strides {tuple(u.stride())} differ from the features' "
                             f"(block {shape.block_stride}, row {shape.ldf}, 1)")


def _dense_f32(count: int, what: str, **tensors):
    """V, S, C and their like are float32, contiguous, with exactly the element count the shape implies."""
    for name, t in tensors.items():
        if t is not None and (t.dtype is not torch.float32 or not t.is_contiguous() or t.numel() != count):
            raise ValueError(f"{name}: need a contiguous float32 tensor of {count} elements ({what}), got "
                             f"{t.dtype} {tuple(t.shape)} contiguous={t.is_contiguous()}")


def _check_step_args(shape: Shape, V, packed, coefs: dict, feats: dict):
    _like_features(shape, **feats)
    _dense_f32(shape.B * shape.D * shape.k, "[B, D, k]", V=V)
    _dense_f32(shape.B * shape.N * shape.k, "[B, N, k]", **coefs)
    if packed is not None:
        need = svdcache_packed_basis_bytes(shape)
        if need == 0 or packed.numel() * packed.element_size() < need or not packed.is_contiguous():
            raise ValueError(f"packed: {packed.numel() * packed.element_size()} bytes, this shape needs {need} "
                             "(a buffer packed for another rank or width?)")


def _fast_call(name: str, *args) -> bool:
    """Whether _fast_calls made the call; False where the arguments are not ordinary (or the module was not built)."""
    if _lib is None:
        load_library()
    code = None if _fast is None else getattr(_fast, name)(*args)
    if code:
        raise SvdcError(code, "svdcache_" + name)
    return code is not None


def _check(code: int, where: str):
    if code != 0:
        raise SvdcError(code, where)


SVDC_FIT_JACOBI_CAPPED, SVDC_FIT_RANK_DEFICIENT = 1, 2


def svdcache_fit_workspace_bytes(shape: Shape, p: int = 0, q: int = 0, seed: int = 0, max_sweeps: int = 0) -> int:
    fp = FitParams(p, q, seed, max_sweeps, 0)
    return load_library().svdcache_fit_workspace_bytes(C.byref(shape), C.byref(fp))


def svdcache_workspace_bytes(shape: Shape, p: int = 0, q: int = 0, seed: int = 0, max_sweeps: int = 0) -> int:
    fp = FitParams(p, q, seed, max_sweeps, 0)
    return load_library().svdcache_workspace_bytes(C.byref(shape), C.byref(fp))


def svdcache_fit_status_offset(shape: Shape, p: int = 0, q: int = 0, seed: int = 0, max_sweeps: int = 0) -> int:
    fp = FitParams(p, q, seed, max_sweeps, 0)
    return load_library().svdcache_fit_status_offset(C.byref(shape), C.byref(fp))


def svdcache_packed_basis_bytes(shape: Shape) -> int:
    return load_library().svdcache_packed_basis_bytes(C.byref(shape))


def svdcache_has_mfma_path(shape: Shape) -> bool:
    return bool(load_library().svdcache_has_mfma_path(C.byref(shape)))


def svdcache_fit_basis(shape: Shape, F, V, sigma, fro2, workspace, p: int = 0, q: int = 0, seed: int = 0,
                       max_sweeps: int = 0):
    _like_features(shape, F=F)
    _dense_f32(shape.B * shape.D * shape.k, "[B, D, k]", V=V)
    _dense_f32(shape.B * shape.k, "[B, k]", sigma=sigma)
    _dense_f32(shape.B, "[B]", fro2=fro2)
    _need_gpu(F, V, sigma, fro2, workspace)
    fp = FitParams(p, q, seed, max_sweeps, 0)
    rc = load_library().svdcache_fit_basis(C.byref(shape), C.byref(fp), _ptr(F), _ptr(V), _ptr(sigma), _ptr(fro2),
                                           _ptr(workspace), workspace.numel() * workspace.element_size(), _stream())
    _check(rc, "svdcache_fit_basis")


SVDC_STATIC_SCRATCH_BYTES = 32 << 20


def svdcache_fit_basis_static(shape: Shape, F, V, sigma, fro2, status=None, p: int = 0, q: int = 0, seed: int = 0,
                              max_sweeps: int = 0):
    """The fit on the library's static device workspace (no allocation inside the call)."""
    _like_features(shape, F=F)
    _dense_f32(shape.B * shape.D * shape.k, "[B, D, k]", V=V)
    _dense_f32(shape.B * shape.k, "[B, k]", sigma=sigma)
    _dense_f32(shape.B, "[B]", fro2=fro2)
    if status is not None and (status.dtype != torch.int32 or not status.is_contiguous() or status.numel() != shape.B):
        raise ValueError("status: need a contiguous int32 tensor of B elements")
    _need_gpu(F, V, sigma, fro2, status)
    fp = FitParams(p, q, seed, max_sweeps, 0)
    rc = load_library().svdcache_fit_basis_static(C.byref(shape), C.byref(fp), _ptr(F), _ptr(V), _ptr(sigma),
                                                  _ptr(fro2), _ptr(status), _stream())
    _check(rc, "svdcache_fit_basis_static")


def svdcache_pack_basis(shape: Shape, V, packed):
    _dense_f32(shape.B * shape.D * shape.k, "[B, D, k]", V=V)
    _need_gpu(V, packed)
    rc = load_library().svdcache_pack_basis(C.byref(shape), _ptr(V), _ptr(packed),
                                            packed.numel() * packed.element_size(), _stream())
    _check(rc, "svdcache_pack_basis")


def svdcache_full_step(shape: Shape, F, V, packed, R, S, Cout, alpha: float, init: bool):
    """C = F V, R = F - C V^T and the update of S.  Cout (or None): the step may form R from it in a second launch, so steps in
    flight on different streams need one each, even where nobody reads it; it must not overlap the other tensors."""
    if _fast_call("full_step", shape, F, V, packed, R, S, Cout, alpha, init):
        return
    _check_step_args(shape, V, packed, {"S": S, "C": Cout}, {"F": F, "R": R})
    _need_gpu(F, V, packed, R, S, Cout)
    rc = load_library().svdcache_full_step(C.byref(shape), _ptr(F), _ptr(V), _ptr(packed), _ptr(R), _ptr(S),
                                           _ptr(Cout), float(alpha), int(bool(init)), _stream())
    _check(rc, "svdcache_full_step")


def svdcache_full_step_residual_ema(shape: Shape, F, V, packed, R_prev, R, S, Cout, alpha: float, alpha_r: float,
                                    init: bool):
    if _fast_call("full_step_residual_ema", shape, F, V, packed, R_prev, R, S, Cout, alpha, alpha_r, init):
        return
    _check_step_args(shape, V, packed, {"S": S, "C": Cout}, {"F": F, "R": R, "R_prev": R_prev})
    _need_gpu(F, V, packed, R_prev, R, S, Cout)
    rc = load_library().svdcache_full_step_residual_ema(C.byref(shape), _ptr(F), _ptr(V), _ptr(packed), _ptr(R_prev),
                                                        _ptr(R), _ptr(S), _ptr(Cout), float(alpha), float(alpha_r),
                                                        int(bool(init)), _stream())
    _check(rc, "svdcache_full_step_residual_ema")


def svdcache_forecast(shape: Shape, S, V, packed, R, Fhat):
    if _fast_call("forecast", shape, S, V, packed, R, Fhat):
        return
    _check_step_args(shape, V, packed, {"S": S}, {"R": R, "Fhat": Fhat})
    _need_gpu(S, V, packed, R, Fhat)
    rc = load_library().svdcache_forecast(C.byref(shape), _ptr(S), _ptr(V), _ptr(packed), _ptr(R), _ptr(Fhat),
                                          _stream())
    _check(rc, "svdcache_forecast")


def svdcache_packed_state_bytes(shape: Shape) -> int:
    return load_library().svdcache_packed_state_bytes(C.byref(shape))


def _check_packed_state(shape: Shape, S_packed):
    need = svdcache_packed_state_bytes(shape)
    if need == 0 or not S_packed.is_contiguous() or S_packed.numel() * S_packed.element_size() < need:
        raise ValueError(f"S_packed: {S_packed.numel() * S_packed.element_size()} bytes, this shape needs {need}")


def svdcache_pack_state(shape: Shape, S, S_packed):
    _dense_f32(shape.B * shape.N * shape.k, "[B, N, k]", S=S)
    _check_packed_state(shape, S_packed)
    _need_gpu(S, S_packed)
    rc = load_library().svdcache_pack_state(C.byref(shape), _ptr(S), _ptr(S_packed),
                                            S_packed.numel() * S_packed.element_size(), _stream())
    _check(rc, "svdcache_pack_state")


def svdcache_full_step_packed(shape: Shape, F, V, packed, R, S, Cout, S_packed, alpha: float, init: bool):
    if _fast_call("full_step_packed", shape, F, V, packed, R, S, Cout, S_packed, alpha, init):
        return
    if packed is None:
        raise ValueError("packed: the packed-state full step needs the packed basis")
    _check_step_args(shape, V, packed, {"S": S, "C": Cout}, {"F": F, "R": R})
    _check_packed_state(shape, S_packed)
    _need_gpu(F, V, packed, R, S, Cout, S_packed)
    rc = load_library().svdcache_full_step_packed(C.byref(shape), _ptr(F), _ptr(V), _ptr(packed), _ptr(R), _ptr(S),
                                                  _ptr(Cout), _ptr(S_packed),
                                                  S_packed.numel() * S_packed.element_size(), float(alpha),
                                                  int(bool(init)), _stream())
    _check(rc, "svdcache_full_step_packed")


def svdcache_forecast_packed(shape: Shape, S_packed, packed, R, Fhat):
    if _fast_call("forecast_packed", shape, S_packed, packed, R, Fhat):
        return
    if packed is None:
        raise ValueError("packed: the packed-state cached step needs the packed basis")
    _like_features(shape, R=R, Fhat=Fhat)
    _check_packed_state(shape, S_packed)
    need = svdcache_packed_basis_bytes(shape)
    if need == 0 or packed.numel() * packed.element_size() < need:
        raise ValueError("packed: too small for this shape")
    _need_gpu(S_packed, packed, R, Fhat)
    rc = load_library().svdcache_forecast_packed(C.byref(shape), _ptr(S_packed), _ptr(packed), _ptr(R), _ptr(Fhat),
                                                 _stream())
    _check(rc, "svdcache_forecast_packed")


def svdcache_select_rank(sigma, fro2, tau: float, k_star, reached=None):
    """k_star [B] int32 (and reached [B] int32, optional) from sigma [B,k] float32 and fro2 [B] float32."""
    _need_gpu(sigma, fro2, k_star, reached)
    B, k = sigma.shape
    rc = load_library().svdcache_select_rank(B, k, _ptr(sigma), _ptr(fro2), float(tau), _ptr(k_star), _ptr(reached),
                                             _stream())
    _check(rc, "svdcache_select_rank")


def svdcache_truncate_basis(shape: Shape, V, sigma, k_star):
    _need_gpu(V, sigma, k_star)
    rc = load_library().svdcache_truncate_basis(C.byref(shape), _ptr(V), _ptr(sigma), _ptr(k_star), _stream())
    _check(rc, "svdcache_truncate_basis")


def svdcache_extrapolation_weights(order: int, offset: float, interval: float):
    """Host-side: the order+1 weights as a list of Python floats (float32 values)."""
    w = (C.c_float * (order + 1 if order >= 0 else 1))()
    rc = load_library().svdcache_extrapolation_weights(int(order), float(offset), float(interval), w)
    _check(rc, "svdcache_extrapolation_weights")
    return [float(x) for x in w]


def svdcache_forecast_combine(shape: Shape, S_list, weights, V, packed, R, X, Out):
    if _fast_call("forecast_combine", shape, S_list, weights, V, packed, R, X, Out):
        return
    m = len(S_list)
    if m != len(weights):
        raise ValueError("one weight per state")
    _check_step_args(shape, V, packed, {f"S_list[{i}]": t for i, t in enumerate(S_list)}, {"R": R, "X": X, "Out": Out})
    _need_gpu(*S_list, V, packed, R, X, Out)
    ptrs = (C.c_void_p * max(m, 1))(*[t.data_ptr() for t in S_list])
    w = (C.c_float * max(m, 1))(*[float(x) for x in weights])
    rc = load_library().svdcache_forecast_combine(C.byref(shape), m, ptrs, w, _ptr(V), _ptr(packed), _ptr(R),
                                                  _ptr(X), _ptr(Out), _stream())
    _check(rc, "svdcache_forecast_combine")


def svdcache_basis_overlap(shape: Shape, V_old, V_new, M):
    _need_gpu(V_old, V_new, M)
    rc = load_library().svdcache_basis_overlap(C.byref(shape), _ptr(V_old), _ptr(V_new), _ptr(M), _stream())
    _check(rc, "svdcache_basis_overlap")


def svdcache_rebase_state(shape: Shape, M, S_in, S_out):
    _need_gpu(M, S_in, S_out)
    rc = load_library().svdcache_rebase_state(C.byref(shape), _ptr(M), _ptr(S_in), _ptr(S_out), _stream())
    _check(rc, "svdcache_rebase_state")


def svdcache_basis_similarity(shape: Shape, V_a, sigma_a, V_b, sigma_b, sim_dir, sim_sigma):
    _need_gpu(V_a, sigma_a, V_b, sigma_b, sim_dir, sim_sigma)
    rc = load_library().svdcache_basis_similarity(C.byref(shape), _ptr(V_a), _ptr(sigma_a), _ptr(V_b), _ptr(sigma_b),
                                                  _ptr(sim_dir), _ptr(sim_sigma), _stream())
    _check(rc, "svdcache_basis_similarity")


# ---- operators of a block in 8 bits -------------------------------------------------------------

SVDC_E4M3 = 2
SVDC_ACT_NONE, SVDC_ACT_GELU, SVDC_ACT_SWIGLU = 0, 1, 2
_ACTS = {"none": SVDC_ACT_NONE, "gelu": SVDC_ACT_GELU, "swiglu": SVDC_ACT_SWIGLU}
_TORCH_OF_8 = {SVDC_F32: torch.float32, SVDC_BF16: torch.bfloat16, SVDC_E4M3: torch.float8_e4m3fn}
_DTYPES_8 = {v: k for k, v in _TORCH_OF_8.items()}


def _row_stride(name: str, t: torch.Tensor):
    """(rows, D, row stride) of a tensor [..., D] whose rows lie at one stride."""
    if t.dim() < 1 or t.shape[-1] < 1 or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name}: need [..., D] with a contiguous last dimension, got {tuple(t.shape)} with strides {t.stride()}")
    D, rows, ld = t.shape[-1], t.numel() // t.shape[-1], None
    step = None                                        # what the next dimension outwards has to have as its stride
    for n, st in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if n == 1:
            continue
        if step is None:
            ld, step = st, st * n
        elif st != step:
            raise ValueError(f"{name}: rows of {tuple(t.shape)} with strides {t.stride()} do not lie at one stride")
        else:
            step *= n
    return rows, D, D if ld is None or rows == 0 else ld


def make_norm8(X: torch.Tensor, F: Optional[torch.Tensor] = None, H: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None,
               eps: float = 1e-6) -> Norm8:
    """Descriptor of a norm of X [..., D] (float32 or bfloat16) for tensors laid out like these; F may be of the other type."""
    rows, D, ldx = _row_stride("X", X)
    if X.dtype not in _DTYPES or (F is not None and F.dtype not in _DTYPES):
        raise ValueError("X and F must be float32 or bfloat16")
    p = Norm8(rows, D, _DTYPES[X.dtype], _DTYPES[(X if F is None else F).dtype], eps, ldx, D, D, D)
    for name, field, t in (("F", "ldf", F), ("H", "ldh", H), ("Y", "ldy", Y)):
        if t is not None:
            r, d, ld = _row_stride(name, t)
            if (r, d) != (rows, D):
                raise ValueError(f"{name}: {tuple(t.shape)} is not {rows} rows of {D} columns")
            setattr(p, field, ld)
    return p


def make_quant8(X: torch.Tensor, block_rows: int = 1) -> Quant8:
    """Descriptor of the quantisation of X [..., D] with a scale per block_rows (1 or 128) rows and 128 columns."""
    rows, D, ldx = _row_stride("X", X)
    if X.dtype not in _DTYPES:
        raise ValueError("X must be float32 or bfloat16")
    return Quant8(rows, D, _DTYPES[X.dtype], ldx, block_rows, 0)


def make_matmul8(M: int, N: int, K: int, dtype: torch.dtype = torch.bfloat16, act: str = "none", ldo: int = 0) -> Matmul8:
    """Descriptor of Out [M, N] = act(A [M, K] W^T + bias) with Out of `dtype` (float32, bfloat16 or float8_e4m3fn) and row stride
    ldo (0: N).  act: "none", "gelu" or "swiglu" (W then holds 2 N rows)."""
    if dtype not in _DTYPES_8 or act not in _ACTS:
        raise ValueError("dtype is one of float32, bfloat16 and float8_e4m3fn, act one of " + ", ".join(_ACTS))
    return Matmul8(M, N, K, _DTYPES_8[dtype], _ACTS[act], ldo or N)


def svdcache_q8_bytes(rows: int, D: int) -> int:
    return load_library().svdcache_q8_bytes(rows, D)


def svdcache_q8_scale_bytes(rows: int, D: int, block_rows: int = 1) -> int:
    return load_library().svdcache_q8_scale_bytes(rows, D, block_rows)


def svdcache_matmul8_workspace_bytes(p: Matmul8) -> int:
    return load_library().svdcache_matmul8_workspace_bytes(C.byref(p))


_BYTES = (torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.uint8)


def _bytes_of(name: str, t, need: int):
    """Q and scales are dense tensors of one byte an element, of exactly the size that the sizes imply."""
    if t.dtype not in _BYTES or not t.is_contiguous() or t.numel() != need:
        raise ValueError(f"{name}: need a contiguous tensor of {need} bytes, got {t.dtype} {tuple(t.shape)} contiguous={t.is_contiguous()}")


def _check_q8(name: str, Q, scales, rows: int, D: int, block_rows: int = 1):
    _bytes_of(name, Q, svdcache_q8_bytes(rows, D))
    _bytes_of(name + " scales", scales, svdcache_q8_scale_bytes(rows, D, block_rows))


def _rows_like(name: str, t, rows: int, D: int, ld: int, dtype: int):
    """The C ABI describes each tensor by (rows, D, row stride, dtype): refuse one that is laid out otherwise."""
    if t.dtype != _TORCH_OF[dtype]:
        raise ValueError(f"{name}: dtype {t.dtype} is not {_TORCH_OF[dtype]}")
    r, d, have = _row_stride(name, t)
    if (r, d) != (rows, D) or (r > 1 and have != ld):
        raise ValueError(f"{name}: {tuple(t.shape)} with row stride {have} is not {rows} rows of {D} columns with row stride {ld}")


def svdcache_rms_norm8(p: Norm8, X, F, gain, H, Y, Q, scales):
    """H = X + F and its norm: Y plain, (Q, scales) in 8 bits.  F, gain, H, Y and (Q, scales) may be None."""
    if _fast_call("rms_norm8", p, X, F, gain, H, Y, Q, scales):
        return
    for name, t, ld, dtype in (("X", X, p.ldx, p.dtype), ("F", F, p.ldf, p.dtype_f), ("H", H, p.ldh, p.dtype), ("Y", Y, p.ldy, p.dtype)):
        if t is not None:
            _rows_like(name, t, p.rows, p.D, ld, dtype)
    _dense_f32(p.D, "[D]", gain=gain)
    if (Q is None) != (scales is None):
        raise ValueError("Q and scales go together")
    if Q is not None:
        _check_q8("Q", Q, scales, p.rows, p.D)
    _need_gpu(X, F, gain, H, Y, Q, scales)
    rc = load_library().svdcache_rms_norm8(C.byref(p), _ptr(X), _ptr(F), _ptr(gain), _ptr(H), _ptr(Y), _ptr(Q), _ptr(scales), _stream())
    _check(rc, "svdcache_rms_norm8")


def svdcache_quantize8(p: Quant8, X, Q, scales):
    if _fast_call("quantize8", p, X, Q, scales):
        return
    _rows_like("X", X, p.rows, p.D, p.ldx, p.dtype)
    _check_q8("Q", Q, scales, p.rows, p.D, p.block_rows)
    _need_gpu(X, Q, scales)
    rc = load_library().svdcache_quantize8(C.byref(p), _ptr(X), _ptr(Q), _ptr(scales), _stream())
    _check(rc, "svdcache_quantize8")


def svdcache_matmul8(p: Matmul8, A, A_scales, W, W_scales, bias, Out, Out_scales=None, workspace=None):
    """Out = act(A W^T + bias).  workspace: alloc_matmul8_workspace(p), one for each call in flight on a stream of its own."""
    if _fast_call("matmul8", p, A, A_scales, W, W_scales, bias, Out, Out_scales, workspace):
        return
    wide = 2 * p.N if p.act == SVDC_ACT_SWIGLU else p.N
    _check_q8("A", A, A_scales, p.M, p.K)
    _bytes_of("W", W, wide * ((p.K + 127) // 128 * 128))
    _bytes_of("W scales", W_scales, svdcache_q8_scale_bytes(wide, p.K, 128))
    _dense_f32(wide, "[rows of W]", bias=bias)
    if p.dtype == SVDC_E4M3:
        if Out_scales is None:
            raise ValueError("Out_scales: a result in 8 bits has scales")
        _check_q8("Out", Out, Out_scales, p.M, p.N)
    else:
        _rows_like("Out", Out, p.M, p.N, p.ldo, p.dtype)
    _need_gpu(A, A_scales, W, W_scales, bias, Out, Out_scales, workspace)
    rc = load_library().svdcache_matmul8(C.byref(p), _ptr(A), _ptr(A_scales), _ptr(W), _ptr(W_scales), _ptr(bias), _ptr(Out), _ptr(Out_scales),
                                         _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(), _stream())
    _check(rc, "svdcache_matmul8")


# ---- operators around a block's attention -------------------------------------------------------

SVDC_PAIRS_NEIGHBOURS, SVDC_PAIRS_HALVES = 0, 1
_PAIRS = {"neighbours": SVDC_PAIRS_NEIGHBOURS, "halves": SVDC_PAIRS_HALVES}


def _on_current_device(*ts):
    _need_gpu(*ts)
    for t in ts:
        if t is not None and t.device.index != torch.cuda.current_device():
            raise RuntimeError(f"svdcache: a tensor is on {t.device}, the call goes to the current device cuda:{torch.cuda.current_device()}")


def _heads_of(name: str, t: torch.Tensor):
    """(batch, rows, heads, head_dim, strides) of a tensor [batch, rows, heads, head_dim] or [rows, heads, head_dim]; strides of dimensions
    that are not walked count as 0."""
    if t.dim() not in (3, 4) or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name}: need [batch, rows, heads, head_dim] or [rows, heads, head_dim] with a contiguous last dimension, got {tuple(t.shape)} "
                         f"with strides {t.stride()}")
    shape = (1, *t.shape) if t.dim() == 3 else tuple(t.shape)
    strides = (0, *t.stride()) if t.dim() == 3 else t.stride()
    return (*shape, Heads(*(st if n > 1 else 0 for n, st in zip(shape[:3], strides))))


def _check_heads(name: str, t, batch: int, rows: int, heads: int, head_dim: int, strides: Heads, dtype: int, out: bool = False):
    """Refuses a tensor that is laid out otherwise than the descriptor says, and an output whose elements share memory."""
    if t.dtype != _TORCH_OF[dtype]:
        raise ValueError(f"{name}: dtype {t.dtype} is not {_TORCH_OF[dtype]}")
    *shape, have = _heads_of(name, t)
    if shape != [batch, rows, heads, head_dim]:
        raise ValueError(f"{name}: {tuple(t.shape)} is not {batch} x {rows} rows of {heads} heads of {head_dim} columns")
    for n, field in zip(shape, ("seq", "row", "head")):
        if n > 1 and getattr(have, field) != getattr(strides, field):
            raise ValueError(f"{name}: strides {t.stride()} are not those of the descriptor ({strides.seq}, {strides.row}, {strides.head})")
    if out:
        reach = head_dim
        for st, n in sorted((getattr(have, field), n) for n, field in zip(shape, ("seq", "row", "head")) if n > 1):
            if st < reach:
                raise ValueError(f"{name}: elements of {tuple(t.shape)} with strides {t.stride()} share memory")
            reach += (n - 1) * st


def make_rotary(positions: torch.Tensor, dims, theta=10000.0) -> Rotary:
    """Descriptor of the angles of positions [..., axes] (float32 or int32) with dims[a] columns of a head turned by axis a; theta: one number or
    one for each axis."""
    dims = [int(n) for n in dims]
    theta = [float(x) for x in theta] if isinstance(theta, (list, tuple)) else [float(theta)] * len(dims)
    if positions.dtype not in (torch.float32, torch.int32):
        raise ValueError("positions must be float32 or int32")
    rows, axes, ld = _row_stride("positions", positions)
    if len(dims) != axes or len(theta) != axes or not 1 <= axes <= SVDC_MAX_AXES:
        raise ValueError(f"positions with {axes} axes need as many dims and thetas, at most {SVDC_MAX_AXES}; got {len(dims)} and {len(theta)}")
    return Rotary(rows, ld, axes, int(positions.dtype == torch.int32), (C.c_int32 * SVDC_MAX_AXES)(*dims), (C.c_double * SVDC_MAX_AXES)(*theta))


def make_norm_rotate(Q=None, K=None, V=None, Qo=None, Ko=None, Vo=None, table=None, layout: str = "neighbours", norm: bool = True,
                     eps: float = 1e-6) -> NormRotate:
    """Descriptor of norm and rotation for tensors [batch, rows, heads, head_dim] (or without batch) laid out like these; V is copied.  table
    [rows, pairs, 2], or [batch, rows, pairs, 2] with one for each sequence; None: nothing is turned."""
    if layout not in _PAIRS:
        raise ValueError("layout is one of " + ", ".join(_PAIRS))
    first, first_out = next(((x, y) for x, y in ((Q, Qo), (K, Ko), (V, Vo)) if x is not None), (None, None))
    if first is None or any((x is None) != (y is None) for x, y in ((Q, Qo), (K, Ko), (V, Vo))):
        raise ValueError("need at least one of Q, K, V, and each with its output")
    if first.dtype not in _DTYPES or first_out.dtype not in _DTYPES:
        raise ValueError("inputs and outputs must be float32 or bfloat16")
    batch, rows, _, d, _ = _heads_of("Q, K or V", first)
    p = NormRotate(batch, rows, 1, 1, d, _DTYPES[first.dtype], _DTYPES[first_out.dtype], int(norm), 0, _PAIRS[layout], eps, 0, 0)
    for field, heads, t in (("q", "heads", Q), ("k", "kv_heads", K), ("v", "kv_heads", V)):
        if t is not None:
            shape = _heads_of(field.upper(), t)
            setattr(p, heads, shape[2])
            setattr(p, field, shape[4])
    for field, t in (("qo", Qo), ("ko", Ko), ("vo", Vo)):
        if t is not None:
            setattr(p, field, _heads_of(field.capitalize(), t)[4])
    if table is not None:
        if table.dim() not in (3, 4) or table.shape[-1] != 2:
            raise ValueError(f"table: need [rows, pairs, 2] or [batch, rows, pairs, 2], got {tuple(table.shape)}")
        p.pairs = table.shape[-2]
        p.table_seq = rows * p.pairs if table.dim() == 4 else 0
    return p


def make_attention(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, Out: torch.Tensor, q_span=None, k_span=None, scale: Optional[float] = None,
                   q_most: Optional[int] = None, k_most: Optional[int] = None) -> Attention:
    """Descriptor of an attention for tensors laid out like these: [batch, rows, heads, head_dim] (or without batch).  Where a span [batch, 2] is
    given, Q and Out (or K and V) are [all rows, heads, head_dim] and q_most (k_most) rows the most that a sequence has; by default all.
    scale: 1 / sqrt(head_dim) by default."""
    if Q.dtype not in _DTYPES:
        raise ValueError("Q, K, V and Out must be float32 or bfloat16")
    nq, rq, heads, d, sq = _heads_of("Q", Q)
    nk, rk, kv_heads, _, sk = _heads_of("K", K)
    for name, span, n in (("q_span", q_span, nq), ("k_span", k_span, nk)):
        if span is not None and n != 1:
            raise ValueError(f"{name}: tensors with spans are [all rows, heads, head_dim]")
    batch = q_span.shape[0] if q_span is not None else k_span.shape[0] if k_span is not None else nq
    return Attention(batch, rq if q_span is None or q_most is None else q_most, rk if k_span is None or k_most is None else k_most, rq, rk, heads, kv_heads, d,
                     _DTYPES[Q.dtype], d ** -0.5 if scale is None else scale, 0, sq, sk, _heads_of("V", V)[4], _heads_of("Out", Out)[4])


def svdcache_rotary_table(p: Rotary, positions, table):
    """table[row][pair] = (cos, sin) of the pair's angle at the row's positions."""
    if _fast_call("rotary_table", p, positions, table):
        return
    want = torch.int32 if p.whole else torch.float32
    if positions.dtype != want:
        raise ValueError(f"positions: dtype {positions.dtype} is not {want}")
    rows, axes, ld = _row_stride("positions", positions)
    if (rows, axes) != (p.rows, p.axes) or (rows > 1 and ld != p.ld):
        raise ValueError(f"positions: {tuple(positions.shape)} with row stride {ld} is not {p.rows} rows of {p.axes} axes with row stride {p.ld}")
    _dense_f32(p.rows * sum(p.dims[:p.axes]), "[rows, pairs, 2]", table=table)
    _on_current_device(positions, table)
    _check(load_library().svdcache_rotary_table(C.byref(p), _ptr(positions), _ptr(table), _stream()), "svdcache_rotary_table")


def svdcache_norm_rotate(p: NormRotate, Q, K, V, gain_q, gain_k, table, Qo, Ko, Vo):
    """Norm and rotation of the heads of Q and K; V is copied.  Outputs may be their inputs."""
    if _fast_call("norm_rotate", p, Q, K, V, gain_q, gain_k, table, Qo, Ko, Vo):
        return
    for name, t, o, heads, s, so in (("Q", Q, Qo, p.heads, p.q, p.qo), ("K", K, Ko, p.kv_heads, p.k, p.ko), ("V", V, Vo, p.kv_heads, p.v, p.vo)):
        if (t is None) != (o is None):
            raise ValueError(f"{name} and {name}o go together")
        if t is not None:
            _check_heads(name, t, p.batch, p.rows, heads, p.head_dim, s, p.dtype)
            _check_heads(name + "o", o, p.batch, p.rows, heads, p.head_dim, so, p.dtype_out, out=True)
    _dense_f32(p.head_dim, "[head_dim]", gain_q=gain_q, gain_k=gain_k)
    if p.pairs and (Q is not None or K is not None):
        if table is None:
            raise ValueError("table: the descriptor's pairs need one")
        if p.table_seq not in (0, p.rows * p.pairs):
            raise ValueError("table: tables of sequences lie one behind the other")
        _dense_f32(p.rows * p.pairs * 2 * (p.batch if p.table_seq else 1), "[rows, pairs, 2]", table=table)
    _on_current_device(Q, K, V, gain_q, gain_k, table, Qo, Ko, Vo)
    rc = load_library().svdcache_norm_rotate(C.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(gain_q), _ptr(gain_k), _ptr(table), _ptr(Qo), _ptr(Ko), _ptr(Vo),
                                             _stream())
    _check(rc, "svdcache_norm_rotate")


def svdcache_attention_workspace_bytes(p: Attention) -> int:
    return load_library().svdcache_attention_workspace_bytes(C.byref(p))


def svdcache_attention(p: Attention, Q, K, V, Out, q_span=None, k_span=None, key_mask=None, workspace=None):
    """Out = softmax(scale Q K^T) V.  key_mask: a byte or truth value for each key, 0 leaves it out.  workspace: alloc_attention_workspace(p), one
    for each call in flight on a stream of its own."""
    if _fast_call("attention", p, Q, K, V, Out, q_span, k_span, key_mask, workspace):
        return
    q_shape = (p.batch, p.q_rows) if q_span is None else (1, p.q_total)
    k_shape = (p.batch, p.k_rows) if k_span is None else (1, p.k_total)
    _check_heads("Q", Q, *q_shape, p.heads, p.head_dim, p.q, p.dtype)
    _check_heads("K", K, *k_shape, p.kv_heads, p.head_dim, p.k, p.dtype)
    _check_heads("V", V, *k_shape, p.kv_heads, p.head_dim, p.v, p.dtype)
    _check_heads("Out", Out, *q_shape, p.heads, p.head_dim, p.o, p.dtype, out=True)
    for name, t in (("q_span", q_span), ("k_span", k_span)):
        if t is not None and (t.dtype != torch.int32 or tuple(t.shape) != (p.batch, 2) or not t.is_contiguous()):
            raise ValueError(f"{name}: need a contiguous int32 tensor [{p.batch}, 2], got {t.dtype} {tuple(t.shape)}")
    if key_mask is not None:
        need = p.batch * p.k_rows if k_span is None else p.k_total
        if key_mask.dtype not in (torch.uint8, torch.bool) or not key_mask.is_contiguous() or key_mask.numel() != need:
            raise ValueError(f"key_mask: need {need} contiguous uint8 or bool, got {key_mask.dtype} {tuple(key_mask.shape)}")
    _on_current_device(Q, K, V, Out, q_span, k_span, key_mask, workspace)
    rc = load_library().svdcache_attention(C.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(q_span), _ptr(k_span), _ptr(key_mask), _ptr(Out), _ptr(workspace),
                                           0 if workspace is None else workspace.numel() * workspace.element_size(), _stream())
    _check(rc, "svdcache_attention")


# ---- conveniences that only allocate (torch owns the memory) ------------------------------------

def fit_basis(F: torch.Tensor, k: int, p: int = 0, q: int = 0, seed: int = 0, max_sweeps: int = 0,
              return_status: bool = False):
    """Allocate outputs + workspace and call svdcache_fit_basis. Returns (V [B,D,k], sigma [B,k], fro2 [B]) and,
    with return_status, the per-block status words [B] int32 (SVDC_FIT_* flags) copied out of the workspace."""
    shape = make_shape(F, k)
    dev = F.device
    V = torch.empty(shape.B, shape.D, k, device=dev, dtype=torch.float32)
    sigma = torch.empty(shape.B, k, device=dev, dtype=torch.float32)
    fro2 = torch.empty(shape.B, device=dev, dtype=torch.float32)
    nbytes = svdcache_workspace_bytes(shape, p, q, seed, max_sweeps)
    if nbytes == 0:
        raise SvdcError(-2, "svdcache_workspace_bytes")
    ws = torch.empty(nbytes, device=dev, dtype=torch.uint8)
    svdcache_fit_basis(shape, F, V, sigma, fro2, ws, p, q, seed, max_sweeps)
    if not return_status:
        return V, sigma, fro2
    off = svdcache_fit_status_offset(shape, p, q, seed, max_sweeps)
    status = ws[off:off + 4 * shape.B].view(torch.int32).clone()
    return V, sigma, fro2, status


def fit_basis_for_energy(F: torch.Tensor, tau: float = 0.85, k_init: int = 32, k_max: int = 128, p: int = 0,
                         q: int = 0, seed: int = 0):
    """Rank chosen by the energy rule (Eq. 6): fit with k_init, let the device pick k*_b per block, and fit
    again with twice the rank (up to k_max) while some block has not reached tau within the fitted values
    (the sketch must be at least as wide as the rank it is asked about).  The loop and its one device-to-host
    read per pass are host policy; every arithmetic step is a library call.
    Returns (V [B,D,k] with the columns >= k*_b zeroed, sigma [B,k] likewise, fro2 [B], k_star [B] int32,
    reached [B] int32) where k is the rank of the last fit."""
    if F.dim() == 2:
        F = F.unsqueeze(0)
    B, N, D = F.shape
    k = max(1, min(k_init, N, D))
    while True:
        V, sigma, fro2 = fit_basis(F, k, p, q, seed)
        k_star = torch.empty(B, dtype=torch.int32, device=F.device)
        reached = torch.empty(B, dtype=torch.int32, device=F.device)
        svdcache_select_rank(sigma, fro2, tau, k_star, reached)
        k_next = min(2 * k, k_max, N, D)
        if bool(reached.all()) or k_next <= k:
            break
        k = k_next
    svdcache_truncate_basis(make_shape(F, k), V, sigma, k_star)
    return V, sigma, fro2, k_star, reached


def save_basis(path: str, V: torch.Tensor, sigma: torch.Tensor, fro2: Optional[torch.Tensor] = None):
    """Write a fitted basis to a file (numpy .npz, plain arrays only): the one-time SVD of a model is done
    offline on a reference prompt and its V and sigma are reused for every later prompt (Sec. 3.3)."""
    import numpy as np
    arrays = {"V": V.detach().float().cpu().numpy(), "sigma": sigma.detach().float().cpu().numpy()}
    if fro2 is not None:
        arrays["fro2"] = fro2.detach().float().cpu().numpy()
    with open(path, "wb") as f:
        np.savez(f, **arrays)


def load_basis(path: str, device="cuda:0"):
    """(V [B,D,k], sigma [B,k], fro2 [B] or None) from a file written by save_basis, as float32 tensors on
    `device`.  Nothing in the file is executed (no pickled objects are accepted)."""
    import numpy as np
    with np.load(path, allow_pickle=False) as z:
        V = torch.from_numpy(z["V"]).to(device).contiguous()
        sigma = torch.from_numpy(z["sigma"]).to(device).contiguous()
        fro2 = torch.from_numpy(z["fro2"]).to(device).contiguous() if "fro2" in z.files else None
    if V.dim() != 3 or sigma.shape != (V.shape[0], V.shape[2]):
        raise ValueError("not a basis file: V must be [B, D, k] and sigma [B, k]")
    return V, sigma, fro2


def alloc_packed_state(shape: Shape, device):
    """Buffer for the packed coefficient state, or None when the shape has no matrix-core path."""
    n = svdcache_packed_state_bytes(shape)
    return torch.empty(n, device=device, dtype=torch.uint8) if n else None


def pack_basis(shape: Shape, V: torch.Tensor):
    """Packed copy of V for the matrix-core kernels, or None when the shape has no such path."""
    n = svdcache_packed_basis_bytes(shape)
    if n == 0:
        return None
    packed = torch.empty(n, device=V.device, dtype=torch.uint8)
    svdcache_pack_basis(shape, V, packed)
    return packed


def alloc_q8(rows: int, D: int, device, block_rows: int = 1):
    """(Q, scales) for a matrix [rows, D] in 8 bits: float8_e4m3fn [rows, D rounded up to 128], float8_e8m0fnu [rows / block_rows, ...]."""
    nq, ns = svdcache_q8_bytes(rows, D), svdcache_q8_scale_bytes(rows, D, block_rows)
    if rows < 0 or (rows and not (nq and ns)):
        raise SvdcError(-2, "svdcache_q8_bytes")
    tall = (rows + block_rows - 1) // block_rows
    Q = torch.empty(nq, device=device, dtype=torch.uint8).view(torch.float8_e4m3fn)
    scales = torch.empty(ns, device=device, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    wide = (D + 127) // 128
    return Q.view(rows, wide * 128), scales.view(tall, (wide + 3) // 4 * 4)


def alloc_matmul8_workspace(p: Matmul8, device):
    """Workspace of svdcache_matmul8 for this product, or None where it needs none."""
    n = svdcache_matmul8_workspace_bytes(p)
    return torch.empty(n, device=device, dtype=torch.uint8) if n else None


def rms_norm8(X: torch.Tensor, F: Optional[torch.Tensor] = None, gain: Optional[torch.Tensor] = None, eps: float = 1e-6):
    """(H, Q, scales): H = X + F and its norm in 8 bits, in new tensors."""
    H = torch.empty(X.shape, device=X.device, dtype=X.dtype)
    p = make_norm8(X, F, H, None, eps)
    Q, scales = alloc_q8(p.rows, p.D, X.device)
    svdcache_rms_norm8(p, X, F, gain, H, None, Q, scales)
    return H, Q, scales


def quantize8(X: torch.Tensor, block_rows: int = 1):
    """(Q, scales) of X [..., D] in new tensors; block_rows 1 for activations, 128 for weights."""
    p = make_quant8(X, block_rows)
    Q, scales = alloc_q8(p.rows, p.D, X.device, block_rows)
    svdcache_quantize8(p, X, Q, scales)
    return Q, scales


def matmul8(A, A_scales, W, W_scales, K: int, bias: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16, act: str = "none"):
    """act(A W^T + bias) in a new tensor [rows of A, N]; (Out, Out_scales) for dtype float8_e4m3fn.  A and W as alloc_q8 shapes them."""
    N = W.shape[0] // 2 if act == "swiglu" else W.shape[0]
    p = make_matmul8(A.shape[0], N, K, dtype, act)
    if dtype == torch.float8_e4m3fn:
        Out, Out_scales = alloc_q8(p.M, p.N, A.device)
    else:
        Out, Out_scales = torch.empty(p.M, p.N, device=A.device, dtype=dtype), None
    svdcache_matmul8(p, A, A_scales, W, W_scales, bias, Out, Out_scales, alloc_matmul8_workspace(p, A.device))
    return Out if Out_scales is None else (Out, Out_scales)


def rotary_table(positions: torch.Tensor, dims, theta=10000.0):
    """(cos, sin) of the angles at positions [..., axes] in a new tensor [rows, pairs, 2]."""
    p = make_rotary(positions, dims, theta)
    table = torch.empty(p.rows, sum(p.dims[:p.axes]) // 2, 2, device=positions.device)
    svdcache_rotary_table(p, positions, table)
    return table


def norm_rotate(Q=None, K=None, V=None, gain_q=None, gain_k=None, table=None, layout: str = "neighbours", norm: bool = True, eps: float = 1e-6,
                dtype: Optional[torch.dtype] = None):
    """(Qo, Ko, Vo) in new tensors of `dtype` (the inputs' by default), None for what is not given."""
    out = [None if t is None else torch.empty(t.shape, device=t.device, dtype=dtype or t.dtype) for t in (Q, K, V)]
    svdcache_norm_rotate(make_norm_rotate(Q, K, V, *out, table, layout, norm, eps), Q, K, V, gain_q, gain_k, table, *out)
    return tuple(out)


def alloc_attention_workspace(p: Attention, device):
    """Workspace of svdcache_attention for this attention, or None where it needs none."""
    n = svdcache_attention_workspace_bytes(p)
    return torch.empty(n, device=device, dtype=torch.uint8) if n else None


def attention(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, scale: Optional[float] = None, q_span=None, k_span=None, key_mask=None,
              q_most: Optional[int] = None, k_most: Optional[int] = None):
    """softmax(scale Q K^T) V in a new tensor of Q's shape; rows that no span has are zeros."""
    Out = (torch.empty if q_span is None else torch.zeros)(Q.shape, device=Q.device, dtype=Q.dtype)
    p = make_attention(Q, K, V, Out, q_span, k_span, scale, q_most, k_most)
    svdcache_attention(p, Q, K, V, Out, q_span, k_span, key_mask, alloc_attention_workspace(p, Q.device))
    return Out
