"""Thin binding over libprobsparse.so (the C ABI in include/probsparse.h).

Argument marshalling only: every step of the forward runs in the library's HIP
kernels.  PyTorch is used for device memory and streams.  The hot entry points
go through the extension module _native (csrc/python), which does the same
marshalling in native code and hands back what it cannot take (None) before anything
is enqueued; the ctypes functions below it serve everything else.  The module is for
speed alone (a short call's time in the interpreter): where it has not been built, or was
built for another torch, every call goes through ctypes.  There is no CPU fallback: if the
library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import os
import warnings
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libprobsparse.so")
NATIVE_PATH = os.path.join(_HERE, "_native.so")

PSA_F32, PSA_BF16 = 0, 1
STAGE_MEASURE, STAGE_SELECT, STAGE_ATTEND, STAGE_ALL = 1, 2, 4, 7
U_LOG, U_RATIO = 0, 1
FILL_MEAN, FILL_VALUE = 0, 1
ROTARY_HALF, ROTARY_INTERLEAVED = 0, 1
ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_BASE, ROTARY_PARTS = 0, 1, 2, 3

EXPORTS = [
    "probsparse_attn_workspace_bytes", "probsparse_attn_fwd", "probsparse_attn_fwd_debug",
    "probsparse_attn_fwd_stages", "probsparse_u_max", "dense_attn_workspace_bytes", "dense_attn_fwd",
    "probsparse_attn_workspace_bytes_opt", "probsparse_u_max_opt", "probsparse_attn_fwd_opt",
    "probsparse_attn_with_indices_workspace_bytes", "probsparse_attn_fwd_with_indices",
    "probsparse_exact_measure", "probsparse_qkv_project", "probsparse_out_project",
    "probsparse_mhsa_workspace_bytes", "probsparse_mhsa_fwd",
    "probsparse_describe_plan", "probsparse_init", "probsparse_strerror", "probsparse_version",
    "probsparse_static_workspace_bytes", "probsparse_attn_fwd_static",
    "probsparse_attn_bwd_workspace_bytes", "probsparse_attn_bwd",
    "probsparse_layer_norm_fwd", "probsparse_layer_norm_bwd_workspace_bytes", "probsparse_layer_norm_bwd",
    "probsparse_rotary_frequencies", "probsparse_rotary_fwd", "probsparse_rotary_bwd",
    "dense_attn_packed_workspace_bytes", "dense_attn_packed_fwd",
    "dense_attn_packed_bwd_workspace_bytes", "dense_attn_packed_bwd",
]


class PsaShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("L_Q", ctypes.c_int32), ("L_K", ctypes.c_int32),
                ("D", ctypes.c_int32), ("U", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class PsaOptions(ctypes.Structure):
    _fields_ = [("u_rule", ctypes.c_int32), ("fill", ctypes.c_int32), ("factor", ctypes.c_double)]


class PsaMhsaWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("Wq", "Wk", "Wv", "Wo", "bq", "bk", "bv", "bo")]


class PsaHeads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("row_stride", ctypes.c_int64)]


class PsaRotary(ctypes.Structure):
    _fields_ = [("dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("scaling", ctypes.c_int32), ("base", ctypes.c_double),
                ("factor", ctypes.c_double), ("original_length", ctypes.c_double), ("fast_turns", ctypes.c_double),
                ("slow_turns", ctypes.c_double), ("magnitude", ctypes.c_double)]


class PsaPackedShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("H_kv", ctypes.c_int32), ("T_q", ctypes.c_int32),
                ("T_k", ctypes.c_int32), ("D", ctypes.c_int32), ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("scale", ctypes.c_double)]


class ProbSparseError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libprobsparse: {msg} (status {code})")
        self.code = code


class _CtypesOnly:
    """Stands in for the extension module where there is none: leaves every call to the ctypes path."""
    @staticmethod
    def attn_fwd(*args):
        return None
    attn_fwd_opt = attn_fwd_with_indices = attn_bwd = mhsa_fwd = attn_fwd
    layer_norm_fwd = layer_norm_bwd = rotary = packed_fwd = packed_bwd = attn_fwd


_lib = None
_native = None          # the extension module or _CtypesOnly, loaded with the library


def _load_native():
    if not os.path.exists(NATIVE_PATH):
        return _CtypesOnly
    try:
        from . import _native as module
        module.on_status(_check)
    except (ImportError, AttributeError) as e:
        warnings.warn(f"{NATIVE_PATH} cannot be loaded ({e}): calls go through ctypes, which takes some microseconds more "
                      "each; build it again with `python -m paper_2106_09236_amd.build`")
        return _CtypesOnly
    return module


def load() -> ctypes.CDLL:
    """Load the library (once).  Raises FileNotFoundError if it was never built."""
    global _lib, _native
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2106_09236_amd.build` "
            "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32p, f32p = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
    shp = ctypes.POINTER(PsaShape)
    fwd_args = [vp, vp, vp, i32p, i32p, ctypes.c_double, vp, shp, vp, ctypes.c_size_t, vp]
    lib.probsparse_attn_workspace_bytes.restype = ctypes.c_size_t
    lib.probsparse_attn_workspace_bytes.argtypes = [shp, ctypes.c_double]
    lib.probsparse_u_max.restype = ctypes.c_int32
    lib.probsparse_u_max.argtypes = [shp, ctypes.c_double]
    lib.probsparse_attn_fwd.restype = ctypes.c_int
    lib.probsparse_attn_fwd.argtypes = fwd_args
    lib.probsparse_static_workspace_bytes.restype = ctypes.c_size_t
    lib.probsparse_static_workspace_bytes.argtypes = []
    lib.probsparse_attn_fwd_static.restype = ctypes.c_int
    lib.probsparse_attn_fwd_static.argtypes = [vp, vp, vp, i32p, i32p, ctypes.c_double, vp, shp, vp]
    lib.probsparse_attn_fwd_debug.restype = ctypes.c_int
    lib.probsparse_attn_fwd_debug.argtypes = fwd_args + [f32p, i32p, i32p]
    lib.probsparse_attn_fwd_stages.restype = ctypes.c_int
    lib.probsparse_attn_fwd_stages.argtypes = fwd_args + [ctypes.c_int]
    optp = ctypes.POINTER(PsaOptions)
    lib.probsparse_attn_workspace_bytes_opt.restype = ctypes.c_size_t
    lib.probsparse_attn_workspace_bytes_opt.argtypes = [shp, optp]
    lib.probsparse_u_max_opt.restype = ctypes.c_int32
    lib.probsparse_u_max_opt.argtypes = [shp, optp]
    lib.probsparse_attn_fwd_opt.restype = ctypes.c_int
    lib.probsparse_attn_fwd_opt.argtypes = [vp, vp, vp, i32p, i32p, optp, vp, shp, vp, ctypes.c_size_t, vp,
                                            f32p, i32p, i32p]
    lib.probsparse_attn_with_indices_workspace_bytes.restype = ctypes.c_size_t
    lib.probsparse_attn_with_indices_workspace_bytes.argtypes = [shp, ctypes.c_int32]
    lib.probsparse_attn_fwd_with_indices.restype = ctypes.c_int
    lib.probsparse_attn_fwd_with_indices.argtypes = [vp, vp, vp, i32p, i32p, i32p, ctypes.c_int32, ctypes.c_int32,
                                                     vp, shp, vp, ctypes.c_size_t, vp]
    lib.probsparse_attn_bwd_workspace_bytes.restype = ctypes.c_size_t
    lib.probsparse_attn_bwd_workspace_bytes.argtypes = [shp, ctypes.c_int32]
    lib.probsparse_attn_bwd.restype = ctypes.c_int
    lib.probsparse_attn_bwd.argtypes = [vp, vp, vp, i32p, i32p, i32p, ctypes.c_int32, ctypes.c_int32,
                                        vp, vp, vp, vp, shp, vp, ctypes.c_size_t, vp]
    lib.probsparse_exact_measure.restype = ctypes.c_int
    lib.probsparse_exact_measure.argtypes = [vp, vp, i32p, f32p, shp, vp]
    wp = ctypes.POINTER(PsaMhsaWeights)
    lib.probsparse_qkv_project.restype = ctypes.c_int
    lib.probsparse_qkv_project.argtypes = [vp, wp, vp, vp, vp, shp, vp]
    lib.probsparse_out_project.restype = ctypes.c_int
    lib.probsparse_out_project.argtypes = [vp, wp, vp, shp, vp]
    lib.probsparse_mhsa_workspace_bytes.restype = ctypes.c_size_t
    lib.probsparse_mhsa_workspace_bytes.argtypes = [shp, optp]
    lib.probsparse_mhsa_fwd.restype = ctypes.c_int
    lib.probsparse_mhsa_fwd.argtypes = [vp, wp, i32p, i32p, optp, vp, shp, vp, ctypes.c_size_t, vp]
    lib.dense_attn_workspace_bytes.restype = ctypes.c_size_t
    lib.dense_attn_workspace_bytes.argtypes = [shp]
    lib.dense_attn_fwd.restype = ctypes.c_int
    lib.dense_attn_fwd.argtypes = [vp, vp, vp, i32p, vp, shp, vp, ctypes.c_size_t, vp]
    lib.probsparse_strerror.restype = ctypes.c_char_p
    lib.probsparse_strerror.argtypes = [ctypes.c_int]
    lib.probsparse_version.restype = ctypes.c_int
    lib.probsparse_version.argtypes = []
    lib.probsparse_init.restype = ctypes.c_int
    lib.probsparse_init.argtypes = []
    hp, rp, kp = ctypes.POINTER(PsaHeads), ctypes.POINTER(PsaRotary), ctypes.POINTER(PsaPackedShape)
    i32, i64 = ctypes.c_int32, ctypes.c_int64
    lib.probsparse_layer_norm_fwd.restype = ctypes.c_int
    lib.probsparse_layer_norm_fwd.argtypes = [vp, vp, vp, ctypes.c_double, vp, f32p, f32p, i64, i32, i32, vp]
    lib.probsparse_layer_norm_bwd_workspace_bytes.restype = ctypes.c_size_t
    lib.probsparse_layer_norm_bwd_workspace_bytes.argtypes = [i64, i32, i32]
    lib.probsparse_layer_norm_bwd.restype = ctypes.c_int
    lib.probsparse_layer_norm_bwd.argtypes = [vp, vp, vp, f32p, f32p, vp, f32p, f32p, i64, i32, i32, vp, ctypes.c_size_t, vp]
    lib.probsparse_rotary_frequencies.restype = ctypes.c_int
    lib.probsparse_rotary_frequencies.argtypes = [rp, ctypes.POINTER(ctypes.c_double)]
    for f in (lib.probsparse_rotary_fwd, lib.probsparse_rotary_bwd):
        f.restype = ctypes.c_int
        f.argtypes = [hp, hp, i32, rp, i32p, i64, i32, hp, hp, shp, vp]
    for f in (lib.dense_attn_packed_workspace_bytes, lib.dense_attn_packed_bwd_workspace_bytes):
        f.restype = ctypes.c_size_t
        f.argtypes = [kp]
    lib.dense_attn_packed_fwd.restype = ctypes.c_int
    lib.dense_attn_packed_fwd.argtypes = [hp, hp, hp, i32p, i32p, hp, f32p, kp, vp, ctypes.c_size_t, vp]
    lib.dense_attn_packed_bwd.restype = ctypes.c_int
    lib.dense_attn_packed_bwd.argtypes = [hp, hp, hp, i32p, i32p, hp, f32p, hp, hp, hp, hp, kp, vp, ctypes.c_size_t, vp]
    lib.probsparse_describe_plan.restype = ctypes.c_int
    lib.probsparse_describe_plan.argtypes = [shp, optp, ctypes.c_int32, ctypes.c_char_p, ctypes.c_size_t]
    _lib, _native = lib, _load_native()
    return lib


def _fast():
    """The extension module, or what stands in for it."""
    if _native is None:
        load()
    return _native


def strerror(code: int) -> str:
    return load().probsparse_strerror(code).decode()


def _check(code: int):
    if code != 0:
        raise ProbSparseError(code, strerror(code))


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return PSA_F32
    if t.dtype == torch.bfloat16:
        return PSA_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def make_shape(B: int, H: int, L: int, U: int, dtype: int, D: int = 64, L_Q: Optional[int] = None) -> PsaShape:
    return PsaShape(B, H, L if L_Q is None else L_Q, L, D, U, dtype)


def _shape_of(Q: torch.Tensor, sample_idx: Optional[torch.Tensor]) -> PsaShape:
    B, H, L, D = Q.shape
    U = 1 if sample_idx is None else sample_idx.shape[-1]
    return make_shape(B, H, L, U, _dtype_code(Q), D)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_ptr() -> int:
    return torch.cuda.current_stream().cuda_stream


def _require_dev(*ts):
    for t in ts:
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("tensors must be contiguous device tensors")


def workspace_bytes(shape: PsaShape, c: float) -> int:
    return load().probsparse_attn_workspace_bytes(ctypes.byref(shape), c)


def u_max(shape: PsaShape, c: float) -> int:
    return load().probsparse_u_max(ctypes.byref(shape), c)


def alloc_workspace(shape: PsaShape, c: float, device="cuda") -> torch.Tensor:
    n = workspace_bytes(shape, c)
    if n == 0:
        raise ProbSparseError(-2, "invalid shape or c for workspace sizing")
    return torch.empty(n, dtype=torch.uint8, device=device)


def probsparse_attn_fwd(Q, K, V, lengths, sample_idx, c: float, out=None, workspace=None):
    """out = prob-sparse self-attention of (Q, K, V); see include/probsparse.h."""
    done = (_native or _fast()).attn_fwd(Q, K, V, lengths, sample_idx, c, out, workspace)
    if done is not None:
        return done
    _require_dev(Q, K, V, lengths, sample_idx, out, workspace)
    shape = _shape_of(Q, sample_idx)
    if out is None:
        out = torch.empty_like(Q)
    if workspace is None:
        workspace = alloc_workspace(shape, c, Q.device)
    _check(load().probsparse_attn_fwd(_ptr(Q), _ptr(K), _ptr(V), _ptr(lengths), _ptr(sample_idx), c, _ptr(out),
                                      ctypes.byref(shape), _ptr(workspace), workspace.numel(), _stream_ptr()))
    return out


def probsparse_attn_fwd_static(Q, K, V, lengths, sample_idx, c: float, out):
    """The forward on the library's own static scratch: no workspace argument, nothing allocated
    (`out` must be given)."""
    _require_dev(Q, K, V, lengths, sample_idx, out)
    shape = _shape_of(Q, sample_idx)
    _check(load().probsparse_attn_fwd_static(_ptr(Q), _ptr(K), _ptr(V), _ptr(lengths), _ptr(sample_idx), c, _ptr(out),
                                             ctypes.byref(shape), _stream_ptr()))
    return out


def probsparse_attn_fwd_debug(Q, K, V, lengths, sample_idx, c: float, out=None, workspace=None):
    """Returns (out, M [B,H,L] f32, sel [B,H,u_max] i32, u [B] i32)."""
    _require_dev(Q, K, V, lengths, sample_idx, out, workspace)
    shape = _shape_of(Q, sample_idx)
    B, H, L, _ = Q.shape
    if out is None:
        out = torch.empty_like(Q)
    if workspace is None:
        workspace = alloc_workspace(shape, c, Q.device)
    um = u_max(shape, c)
    M = torch.empty((B, H, L), dtype=torch.float32, device=Q.device)
    sel = torch.empty((B, H, um), dtype=torch.int32, device=Q.device)
    u = torch.empty((B,), dtype=torch.int32, device=Q.device)
    _check(load().probsparse_attn_fwd_debug(_ptr(Q), _ptr(K), _ptr(V), _ptr(lengths), _ptr(sample_idx), c, _ptr(out),
                                            ctypes.byref(shape), _ptr(workspace), workspace.numel(), _stream_ptr(),
                                            _ptr(M), _ptr(sel), _ptr(u)))
    return out, M, sel, u


def probsparse_attn_fwd_stages(Q, K, V, lengths, sample_idx, c: float, out, workspace, stage_mask: int):
    _require_dev(Q, K, V, lengths, sample_idx, out, workspace)
    shape = _shape_of(Q, sample_idx)
    _check(load().probsparse_attn_fwd_stages(_ptr(Q), _ptr(K), _ptr(V), _ptr(lengths), _ptr(sample_idx), c, _ptr(out),
                                             ctypes.byref(shape), _ptr(workspace), workspace.numel(), _stream_ptr(),
                                             stage_mask))
    return out


def probsparse_attn_fwd_opt(Q, K, V, lengths, sample_idx, u_rule: int, factor: float, fill: int,
                            out=None, workspace=None, taps: bool = True):
    """The forward with the rule for u (U_LOG: ceil(factor ln n), U_RATIO: ceil(factor n))
    and the fill (FILL_MEAN, FILL_VALUE) selectable.  Returns (out, M, sel, u) with
    taps, else out."""
    if not taps:
        done = (_native or _fast()).attn_fwd_opt(Q, K, V, lengths, sample_idx, u_rule, factor, fill, out, workspace)
        if done is not None:
            return done
    _require_dev(Q, K, V, lengths, sample_idx, out, workspace)
    shape = _shape_of(Q, sample_idx)
    opt = PsaOptions(u_rule, fill, factor)
    B, H, L, _ = Q.shape
    lib = load()
    if out is None:
        out = torch.empty_like(Q)
    if workspace is None:
        n = lib.probsparse_attn_workspace_bytes_opt(ctypes.byref(shape), ctypes.byref(opt))
        if n == 0:
            raise ProbSparseError(-4, "invalid shape or options for workspace sizing")
        workspace = torch.empty(n, dtype=torch.uint8, device=Q.device)
    M = sel = u = None
    if taps:
        um = lib.probsparse_u_max_opt(ctypes.byref(shape), ctypes.byref(opt))
        M = torch.empty((B, H, L), dtype=torch.float32, device=Q.device)
        sel = torch.empty((B, H, um), dtype=torch.int32, device=Q.device)
        u = torch.empty((B,), dtype=torch.int32, device=Q.device)
    _check(lib.probsparse_attn_fwd_opt(_ptr(Q), _ptr(K), _ptr(V), _ptr(lengths), _ptr(sample_idx), ctypes.byref(opt),
                                       _ptr(out), ctypes.byref(shape), _ptr(workspace), workspace.numel(),
                                       _stream_ptr(), _ptr(M), _ptr(sel), _ptr(u)))
    return (out, M, sel, u) if taps else out


def probsparse_attn_fwd_with_indices(Q, K, V, lengths, sel, u, fill: int = FILL_MEAN, out=None, workspace=None):
    """Steps a3 + a4 for given index sets: sel [B, H, u_stride] int32, u [B] int32."""
    done = (_native or _fast()).attn_fwd_with_indices(Q, K, V, lengths, sel, u, fill, out, workspace)
    if done is not None:
        return done
    _require_dev(Q, K, V, lengths, sel, u, out, workspace)
    shape = _shape_of(Q, None)
    u_stride = sel.shape[-1]
    lib = load()
    if out is None:
        out = torch.empty_like(Q)
    if workspace is None:
        n = lib.probsparse_attn_with_indices_workspace_bytes(ctypes.byref(shape), u_stride)
        if n == 0:
            raise ProbSparseError(-4, "invalid shape or u_stride for workspace sizing")
        workspace = torch.empty(n, dtype=torch.uint8, device=Q.device)
    _check(lib.probsparse_attn_fwd_with_indices(_ptr(Q), _ptr(K), _ptr(V), _ptr(lengths), _ptr(sel), _ptr(u),
                                                u_stride, fill, _ptr(out), ctypes.byref(shape), _ptr(workspace),
                                                workspace.numel(), _stream_ptr()))
    return out


def probsparse_attn_bwd(Q, K, V, lengths, sel, u, dOut, fill: int = FILL_MEAN, workspace=None):
    """Gradients (dQ, dK, dV) of steps a3 + a4 for the index sets sel [B, H, u_stride], u [B]."""
    done = (_native or _fast()).attn_bwd(Q, K, V, lengths, sel, u, dOut, fill, workspace)
    if done is not None:
        return done
    _require_dev(Q, K, V, lengths, sel, u, dOut, workspace)
    shape = _shape_of(Q, None)
    u_stride = sel.shape[-1]
    lib = load()
    if workspace is None:
        n = lib.probsparse_attn_bwd_workspace_bytes(ctypes.byref(shape), u_stride)
        if n == 0:
            raise ProbSparseError(-4, "invalid shape or u_stride for workspace sizing")
        workspace = torch.empty(n, dtype=torch.uint8, device=Q.device)
    dQ, dK, dV = torch.empty_like(Q), torch.empty_like(Q), torch.empty_like(Q)
    _check(lib.probsparse_attn_bwd(_ptr(Q), _ptr(K), _ptr(V), _ptr(lengths), _ptr(sel), _ptr(u), u_stride, fill,
                                   _ptr(dOut), _ptr(dQ), _ptr(dK), _ptr(dV), ctypes.byref(shape), _ptr(workspace),
                                   workspace.numel(), _stream_ptr()))
    return dQ, dK, dV


def probsparse_exact_measure(Q, K, lengths, M_out=None):
    """The exact sparsity measure of Eq. 10, [B, H, L] float32 (a diagnostic; dense in the keys)."""
    _require_dev(Q, K, lengths, M_out)
    shape = _shape_of(Q, None)
    B, H, L, _ = Q.shape
    if M_out is None:
        M_out = torch.empty((B, H, L), dtype=torch.float32, device=Q.device)
    _check(load().probsparse_exact_measure(_ptr(Q), _ptr(K), _ptr(lengths), _ptr(M_out), ctypes.byref(shape),
                                           _stream_ptr()))
    return M_out


def make_weights(Wq=None, Wk=None, Wv=None, Wo=None, bq=None, bk=None, bv=None, bo=None) -> PsaMhsaWeights:
    _require_dev(Wq, Wk, Wv, Wo, bq, bk, bv, bo)
    return PsaMhsaWeights(*[_ptr(t) for t in (Wq, Wk, Wv, Wo, bq, bk, bv, bo)])


def _mhsa_shape(X: torch.Tensor, U: int) -> PsaShape:
    B, L, dm = X.shape
    return make_shape(B, dm // 64, L, U, _dtype_code(X))


def probsparse_qkv_project(X, weights: PsaMhsaWeights):
    """X [B, L, H*64] -> Q, K, V [B, H, L, 64] (Sec. 3.1)."""
    _require_dev(X)
    shape = _mhsa_shape(X, 1)
    B, L, _ = X.shape
    Q, K, V = (torch.empty((B, shape.H, L, 64), dtype=X.dtype, device=X.device) for _ in range(3))
    _check(load().probsparse_qkv_project(_ptr(X), ctypes.byref(weights), _ptr(Q), _ptr(K), _ptr(V), ctypes.byref(shape),
                                         _stream_ptr()))
    return Q, K, V


def probsparse_out_project(A, weights: PsaMhsaWeights):
    """A [B, H, L, 64] -> Y [B, L, H*64]."""
    _require_dev(A)
    B, H, L, _ = A.shape
    shape = make_shape(B, H, L, 1, _dtype_code(A))
    Y = torch.empty((B, L, H * 64), dtype=A.dtype, device=A.device)
    _check(load().probsparse_out_project(_ptr(A), ctypes.byref(weights), _ptr(Y), ctypes.byref(shape), _stream_ptr()))
    return Y


def probsparse_mhsa_fwd(X, weights: PsaMhsaWeights, lengths, sample_idx, u_rule: int, factor: float, fill: int,
                        Y=None, workspace=None):
    """The whole module: projections, prob-sparse attention per head, output matrix."""
    done = (_native or _fast()).mhsa_fwd(X, weights, lengths, sample_idx, u_rule, factor, fill, Y, workspace)
    if done is not None:
        return done
    _require_dev(X, lengths, sample_idx, Y, workspace)
    shape = _mhsa_shape(X, sample_idx.shape[-1])
    opt = PsaOptions(u_rule, fill, factor)
    lib = load()
    if Y is None:
        Y = torch.empty_like(X)
    if workspace is None:
        n = lib.probsparse_mhsa_workspace_bytes(ctypes.byref(shape), ctypes.byref(opt))
        if n == 0:
            raise ProbSparseError(-4, "invalid shape or options for workspace sizing")
        workspace = torch.empty(n, dtype=torch.uint8, device=X.device)
    _check(lib.probsparse_mhsa_fwd(_ptr(X), ctypes.byref(weights), _ptr(lengths), _ptr(sample_idx), ctypes.byref(opt),
                                   _ptr(Y), ctypes.byref(shape), _ptr(workspace), workspace.numel(), _stream_ptr()))
    return Y


def dense_workspace_bytes(shape: PsaShape) -> int:
    return load().dense_attn_workspace_bytes(ctypes.byref(shape))


def dense_attn_fwd(Q, K, V, lengths, out=None, workspace=None):
    """Baseline: dense softmax(QK^T/sqrt(d))V over the valid keys."""
    _require_dev(Q, K, V, lengths, out, workspace)
    shape = _shape_of(Q, None)
    if out is None:
        out = torch.empty_like(Q)
    if workspace is None:
        workspace = torch.empty(max(256, dense_workspace_bytes(shape)), dtype=torch.uint8, device=Q.device)
    _check(load().dense_attn_fwd(_ptr(Q), _ptr(K), _ptr(V), _ptr(lengths), _ptr(out), ctypes.byref(shape),
                                 _ptr(workspace), workspace.numel(), _stream_ptr()))
    return out


# ---- what stands around the attention: layer norm, rotary positions, dense attention over packed sequences.
# Tensors of heads may have any strides the library takes (see psa_heads_t): [B, H, L, 64] or [H, T, 64] views of tensors
# that lie by head, by frame or inside a larger one.  Calls run on the tensors' own device, on its current stream.

def _device_of(*ts) -> torch.device:
    device = ts[0].device
    for t in ts:
        if t is not None and (not t.is_cuda or t.device != device):
            raise ValueError("tensors must be on one GPU")
    return device


def _require(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _require_like(t: Optional[torch.Tensor], shape, dtype, what: str, contiguous: bool = True):
    """`t` is None or has this shape and type (and, unless it is a tensor of heads, no strides)."""
    if t is not None:
        _require(tuple(t.shape) == tuple(shape), f"{what} must have shape {tuple(shape)}, not {tuple(t.shape)}")
        if t.dtype != dtype:
            raise TypeError(f"{what} must be {dtype}, not {t.dtype}")
        _require(t.is_contiguous() if contiguous else t.stride(-1) == 1,
                 f"{what} must be contiguous" + ("" if contiguous else " in its last dimension"))


def _launch(device: torch.device, function, *args):
    """One call of the library on the current stream of `device`."""
    if device.index == torch.cuda.current_device():
        _check(function(*args, torch.cuda.current_stream(device).cuda_stream))
    else:
        with torch.cuda.device(device):
            _check(function(*args, torch.cuda.current_stream(device).cuda_stream))


def _room(n: int, device: torch.device, given: Optional[torch.Tensor]) -> torch.Tensor:
    """The caller's workspace, or one of n bytes."""
    if n == 0:
        raise ProbSparseError(-2, "invalid shape or options for workspace sizing")
    if given is None:
        return torch.empty(n, dtype=torch.uint8, device=device)
    _require(given.is_contiguous() and given.device == device, "the workspace must be contiguous and on the tensors' device")
    return given


def _heads(t: torch.Tensor) -> PsaHeads:
    return PsaHeads(t.data_ptr(), t.stride(0) if t.dim() == 4 else 0, t.stride(-3), t.stride(-2))


def probsparse_layer_norm_fwd(X, gamma=None, beta=None, eps: float = 1e-5, Y=None, stats: bool = True):
    """Layer norm over the last dimension of X.  Returns (Y, mean, rstd) with stats (what the backward reads: float32, one
    for each row), else Y.  Y may be X."""
    done = (_native or _fast()).layer_norm_fwd(X, gamma, beta, eps, Y, stats)
    if done is not None:
        return done
    device = _device_of(X, gamma, beta, Y)
    _require(X.dim() >= 1 and X.numel() > 0 and X.is_contiguous(), "X must be contiguous and not empty")
    dtype, cols = _dtype_code(X), X.shape[-1]
    for t, what in ((gamma, "gamma"), (beta, "beta")):
        _require_like(t, (cols,), X.dtype, what)
    _require_like(Y, X.shape, X.dtype, "Y")
    if Y is None:
        Y = torch.empty_like(X)
    mean = rstd = None
    if stats:
        mean, rstd = (torch.empty(X.shape[:-1], dtype=torch.float32, device=device) for _ in range(2))
    _launch(device, load().probsparse_layer_norm_fwd, _ptr(X), _ptr(gamma), _ptr(beta), eps, _ptr(Y), _ptr(mean), _ptr(rstd),
            X.numel() // cols, cols, dtype)
    return (Y, mean, rstd) if stats else Y


def probsparse_layer_norm_bwd(dY, X, gamma, mean, rstd, workspace=None):
    """Gradients (dX, dgamma, dbeta) of probsparse_layer_norm_fwd; dgamma and dbeta are float32."""
    done = (_native or _fast()).layer_norm_bwd(dY, X, gamma, mean, rstd, workspace)
    if done is not None:
        return done
    device = _device_of(X, dY, gamma, mean, rstd, workspace)
    _require(X.dim() >= 1 and X.numel() > 0 and X.is_contiguous(), "X must be contiguous and not empty")
    dtype, cols = _dtype_code(X), X.shape[-1]
    rows = X.numel() // cols
    _require_like(dY, X.shape, X.dtype, "dY")
    _require_like(gamma, (cols,), X.dtype, "gamma")
    for t, what in ((mean, "mean"), (rstd, "rstd")):
        _require_like(t, X.shape[:-1], torch.float32, what)
    lib = load()
    workspace = _room(lib.probsparse_layer_norm_bwd_workspace_bytes(rows, cols, dtype), device, workspace)
    dX = torch.empty_like(X)
    dgamma, dbeta = (torch.empty(cols, dtype=torch.float32, device=device) for _ in range(2))
    _launch(device, lib.probsparse_layer_norm_bwd, _ptr(dY), _ptr(X), _ptr(gamma), _ptr(mean), _ptr(rstd), _ptr(dX), _ptr(dgamma),
            _ptr(dbeta), rows, cols, dtype, _ptr(workspace), workspace.numel() * workspace.element_size())
    return dX, dgamma, dbeta


def make_rotary(dim: int, layout: int = ROTARY_HALF, base: float = 10000.0, scaling: int = ROTARY_PLAIN, factor: float = 1.0,
                original_length: float = 0.0, fast_turns: float = 32.0, slow_turns: float = 1.0, magnitude: float = 1.0) -> PsaRotary:
    """How positions turn the first `dim` elements of a head (see psa_rotary_t); checked here."""
    rotary = PsaRotary(dim, layout, scaling, base, factor, original_length, fast_turns, slow_turns, magnitude)
    _check(load().probsparse_rotary_frequencies(ctypes.byref(rotary), (ctypes.c_double * 32)()))
    return rotary


def rotary_frequencies(rotary: PsaRotary) -> list:
    """Radians per position of each of the dim / 2 pairs."""
    freq = (ctypes.c_double * 32)()
    _check(load().probsparse_rotary_frequencies(ctypes.byref(rotary), freq))
    return list(freq)[:rotary.dim // 2]


def _rotary(back, Q, K, rotary, positions, first, Q_out, K_out):
    done = (_native or _fast()).rotary(back, Q, K, rotary, positions, first, Q_out, K_out)
    if done is not None:
        return done
    lib = load()
    function = lib.probsparse_rotary_bwd if back else lib.probsparse_rotary_fwd
    device = _device_of(Q, K, positions, Q_out, K_out)
    _require(Q.dim() in (3, 4) and Q.shape[-1] == 64, "Q must be [B, H, L, 64] or [H, T, 64]")
    dtype = _dtype_code(Q)
    B, (H, L) = Q.shape[0] if Q.dim() == 4 else 1, Q.shape[-3:-1]
    _require_like(Q, Q.shape, Q.dtype, "Q", contiguous=False)
    stride = 0
    if positions is not None:
        _require(positions.shape in ((L,), (B, L)), f"positions must be [{L}] or [{B}, {L}]")
        _require_like(positions, positions.shape, torch.int32, "positions")
        stride = L if positions.dim() == 2 else 0
    _require(K is not None or K_out is None, "K_out needs K")
    if K is not None:
        _require(K.dim() == Q.dim() and K.shape[:-3] == Q.shape[:-3] and K.shape[-2:] == Q.shape[-2:], "K must be Q but for its number of heads")
        _require_like(K, K.shape, Q.dtype, "K", contiguous=False)
        _require_like(K_out, K.shape, Q.dtype, "K_out", contiguous=False)
        if K_out is None:
            K_out = torch.empty_like(K)
    _require_like(Q_out, Q.shape, Q.dtype, "Q_out", contiguous=False)
    if Q_out is None:
        Q_out = torch.empty_like(Q)
    shape = make_shape(B, H, L, 1, dtype)
    q, qo = _heads(Q), _heads(Q_out)
    k, ko = (None, None) if K is None else (_heads(K), _heads(K_out))
    _launch(device, function, ctypes.byref(q), None if k is None else ctypes.byref(k), 0 if K is None else K.shape[-3], ctypes.byref(rotary),
            _ptr(positions), stride, first, ctypes.byref(qo), None if ko is None else ctypes.byref(ko), ctypes.byref(shape))
    return Q_out if K is None else (Q_out, K_out)


def probsparse_rotary_fwd(Q, K, rotary: PsaRotary, positions=None, first: int = 0, Q_out=None, K_out=None):
    """Q [B, H, L, 64] and K [B, H_kv, L, 64] (or [H, T, 64] and [H_kv, T, 64]) turned by their positions: `positions` int32 [L] or
    [B, L], or row l stands at first + l.  K may be None.  Returns (Q_out, K_out), or Q_out alone; an output may be its input."""
    return _rotary(False, Q, K, rotary, positions, first, Q_out, K_out)


def probsparse_rotary_bwd(dQ_out, dK_out, rotary: PsaRotary, positions=None, first: int = 0, dQ=None, dK=None):
    """The gradients of probsparse_rotary_fwd's inputs from those of its outputs."""
    return _rotary(True, dQ_out, dK_out, rotary, positions, first, dQ, dK)


def _packed(Q, K, V, q_offsets, k_offsets, causal, scale):
    _require(Q.dim() == 3 and Q.shape[-1] == 64, "Q must be [H, T_q, 64]")
    _require(K.dim() == 3 and K.shape[-1] == 64, "K must be [H_kv, T_k, 64]")
    _require(K.shape[0] > 0 and Q.shape[0] % K.shape[0] == 0, "the heads of Q must be a multiple of those of K")
    _require_like(Q, Q.shape, Q.dtype, "Q", contiguous=False)
    _require_like(K, K.shape, Q.dtype, "K", contiguous=False)
    _require_like(V, K.shape, Q.dtype, "V", contiguous=False)
    if k_offsets is None and q_offsets is not None:
        _require(Q.shape[1] == K.shape[1], "without k_offsets Q and K must have the same rows")
        k_offsets = q_offsets
    _require((q_offsets is None) == (k_offsets is None), "k_offsets need q_offsets")
    B = 1
    if q_offsets is not None:
        _require(q_offsets.dim() == 1 and q_offsets.numel() >= 2, "q_offsets must be [B + 1]")
        B = q_offsets.numel() - 1
        _require_like(q_offsets, (B + 1,), torch.int32, "q_offsets")
        _require_like(k_offsets, (B + 1,), torch.int32, "k_offsets")
    return k_offsets, PsaPackedShape(B, Q.shape[0], K.shape[0], Q.shape[1], K.shape[1], 64, _dtype_code(Q), int(bool(causal)),
                                     0.125 if scale is None else scale)


def dense_attn_packed_fwd(Q, K, V, q_offsets=None, k_offsets=None, causal: bool = False, scale: Optional[float] = None,
                          out=None, lse: bool = False, workspace=None):
    """Dense attention over packed sequences: Q [H, T_q, 64], K and V [H_kv, T_k, 64]; sequence s has the query rows
    q_offsets[s] .. q_offsets[s + 1] - 1 (int32 [B + 1]; None: one sequence) and the key rows of k_offsets (None: the same).
    `scale` is 1 / 8 unless given.  Returns out, or (out, lse) with lse [H, T_q] float32."""
    done = (_native or _fast()).packed_fwd(Q, K, V, q_offsets, k_offsets, causal, scale, out, lse, workspace)
    if done is not None:
        return done
    device = _device_of(Q, K, V, q_offsets, k_offsets, out, workspace)
    k_offsets, shape = _packed(Q, K, V, q_offsets, k_offsets, causal, scale)
    _require_like(out, Q.shape, Q.dtype, "out", contiguous=False)
    lib = load()
    workspace = _room(lib.dense_attn_packed_workspace_bytes(ctypes.byref(shape)), device, workspace)
    if out is None:
        out = torch.empty_like(Q)
    norm = torch.empty(Q.shape[:2], dtype=torch.float32, device=device) if lse else None
    q, k, v, o = _heads(Q), _heads(K), _heads(V), _heads(out)
    _launch(device, lib.dense_attn_packed_fwd, ctypes.byref(q), ctypes.byref(k), ctypes.byref(v), _ptr(q_offsets), _ptr(k_offsets),
            ctypes.byref(o), _ptr(norm), ctypes.byref(shape), _ptr(workspace), workspace.numel() * workspace.element_size())
    return (out, norm) if lse else out


def dense_attn_packed_bwd(Q, K, V, out, lse, dOut, q_offsets=None, k_offsets=None, causal: bool = False,
                          scale: Optional[float] = None, dQ=None, dK=None, dV=None, workspace=None):
    """Gradients (dQ, dK, dV) of dense_attn_packed_fwd, from its out and lse."""
    done = (_native or _fast()).packed_bwd(Q, K, V, out, lse, dOut, q_offsets, k_offsets, causal, scale, dQ, dK, dV, workspace)
    if done is not None:
        return done
    device = _device_of(Q, K, V, out, lse, dOut, q_offsets, k_offsets, dQ, dK, dV, workspace)
    k_offsets, shape = _packed(Q, K, V, q_offsets, k_offsets, causal, scale)
    for t, like, what in ((out, Q, "out"), (dOut, Q, "dOut"), (dQ, Q, "dQ"), (dK, K, "dK"), (dV, V, "dV")):
        _require_like(t, like.shape, Q.dtype, what, contiguous=False)
    _require_like(lse, Q.shape[:2], torch.float32, "lse")
    lib = load()
    workspace = _room(lib.dense_attn_packed_bwd_workspace_bytes(ctypes.byref(shape)), device, workspace)
    dQ, dK, dV = (torch.empty_like(t) if g is None else g for t, g in ((Q, dQ), (K, dK), (V, dV)))
    heads = [ctypes.byref(_heads(t)) for t in (Q, K, V, out, dOut, dQ, dK, dV)]
    _launch(device, lib.dense_attn_packed_bwd, *heads[:3], _ptr(q_offsets), _ptr(k_offsets), heads[3], _ptr(lse), *heads[4:],
            ctypes.byref(shape), _ptr(workspace), workspace.numel() * workspace.element_size())
    return dQ, dK, dV


def version() -> int:
    return load().probsparse_version()


def probsparse_describe_plan(shape, opt=None, u_stride: int = 0) -> dict:
    """The kernels a call with this shape would launch (host only), as a dict of the words of
    probsparse_describe_plan(); `opt` is a PsaOptions (selection rule) or None with u_stride > 0."""
    buf = ctypes.create_string_buffer(512)
    _check(load().probsparse_describe_plan(ctypes.byref(shape), None if opt is None else ctypes.byref(opt),
                                           u_stride, buf, len(buf)))
    return dict(word.split("=", 1) for word in buf.value.decode().split())


def probsparse_init() -> None:
    """Optional per-device set-up (see include/probsparse.h); needed only before capturing the first call on a device."""
    _check(load().probsparse_init())
