"""Python binding of the C ABI in ``include/forge.h`` and ``include/forge_ops.h`` (argument
marshalling only).

Every function here has the name of the C entry point it calls.  Tensors are torch
tensors on the current HIP device; their data pointers, shapes and the current torch
stream are passed through ctypes.  All arithmetic runs in the HIP kernels of
``libforge.so``; there is no fallback: if the library is not built, calls raise.
"""
from __future__ import annotations

import ctypes
import functools
import os
import re
import threading

from . import build as _build

FORGE_MOMENT_F32, FORGE_MOMENT_BF16, FORGE_MOMENT_I8, FORGE_MOMENT_I8_ROW64, FORGE_MOMENT_FP8 = 0, 1, 2, 3, 4
AMAX_SLOTS = 4
FORGE_GRAD_BF16, FORGE_GRAD_F32 = 0, 1

STATUS = {
    0: "FORGE_OK", 1: "FORGE_ERR_NULL_POINTER", 2: "FORGE_ERR_INVALID_SHAPE",
    3: "FORGE_ERR_UNSUPPORTED_SHAPE", 4: "FORGE_ERR_INVALID_HYPERPARAM",
    5: "FORGE_ERR_INVALID_DTYPE", 6: "FORGE_ERR_MISALIGNED", 7: "FORGE_ERR_ALIASING",
    8: "FORGE_ERR_NO_DEVICE", 9: "FORGE_ERR_LAUNCH", 10: "FORGE_ERR_INVALID_OPTIMIZER",
    11: "FORGE_ERR_SCRATCH_LIMIT",
}
# bytes of the library's fixed device buffer (FORGE_SCRATCH_BYTES)
FORGE_SCRATCH_BYTES = 64 << 20
# forge_optimizer codes of include/forge.h
OPTIMIZERS = {"adamw": 0, "sgd": 1, "sgd_momentum": 2, "adagrad": 3, "rmsprop": 4, "lion": 5, "nadam": 6,
              "radam": 7, "adamax": 8, "muon_accumulate": 9}
# state tensors each update rule reads and writes
OPTIMIZER_STATES = {"adamw": 2, "sgd": 0, "sgd_momentum": 1, "adagrad": 1, "rmsprop": 1, "lion": 1, "nadam": 2,
                    "radam": 2, "adamax": 2, "muon_accumulate": 1}
HEADER = os.path.join(_build.ROOT, "include", "forge.h")
OPS_HEADER = os.path.join(_build.ROOT, "include", "forge_ops.h")


class ForgeError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        self.name = STATUS.get(code, "unknown")
        super().__init__(f"{where}: {forge_status_string(code)}")


_lock = threading.Lock()
_lib = None

_P, _I64, _I32, _F = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float
FORGE_MAX_GROUP = 8


class forge_hparams(ctypes.Structure):
    """``forge_hparams`` of ``include/forge.h``."""
    _fields_ = [("lr", _F), ("beta1", _F), ("beta2", _F), ("eps", _F), ("weight_decay", _F),
                ("lr_decay", _F), ("momentum_decay", _F)]


class forge_matrix(ctypes.Structure):
    """``forge_matrix`` of ``include/forge.h``: one matrix of a grouped step."""
    _fields_ = [("X", _P), ("dY", _P), ("W", _P), ("m", _P), ("v", _P), ("m_scale", _P),
                ("v_scale", _P), ("d_in", _I64), ("d_out", _I64)]


_SIGS = {
    "forge_linear_step": [_P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _I32, _F, _F, _F, _F, _F, _I64, _P],
    "forge_linear_step_grouped": [ctypes.POINTER(forge_matrix), _I32, _I64, _I32, _F, _F, _F, _F, _F,
                                  _I64, _P],
    "forge_linear_step_opt": [_P, _P, _P, _P, _P, _I64, _I64, _I64, _I32, _I32, ctypes.POINTER(forge_hparams),
                              _I64, _P],
    "forge_linear_step_wfp8": [_P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _I32, _F, _F, _F, _F, _F, _I64,
                               _P],
    "forge_input_grad": [_P, _P, _P, _I64, _I64, _I64, _P],
    "forge_linear_backward": [_P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _I32, _F, _F, _F, _F, _F,
                              _I64, _P],
    "forge_linear_backward_grouped": [ctypes.POINTER(forge_matrix), _I32, _I64, _P, _I32, _F, _F, _F, _F,
                                      _F, _I64, _P],
    "forge_wgrad": [_P, _P, _P, _I64, _I64, _I64, _I32, _P],
    "forge_adamw": [_P, _I32, _P, _P, _P, _P, _P, _I64, _I64, _I32, _F, _F, _F, _F, _F, _I64, _P],
    "forge_linear_step_unfused": [_P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _I32, _F, _F, _F, _F,
                                  _F, _I64, _P, _I32, _P],
    "forge_linear_step_unfused_noalloc": [_P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _I32, _F, _F, _F, _F,
                                          _F, _I64, _I32, _P],
    "forge_status_string": [_I32],
    "forge_query_tile": [_I64, _I64, _I64, _I32, ctypes.POINTER(_I32), ctypes.POINTER(_I32),
                         ctypes.POINTER(_I32)],
}


class forge_tensor(ctypes.Structure):
    """``forge_tensor`` of ``include/forge_ops.h``: one tensor of a list."""
    _fields_ = [("W", _P), ("G", _P), ("m", _P), ("v", _P), ("m_scale", _P), ("v_scale", _P), ("numel", _I64),
                ("lr_scale", _F), ("weight_decay", _F), ("w_dtype", _I32), ("g_dtype", _I32), ("state_dtype", _I32),
                ("reserved", _I32)]


class forge_tensor_list(ctypes.Structure):
    """``forge_tensor_list`` of ``include/forge_ops.h``."""
    _fields_ = [("table_bytes", _I64), ("chunks", _I64), ("n", _I32), ("steppable", _I32)]


_LIST = ctypes.POINTER(forge_tensor_list)
# include/forge_ops.h
_OPS_SIGS = {
    "forge_rmsnorm": [_P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I32, _I32, _I32, _F, _P],
    "forge_rmsnorm_backward": [_P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I32, _I32, _F, _P, _I64, _P],
    "forge_rmsnorm_backward_workspace": [_I64, _I64],
    "forge_tensor_list_bytes": [ctypes.POINTER(forge_tensor), _I32],
    "forge_tensor_list_build": [ctypes.POINTER(forge_tensor), _I32, _P, _I64, _LIST],
    "forge_grad_norm": [_LIST, _P, _F, _P, _P, _I64, _P],
    "forge_grad_norm_workspace": [_LIST],
    "forge_adamw_multi": [_LIST, _P, _F, _F, _F, _F, _P, _I64, _P],
}


def lib():
    """The loaded ``libforge.so`` (raises if it has not been built)."""
    global _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(_build.LIB):
                raise RuntimeError(
                    f"{_build.LIB} is not built: run `python -m paper_2606_22932_amd.build` "
                    "(or __graft_entry__.build()) first; there is no non-HIP fallback")
            L = ctypes.CDLL(_build.LIB)
            for name, args in _SIGS.items():
                fn = getattr(L, name)
                fn.argtypes = args
                fn.restype = ctypes.c_char_p if name == "forge_status_string" else ctypes.c_int32
            _lib = L
    return _lib


def header_functions(path=None):
    """Names of the functions ``include/forge.h`` (or the header at ``path``) declares."""
    text = open(path or HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(forge_[a-z_0-9]+)\s*\(", text)))


def forge_status_string(code: int) -> str:
    return lib().forge_status_string(int(code)).decode()


def forge_query_tile(T: int, d_in: int, d_out: int, moment_dtype: int):
    r, c, t = _I32(), _I32(), _I32()
    st = lib().forge_query_tile(int(T), int(d_in), int(d_out), int(moment_dtype), ctypes.byref(r),
                                ctypes.byref(c), ctypes.byref(t))
    _check(st, "forge_query_tile")
    return r.value, c.value, t.value


# ----------------------------------------------------------------------------- marshalling

def _check(status: int, where: str):
    if status != 0:
        raise ForgeError(status, where)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream, ref):
    if stream is not None:
        return ctypes.c_void_p(int(stream))
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream(ref.device).cuda_stream)


def _moment_code(m, m_scale=None):
    """Moment dtype code; int8 moments name their layout through the scale tensor's shape:
    [ceil(d_out/256), d_in] (256-row column blocks) or [d_out, ceil(d_in/64)] (64-wide row
    blocks)."""
    import torch
    codes = {torch.float32: FORGE_MOMENT_F32, torch.bfloat16: FORGE_MOMENT_BF16,
             torch.float8_e4m3fn: FORGE_MOMENT_FP8}
    if m.dtype in codes:
        if m.dtype == torch.float8_e4m3fn and (m_scale is None or m_scale.numel() != AMAX_SLOTS):
            raise ValueError(f"fp8 moments need amax rings of {AMAX_SLOTS} float32 (m_scale, v_scale)")
        return codes[m.dtype]
    if m.dtype != torch.int8:
        raise TypeError(f"moments must be float32, bfloat16 or int8, got {m.dtype}")
    if m_scale is None:
        raise ValueError("int8 moments need their scale tensors")
    d_out, d_in = m.shape
    if tuple(m_scale.shape) == ((d_out + 255) // 256, d_in):
        return FORGE_MOMENT_I8
    if tuple(m_scale.shape) == (d_out, (d_in + 63) // 64):
        return FORGE_MOMENT_I8_ROW64
    raise ValueError(f"int8 scale shape {tuple(m_scale.shape)} matches neither layout for moments {tuple(m.shape)}")


def _grad_code(G):
    import torch
    codes = {torch.bfloat16: FORGE_GRAD_BF16, torch.float32: FORGE_GRAD_F32}
    if G.dtype not in codes:
        raise TypeError(f"gradient must be bfloat16 or float32, got {G.dtype}")
    return codes[G.dtype]


def _dev(*ts):
    for t in ts:
        if t is not None:
            if not t.is_cuda:
                raise ValueError("forge tensors must live on a HIP device")
            if not t.is_contiguous():
                raise ValueError("forge tensors must be contiguous")


def _shapes(X, dY, W):
    import torch
    if W.dtype != torch.bfloat16 or X.dtype != torch.bfloat16 or dY.dtype != torch.bfloat16:
        raise TypeError("X, dY and W must be bfloat16")
    T, d_in = X.shape
    T2, d_out = dY.shape
    if T2 != T or tuple(W.shape) != (d_out, d_in):
        raise ValueError(f"shape mismatch: X {tuple(X.shape)}, dY {tuple(dY.shape)}, W {tuple(W.shape)}")
    return T, d_in, d_out


def forge_linear_step(X, dY, W, m, v, m_scale=None, v_scale=None, *, lr, beta1, beta2, eps,
                      weight_decay, step, stream=None):
    """The fused step: W, m, v (and int8 scales) updated in place; G is never stored."""
    _dev(X, dY, W, m, v, m_scale, v_scale)
    T, d_in, d_out = _shapes(X, dY, W)
    st = lib().forge_linear_step(_ptr(X), _ptr(dY), _ptr(W), _ptr(m), _ptr(v), _ptr(m_scale),
                                 _ptr(v_scale), T, d_in, d_out, _moment_code(m, m_scale), lr, beta1, beta2,
                                 eps, weight_decay, int(step), _stream(stream, W))
    _check(st, "forge_linear_step")


def forge_linear_step_opt(X, dY, W, s1=None, s2=None, *, optimizer, lr, beta1=0.0, beta2=0.0, eps=1e-8,
                          weight_decay=0.0, lr_decay=0.0, momentum_decay=0.004, step, stream=None):
    """The fused step with update rule ``optimizer`` (a key of OPTIMIZERS) on fp32 or bf16
    state tensors s1, s2 (as many as the rule has).  W may be None for 'muon_accumulate'."""
    import torch
    if optimizer not in OPTIMIZERS:
        raise ValueError(f"unknown optimizer {optimizer!r}; one of {sorted(OPTIMIZERS)}")
    ns = OPTIMIZER_STATES[optimizer]
    states = [t for t in (s1, s2)[:ns]]
    if any(t is None for t in states):
        raise ValueError(f"{optimizer} needs {ns} state tensor(s)")
    _dev(X, dY, W, *states)
    if X.dtype != torch.bfloat16 or dY.dtype != torch.bfloat16:
        raise TypeError("X and dY must be bfloat16")
    T, d_in = X.shape
    T2, d_out = dY.shape
    if T2 != T:
        raise ValueError("X and dY disagree on T")
    for t in ([W] if W is not None else []):
        if t.dtype != torch.bfloat16 or tuple(t.shape) != (d_out, d_in):
            raise ValueError("W must be bfloat16 [d_out, d_in]")
    code = FORGE_MOMENT_BF16
    if states:
        if states[0].dtype == torch.int8:
            raise ValueError("forge_linear_step_opt takes float32 or bfloat16 state")
        code = _moment_code(states[0])
        if any(t.dtype != states[0].dtype or tuple(t.shape) != (d_out, d_in)
                                          for t in states):
            raise ValueError("state tensors must all be float32 or all bfloat16, [d_out, d_in]")
    hp = forge_hparams(lr, beta1, beta2, eps, weight_decay, lr_decay, momentum_decay)
    ref = W if W is not None else dY
    st = lib().forge_linear_step_opt(_ptr(X), _ptr(dY), _ptr(W), _ptr(s1 if ns >= 1 else None),
                                     _ptr(s2 if ns >= 2 else None), T, d_in, d_out, OPTIMIZERS[optimizer], code,
                                     ctypes.byref(hp), int(step), _stream(stream, ref))
    _check(st, "forge_linear_step_opt")


def forge_linear_step_wfp8(X, dY, W, w_amax, m, v, m_amax=None, v_amax=None, *, lr, beta1, beta2, eps,
                           weight_decay, step, stream=None):
    """The fused step with W in fp8 (float8_e4m3fn codes, amax ring ``w_amax`` of 4 float32)
    and bf16 moments, or fp8 moments (float8_e4m3fn codes of m and sqrt(v) with their rings)."""
    import torch
    _dev(X, dY, W, w_amax, m, v, m_amax, v_amax)
    if X.dtype != torch.bfloat16 or dY.dtype != torch.bfloat16 or W.dtype != torch.float8_e4m3fn:
        raise TypeError("X, dY must be bfloat16 and W float8_e4m3fn")
    T, d_in = X.shape
    T2, d_out = dY.shape
    if T2 != T or tuple(W.shape) != (d_out, d_in):
        raise ValueError(f"shape mismatch: X {tuple(X.shape)}, dY {tuple(dY.shape)}, W {tuple(W.shape)}")
    if w_amax.dtype != torch.float32 or w_amax.numel() != AMAX_SLOTS:
        raise ValueError(f"w_amax must be {AMAX_SLOTS} float32")
    code = _moment_code(m, m_amax)
    if code not in (FORGE_MOMENT_BF16, FORGE_MOMENT_FP8):
        raise TypeError("moments must be bfloat16 or float8_e4m3fn")
    st = lib().forge_linear_step_wfp8(_ptr(X), _ptr(dY), _ptr(W), _ptr(w_amax), _ptr(m), _ptr(v), _ptr(m_amax),
                                      _ptr(v_amax), T, d_in, d_out, code, lr, beta1, beta2, eps, weight_decay,
                                      int(step), _stream(stream, W))
    _check(st, "forge_linear_step_wfp8")


def _group(mats):
    """ctypes array of forge_matrix for (X, dY, W, m, v[, m_scale, v_scale]) tuples, T, dtype code."""
    mats = [tuple(x) + (None,) * (7 - len(x)) for x in mats]
    if not mats:
        raise ValueError("empty group")
    arr = (forge_matrix * len(mats))()
    T = code = None
    for i, (X, dY, W, m, v, ms, vs) in enumerate(mats):
        _dev(X, dY, W, m, v, ms, vs)
        Ti, d_in, d_out = _shapes(X, dY, W)
        ci = _moment_code(m, ms)
        if T is None:
            T, code = Ti, ci
        elif Ti != T or ci != code:
            raise ValueError("all matrices of a group share T and the moment dtype")
        arr[i] = forge_matrix(X.data_ptr(), dY.data_ptr(), W.data_ptr(), m.data_ptr(), v.data_ptr(),
                              None if ms is None else ms.data_ptr(), None if vs is None else vs.data_ptr(),
                              d_in, d_out)
    return arr, len(mats), T, code, mats[0][2]


def forge_linear_step_grouped(mats, *, lr, beta1, beta2, eps, weight_decay, step, stream=None):
    """The fused step on several independent matrices in one launch.

    ``mats``: sequence of ``(X, dY, W, m, v)`` or ``(X, dY, W, m, v, m_scale, v_scale)``
    tuples sharing the token count T and the moment dtype (at most FORGE_MAX_GROUP).
    """
    arr, n, T, code, ref = _group(mats)
    st = lib().forge_linear_step_grouped(arr, n, T, code, lr, beta1, beta2, eps, weight_decay,
                                         int(step), _stream(stream, ref))
    _check(st, "forge_linear_step_grouped")


def _dx(dX, T, d_in):
    import torch
    _dev(dX)
    if dX.dtype != torch.bfloat16 or tuple(dX.shape) != (T, d_in):
        raise ValueError(f"dX must be bfloat16 [{T}, {d_in}], got {dX.dtype} {tuple(dX.shape)}")


def forge_input_grad(dY, W, dX, *, stream=None):
    """dX = dY W (bf16 out, fp32 accumulation): the layer's input gradient."""
    import torch
    _dev(dY, W)
    if dY.dtype != torch.bfloat16 or W.dtype != torch.bfloat16:
        raise TypeError("dY and W must be bfloat16")
    T, d_out = dY.shape
    if W.shape[0] != d_out:
        raise ValueError(f"shape mismatch: dY {tuple(dY.shape)}, W {tuple(W.shape)}")
    d_in = W.shape[1]
    _dx(dX, T, d_in)
    st = lib().forge_input_grad(_ptr(dY), _ptr(W), _ptr(dX), T, d_in, d_out, _stream(stream, dX))
    _check(st, "forge_input_grad")


def forge_linear_backward(X, dY, W, m, v, m_scale=None, v_scale=None, *, dX, lr, beta1, beta2, eps,
                          weight_decay, step, stream=None):
    """The layer-level backward: dX = dY W from the pre-update W, then the fused step."""
    _dev(X, dY, W, m, v, m_scale, v_scale)
    T, d_in, d_out = _shapes(X, dY, W)
    _dx(dX, T, d_in)
    st = lib().forge_linear_backward(_ptr(X), _ptr(dY), _ptr(W), _ptr(m), _ptr(v), _ptr(m_scale),
                                     _ptr(v_scale), _ptr(dX), T, d_in, d_out, _moment_code(m, m_scale), lr, beta1,
                                     beta2, eps, weight_decay, int(step), _stream(stream, W))
    _check(st, "forge_linear_backward")


def forge_linear_backward_grouped(mats, *, dX, lr, beta1, beta2, eps, weight_decay, step, stream=None):
    """Backward of several projections of one input: dX = sum_i dY_i W_i (pre-update
    weights, one launch), then the grouped fused step.  ``mats`` as for
    ``forge_linear_step_grouped``; all share d_in."""
    arr, n, T, code, ref = _group(mats)
    _dx(dX, T, arr[0].d_in)
    st = lib().forge_linear_backward_grouped(arr, n, T, _ptr(dX), code, lr, beta1, beta2, eps,
                                             weight_decay, int(step), _stream(stream, ref))
    _check(st, "forge_linear_backward_grouped")


def forge_wgrad(X, dY, G, *, stream=None):
    """G = dY^T X stored in G's dtype (bfloat16 or float32)."""
    _dev(X, dY, G)
    T, d_in = X.shape
    d_out = dY.shape[1]
    if tuple(G.shape) != (d_out, d_in):
        raise ValueError("G must be [d_out, d_in]")
    st = lib().forge_wgrad(_ptr(X), _ptr(dY), _ptr(G), T, d_in, d_out, _grad_code(G), _stream(stream, G))
    _check(st, "forge_wgrad")


def forge_adamw(G, W, m, v, m_scale=None, v_scale=None, *, lr, beta1, beta2, eps, weight_decay,
                step, stream=None):
    """The stand-alone optimizer kernel over a materialised gradient G."""
    _dev(G, W, m, v, m_scale, v_scale)
    d_out, d_in = W.shape
    if tuple(G.shape) != (d_out, d_in):
        raise ValueError("G must match W")
    st = lib().forge_adamw(_ptr(G), _grad_code(G), _ptr(W), _ptr(m), _ptr(v), _ptr(m_scale),
                           _ptr(v_scale), d_in, d_out, _moment_code(m, m_scale), lr, beta1, beta2, eps,
                           weight_decay, int(step), _stream(stream, W))
    _check(st, "forge_adamw")


def forge_linear_step_unfused(X, dY, W, m, v, m_scale=None, v_scale=None, *, G_ws, lr, beta1,
                              beta2, eps, weight_decay, step, stream=None):
    """GEMM writes G into G_ws, then the optimizer kernel reads it (same stream)."""
    _dev(X, dY, W, m, v, m_scale, v_scale, G_ws)
    T, d_in, d_out = _shapes(X, dY, W)
    if G_ws.numel() < d_in * d_out:
        raise ValueError("G_ws too small")
    st = lib().forge_linear_step_unfused(_ptr(X), _ptr(dY), _ptr(W), _ptr(m), _ptr(v),
                                         _ptr(m_scale), _ptr(v_scale), T, d_in, d_out,
                                         _moment_code(m, m_scale), lr, beta1, beta2, eps, weight_decay,
                                         int(step), _ptr(G_ws), _grad_code(G_ws), _stream(stream, W))
    _check(st, "forge_linear_step_unfused")


def forge_linear_step_unfused_noalloc(X, dY, W, m, v, m_scale=None, v_scale=None, *, grad_dtype, lr, beta1,
                                      beta2, eps, weight_decay, step, stream=None):
    """forge_linear_step_unfused with G in the library's fixed device buffer: allocates
    nothing.  grad_dtype: "bf16" or "f32"."""
    _dev(X, dY, W, m, v, m_scale, v_scale)
    T, d_in, d_out = _shapes(X, dY, W)
    gd = {"bf16": FORGE_GRAD_BF16, "f32": FORGE_GRAD_F32}[grad_dtype]
    st = lib().forge_linear_step_unfused_noalloc(_ptr(X), _ptr(dY), _ptr(W), _ptr(m), _ptr(v),
                                                 _ptr(m_scale), _ptr(v_scale), T, d_in, d_out,
                                                 _moment_code(m, m_scale), lr, beta1, beta2, eps, weight_decay,
                                                 int(step), gd, _stream(stream, W))
    _check(st, "forge_linear_step_unfused_noalloc")


# ----------------------------------------------------------------------------- include/forge_ops.h

FORGE_DTYPE_F32, FORGE_DTYPE_BF16, FORGE_DTYPE_FP8 = 0, 1, 2
FORGE_Q_GROUP, FORGE_STATE_BLOCK = 128, 64
_ops_lib = None


def _ops():
    """``lib()`` with the prototypes of ``include/forge_ops.h``."""
    global _ops_lib
    if _ops_lib is None:
        L = lib()
        for name, args in _OPS_SIGS.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = _I64 if name.endswith(("_workspace", "_bytes")) else _I32
        _ops_lib = L
    return _ops_lib


def _adr(t):
    return None if t is None else t.data_ptr()


def _float_code(t, what):
    import torch
    dt = t.dtype
    if dt is torch.bfloat16:
        return FORGE_DTYPE_BF16
    if dt is torch.float32:
        return FORGE_DTYPE_F32
    raise TypeError(f"{what} must be bfloat16 or float32, got {dt}")


def _bytes_ws(ws, need):
    if ws is None:
        if need:
            raise ValueError(f"ws of {need} bytes needed")
        return 0
    if ws.nbytes < need:
        raise ValueError(f"ws too small: {ws.nbytes} bytes, {need} needed")
    return ws.nbytes


def _one_device(*specs):
    """Index of the HIP device that the tensors of (tensor or None, name, shape, dtype) live on,
    contiguous and as said (a shape or dtype of None: any).  One loop, for the calls on a single
    token, which take as long as their binding."""
    dev = None
    for t, what, shape, dtype in specs:
        if t is None:
            continue
        at = t.get_device()
        if at != dev or not t.is_contiguous():
            _dev(t)
            if dev is not None:
                raise ValueError(f"tensors on different devices: {dev} and {at}")
            dev = at
        if (shape is not None and t.shape != shape) or (dtype is not None and t.dtype is not dtype):
            raise ValueError(f"{what} must be {dtype or 'a tensor'} {'' if shape is None else tuple(shape)}, "
                             f"got {t.dtype} {tuple(t.shape)}")
    return dev


def _launch(name, dev, stream, *args):
    """The C entry point with ``dev`` current, on ``stream`` or torch's current one there."""
    import torch
    if stream is None:
        # the handle alone: torch.cuda.current_stream makes an object for it, 2 us a call
        stream = torch._C._cuda_getCurrentRawStream(dev)
    fn = getattr(_ops_lib or _ops(), name)
    if torch.cuda.current_device() == dev:
        st = fn(*args, stream)
    else:
        with torch.cuda.device(dev):
            st = fn(*args, stream)
    if st:
        raise ForgeError(st, name)


def forge_rmsnorm(x, w, *, residual=None, h=None, y=None, q=None, q_scale=None, eps, stream=None):
    """h = residual + x (rounded to the residual's type), y = h / sqrt(mean(h^2) + eps) * w over
    the last axis of [T, d] tensors; without a residual y is that of x itself.

    ``y`` is bfloat16; ``q`` float8_e4m3fn with ``q_scale`` float32 [T] (a scale per row) or
    [T, ceil(d / 128)] (per 128 columns).  ``h`` goes with a residual and may be the residual.
    """
    import torch
    bf16 = torch.bfloat16
    shape = T, d = x.shape
    s = x if residual is None else residual
    group, scales = 0, None
    if q is not None and q_scale is not None:
        group = FORGE_Q_GROUP if q_scale.dim() == 2 else 0
        scales = (T, (d + 127) // 128) if group else (T,)
    dev = _one_device((x, "x beside a residual", shape, None if residual is None else bf16), (w, "w", (d,), None),
                      (residual, "residual", shape, None), (h, "h", shape, s.dtype), (y, "y", shape, bf16),
                      (q, "q", shape, torch.float8_e4m3fn), (q_scale, "q_scale", scales, torch.float32))
    _launch("forge_rmsnorm", dev, stream, x.data_ptr(), _adr(residual), w.data_ptr(), _adr(h), _adr(y), _adr(q),
            _adr(q_scale), T, d, _float_code(s, "the stream"), _float_code(w, "w"), group, eps)


@functools.lru_cache(maxsize=256)
def forge_rmsnorm_backward_workspace(T, d):
    """Bytes of the workspace of ``forge_rmsnorm_backward`` on [T, d]."""
    return _ops().forge_rmsnorm_backward_workspace(int(T), int(d))


def forge_rmsnorm_backward(dy, h, w, *, dres=None, dh=None, dx=None, dw, eps, ws, stream=None):
    """The gradient of ``forge_rmsnorm``: dh (in h's type) and / or dx (bfloat16), both
    dres + the norm's gradient, and dw (float32).  ``h`` is what the norm was taken of; dh may be
    dres.  ``ws``: any tensor of at least ``forge_rmsnorm_backward_workspace(T, d)`` bytes."""
    import torch
    bf16 = torch.bfloat16
    shape = T, d = dy.shape
    ht = h.dtype
    dev = _one_device((dy, "dy", shape, bf16), (h, "h", shape, None), (w, "w", (d,), None), (dres, "dres", shape, ht),
                      (dh, "dh", shape, ht), (dx, "dx", shape, bf16), (dw, "dw", (d,), torch.float32),
                      (ws, "ws", None, None))
    n = _bytes_ws(ws, forge_rmsnorm_backward_workspace(T, d))
    _launch("forge_rmsnorm_backward", dev, stream, dy.data_ptr(), h.data_ptr(), w.data_ptr(), _adr(dres), _adr(dh),
            _adr(dx), dw.data_ptr(), T, d, _float_code(h, "h"), _float_code(w, "w"), eps, _adr(ws), n)


class TensorList:
    """Tensors that ``forge_adamw_multi`` steps and ``forge_grad_norm`` reads together.

    ``tensors``: sequence of ``(W, G, m, v)`` or ``(W, G, m, v, m_scale, v_scale)`` tuples of
    one device, of any shapes and types (W, G float32 or bfloat16; m and v float32, bfloat16, or
    float8_e4m3fn with float32 scales of ceil(numel / 64) elements); ``(None, G)`` for a list
    that is only normed.  ``lr_scale`` and ``weight_decay``: a number, or one per tensor.

    Built once for tensors that stay where they are, and held on to while calls or captured
    graphs use it; it keeps the tensors alive.  Their types are checked and their addresses laid
    out and copied to the device here, not at each call: after gradients (or anything else) were
    allocated anew, build another, or give the new ones to ``with_gradients``.  Either takes some
    hundred microseconds for some hundred tensors and waits for the work queued on the current
    stream.  A stream that calls were given by its handle outlives the list.
    """

    def __init__(self, tensors, *, lr_scale=1.0, weight_decay=0.0):
        import torch
        self.tensors = [tuple(x) + (None,) * (6 - len(x)) for x in tensors]
        n = len(self.tensors)
        if n and torch.cuda.is_available() and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("a TensorList is built (and its table copied to the device) outside of graph capture")
        each = lambda x: [float(x)] * n if isinstance(x, (int, float)) else [float(y) for y in x]
        self.lr_scale, self.weight_decay = each(lr_scale), each(weight_decay)
        if len(self.lr_scale) != n or len(self.weight_decay) != n:
            raise ValueError("lr_scale and weight_decay: one number, or one per tensor")
        if any(t[1] is None for t in self.tensors):
            raise ValueError("a tensor of a list needs its gradient")
        arr = (forge_tensor * max(n, 1))()
        self.device = self.tensors[0][1].device if n else None
        for i, (t, ls, wd) in enumerate(zip(self.tensors, self.lr_scale, self.weight_decay)):
            arr[i] = self._entry(t, ls, wd)
        L = _ops()
        self.list = forge_tensor_list()
        host = torch.zeros(max(L.forge_tensor_list_bytes(arr, n), 16), dtype=torch.uint8)
        _check(L.forge_tensor_list_build(arr, n, host.data_ptr(), host.nbytes, ctypes.byref(self.list)), "TensorList")
        self.table = host.to(self.device) if n else None
        self._ref = ctypes.byref(self.list)
        self._norm_ws = L.forge_grad_norm_workspace(self._ref)
        # the table belongs to the stream that is current here (the copy itself has ended)
        self._home = torch.cuda.current_stream(self.device).cuda_stream if n else 0

    def _entry(self, t, lr_scale, weight_decay):
        import torch
        W, G, m, v, ms, vs = t
        at = self.device.index if self.device.type == "cuda" else -1
        for x in t:
            if x is not None:
                if x.get_device() != at or at < 0:
                    _dev(x)
                    raise ValueError("the tensors of a list live on one device")
                if not x.is_contiguous():
                    _dev(x)
        n, g = G.numel(), _float_code(G, "gradients")
        if W is None:
            return forge_tensor(None, G.data_ptr(), None, None, None, None, n, lr_scale, weight_decay, 0, g, 0, 0)
        shape = G.shape
        if m is None or v is None or W.shape != shape or m.shape != shape or v.shape != shape:
            raise ValueError("W, G, m and v of a tensor have one shape")
        dt = m.dtype
        if dt is not v.dtype:
            raise TypeError(f"m and v have one type, got {m.dtype} and {v.dtype}")
        if dt is torch.float8_e4m3fn:
            for s in (ms, vs):
                if s is None or s.dtype is not torch.float32 or s.numel() != (n + 63) // 64:
                    raise ValueError("fp8 moments need float32 scales of ceil(numel / 64) elements")
            st = FORGE_DTYPE_FP8
        else:
            st, ms, vs = _float_code(m, "moments"), None, None
        return forge_tensor(W.data_ptr(), G.data_ptr(), m.data_ptr(), v.data_ptr(), _adr(ms), _adr(vs), n, lr_scale,
                            weight_decay, _float_code(W, "weights"), g, st, 0)

    def with_gradients(self, gradients):
        """A list of the same weights and state with other gradients."""
        g = list(gradients)
        if len(g) != len(self.tensors):
            raise ValueError("one gradient per tensor")
        return TensorList([(t[0], x) + t[2:] for t, x in zip(self.tensors, g)], lr_scale=self.lr_scale,
                          weight_decay=self.weight_decay)

    def _use(self, stream):
        """The stream's handle, the table kept from reuse until that stream is done with it."""
        import torch
        if stream is None:
            stream = torch._C._cuda_getCurrentRawStream(self.device.index)
        stream = int(stream)
        if stream != self._home:
            self.table.record_stream(torch.cuda.ExternalStream(stream, self.device))
        return stream


def forge_grad_norm_workspace(tensors):
    """Bytes of the workspace of ``forge_grad_norm`` on a TensorList."""
    return tensors._norm_ws


def forge_grad_norm(tensors, out, *, max_norm, ws, stream=None):
    """out[0] = the 2-norm of all gradients of a TensorList, out[1] = min(1, max_norm / (out[0] +
    1e-6)); ``out`` float32 [2], ``out[1:]`` is what ``forge_adamw_multi`` takes as grad_scale."""
    import torch
    dev = _one_device((out, "out", (2,), torch.float32), (ws, "ws", None, None), (tensors.table, "table", None, None))
    n = _bytes_ws(ws, forge_grad_norm_workspace(tensors))
    _launch("forge_grad_norm", dev, stream if tensors.table is None else tensors._use(stream), tensors._ref,
            _adr(tensors.table), max_norm, out.data_ptr(), _adr(ws), n)


def forge_adamw_multi(tensors, *, lr, beta1, beta2, eps, step, grad_scale=None, stream=None):
    """One AdamW step on every tensor of a TensorList in one launch; learning rate and weight
    decay per tensor as the list says, gradients times ``grad_scale`` (one float32 on the
    device, read when the step runs)."""
    import torch
    if tensors.table is None:
        return
    dev = _one_device((tensors.table, "table", None, None), (grad_scale, "grad_scale", None, torch.float32))
    if grad_scale is not None and grad_scale.numel() != 1:
        raise ValueError("grad_scale must be one float32")
    _launch("forge_adamw_multi", dev, tensors._use(stream), tensors._ref, tensors.table.data_ptr(), lr, beta1, beta2,
            eps, _adr(grad_scale), int(step))
