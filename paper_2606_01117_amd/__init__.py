"""Python binding of libhaste.so: the MI355X (gfx950) group-shared fixed fan-in output layer.

The functions below carry the names of the C ABI in ``include/haste.h`` and only marshal
arguments: torch tensors provide device memory and the current HIP stream, every step of the
layer runs in the library's HIP kernels.  The library must be built (``build.build()``); importing
this package without it raises immediately, there is no fallback implementation.

Layer (paper Section 3.1): labels in contiguous groups of G share one sorted support
idx[k, 0..F_in-1] of input features; label l keeps its own weights W[l, 0..F_in-1].
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libhaste.so")

HASTE_DTYPE_F32 = 0
HASTE_DTYPE_BF16 = 1
(HASTE_OP_FWD, HASTE_OP_BWD_W, HASTE_OP_BWD_X, HASTE_OP_FWD_BCE, HASTE_OP_FWD_BCE_SGD, HASTE_OP_REWIRE,
 HASTE_OP_TAIL_STEP, HASTE_OP_TAIL_STEP_SGD) = range(8)
STATUS = {0: "ok", 1: "invalid argument", 2: "unsupported", 3: "workspace too small", 4: "HIP error"}


class HasteError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class haste_desc_t(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("F_s", ctypes.c_int64), ("L", ctypes.c_int64), ("G", ctypes.c_int64),
                ("F_in", ctypes.c_int64), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class haste_sgd_t(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("momentum", ctypes.c_float), ("weight_decay", ctypes.c_float),
                ("reserved", ctypes.c_int32)]


class haste_group_opts_t(ctypes.Structure):
    _fields_ = [("G", ctypes.c_int64), ("beta", ctypes.c_int64), ("iters", ctypes.c_int64), ("seed", ctypes.c_uint64)]


class haste_param_t(ctypes.Structure):
    _fields_ = [("W", ctypes.c_void_p), ("W32", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("lr_scale", ctypes.c_float), ("weight_decay", ctypes.c_float), ("dtype", ctypes.c_int32),
                ("grad_dtype", ctypes.c_int32), ("state_bits", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class haste_adamw_opts_t(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_int64), ("seed", ctypes.c_uint64),
                ("lr_dev", ctypes.c_void_p), ("step_dev", ctypes.c_void_p), ("grad_scale", ctypes.c_void_p)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"libhaste.so is not built ({LIB_PATH}); run paper_2606_01117_amd.build.build()")
    lib = ctypes.CDLL(LIB_PATH)
    P, I64, I32, SZ, F32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t, ctypes.c_float
    L = ctypes.POINTER(haste_param_t)
    D = ctypes.POINTER(haste_desc_t)
    sigs = {
        "haste_fwd": [D, P, P, P, P, P, P, SZ, P],
        "haste_bwd_w": [D, P, P, P, P, P, ctypes.c_int, P, SZ, P],
        "haste_bwd_x": [D, P, P, P, P, ctypes.c_int, P, SZ, P],
        "haste_fwd_bce": [D, P, P, P, P, P, I32, P, P, P, ctypes.c_int, P, SZ, P],
        "haste_fwd_bce_static": [D, P, P, P, P, P, I32, P, P, P, ctypes.c_int, P],
        "haste_bce_grad": [I64, I64, I32, P, P, I32, P, P],
        "haste_fwd_bce_sgd": [D, P, P, P, P, P, I32, P, P, ctypes.POINTER(haste_sgd_t), P, P, P, SZ, P],
        "haste_sgd_momentum": [I64, I32, P, P, P, ctypes.POINTER(haste_sgd_t), P, P],
        "haste_rewire": [D, P, P, P, ctypes.c_double, I32, ctypes.c_uint64, P, P, SZ, P],
        "haste_group_labels": [I64, I64, P, ctypes.POINTER(haste_group_opts_t), P, P, P, P, P, SZ, P],
        "haste_head_fwd": [I64, I64, I64, I32, P, P, P, P, P],
        "haste_tail_step": [D, P, P, P, P, P, I32, P, P, P, ctypes.c_int, P, ctypes.c_int, P, SZ, P],
        "haste_tail_step_sgd": [D, P, P, P, P, P, I32, P, P, ctypes.POINTER(haste_sgd_t), P, P, P, ctypes.c_int, P, SZ,
                                P],
        "haste_head_fwd_bce": [I64, I64, I64, I32, P, P, P, P, I32, P, P],
        "haste_head_bwd": [I64, I64, I64, I32, P, P, P, P, P, ctypes.c_int, P, SZ, P],
        "haste_layer_norm_fwd": [I64, I64, I32, P, I64, P, P, F32, I32, P, I64, P, P, P],
        "haste_layer_norm_bwd": [I64, I64, I32, P, I64, P, P, P, I32, P, I64, P, I64, P, P, ctypes.c_int, P, SZ, P],
        "haste_grad_norm": [L, I64, F32, P, P, SZ, P],
        "haste_adamw": [L, I64, ctypes.POINTER(haste_adamw_opts_t), P],
        "haste_validate_idx": [D, P, P, P],
        "haste_debug_gather": [D, P, P, I64, I64, P, P],
    }
    for name, args in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    lib.haste_workspace_bytes.argtypes = [D, ctypes.c_int]
    lib.haste_workspace_bytes.restype = SZ
    lib.haste_head_workspace_bytes.argtypes = [I64, I64, I64, I32]
    lib.haste_head_workspace_bytes.restype = SZ
    lib.haste_group_workspace_bytes.argtypes = [I64, I64, ctypes.POINTER(haste_group_opts_t)]
    lib.haste_group_workspace_bytes.restype = SZ
    lib.haste_layer_norm_workspace_bytes.argtypes = [I64, I64]
    lib.haste_layer_norm_workspace_bytes.restype = SZ
    lib.haste_grad_norm_workspace_bytes.argtypes = [L, I64]
    lib.haste_grad_norm_workspace_bytes.restype = SZ
    lib.haste_fwd_bce_static_max_bytes.argtypes = []
    lib.haste_fwd_bce_static_max_bytes.restype = SZ
    for name in ("haste_status_str", "haste_last_error", "haste_version"):
        getattr(lib, name).restype = ctypes.c_char_p
    lib.haste_status_str.argtypes = [ctypes.c_int]
    return lib


lib = _load()

# every symbol the header declares
EXPORTS = ("haste_fwd", "haste_bwd_w", "haste_bwd_x", "haste_fwd_bce", "haste_fwd_bce_static",
           "haste_fwd_bce_static_max_bytes", "haste_fwd_bce_sgd", "haste_sgd_momentum",
           "haste_rewire", "haste_group_labels", "haste_group_workspace_bytes", "haste_bce_grad", "haste_head_fwd",
           "haste_layer_norm_fwd", "haste_layer_norm_bwd", "haste_layer_norm_workspace_bytes", "haste_grad_norm",
           "haste_grad_norm_workspace_bytes", "haste_adamw",
           "haste_head_fwd_bce", "haste_head_bwd", "haste_tail_step", "haste_tail_step_sgd", "haste_workspace_bytes", "haste_head_workspace_bytes", "haste_validate_idx", "haste_debug_gather", "haste_status_str",
           "haste_last_error", "haste_version")


def haste_version() -> str:
    return lib.haste_version().decode()


def haste_status_str(status: int) -> str:
    return lib.haste_status_str(status).decode()


def haste_last_error() -> str:
    return lib.haste_last_error().decode()


def _check(rc: int):
    if rc != 0:
        raise HasteError(rc, haste_last_error())


def make_desc(B: int, F_s: int, L: int, G: int, F_in: int, dtype: int) -> haste_desc_t:
    return haste_desc_t(B, F_s, L, G, F_in, dtype, 0)


# ---- marshalling helpers (torch only supplies memory and the stream) ------------------------
def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_contiguous():
        raise ValueError("tensors passed to libhaste must be contiguous")
    return t.data_ptr()


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _stream(stream, device=None) -> Optional[int]:
    """The handle of a stream; None is the current one (of the current device, if the caller knows it)."""
    if stream is None:
        torch = _torch()
        # the current stream's handle; without this entry, through a Stream object, which takes ten times as long
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return raw(torch.cuda.current_device() if device is None else device)
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _ws(ws):
    if ws is None:
        return None, 0
    if isinstance(ws, tuple):
        return ws
    return ws.data_ptr(), ws.numel() * ws.element_size()


def workspace(nbytes: int, device="cuda"):
    """A caller-owned device workspace of nbytes bytes (None when nothing is needed)."""
    if nbytes == 0:
        return None
    import torch
    return torch.empty(int(nbytes), dtype=torch.uint8, device=device)


# ---- the C ABI ----------------------------------------------------------------------------
def haste_workspace_bytes(desc: haste_desc_t, op: int) -> int:
    return int(lib.haste_workspace_bytes(ctypes.byref(desc), op))


def haste_head_workspace_bytes(B: int, F_s: int, H: int, dtype: int) -> int:
    return int(lib.haste_head_workspace_bytes(B, F_s, H, dtype))


def haste_fwd(desc, X, idx, W, bias, Y, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib.haste_fwd(ctypes.byref(desc), _ptr(X), _ptr(idx), _ptr(W), _ptr(bias), _ptr(Y), p, n, _stream(stream)))


def haste_bwd_w(desc, X, idx, dY, dW, dbias=None, beta=0, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib.haste_bwd_w(ctypes.byref(desc), _ptr(X), _ptr(idx), _ptr(dY), _ptr(dW), _ptr(dbias), int(beta), p, n,
                           _stream(stream)))


def haste_bwd_x(desc, idx, W, dY, dX, beta=0, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib.haste_bwd_x(ctypes.byref(desc), _ptr(idx), _ptr(W), _ptr(dY), _ptr(dX), int(beta), p, n,
                           _stream(stream)))


def _npos(pos) -> int:
    return 0 if pos is None else int(pos.shape[1])


def haste_fwd_bce(desc, X, idx, W, bias, pos, dY, dW=None, dbias=None, beta=0, ws=None, stream=None):
    """pos: [B, P] int32 tensor of positive tail column ids (or None for no positives)."""
    p, n = _ws(ws)
    _check(lib.haste_fwd_bce(ctypes.byref(desc), _ptr(X), _ptr(idx), _ptr(W), _ptr(bias), _ptr(pos), _npos(pos),
                             _ptr(dY), _ptr(dW), _ptr(dbias), int(beta), p, n, _stream(stream)))


def haste_fwd_bce_static(desc, X, idx, W, bias, pos, dY, dW=None, dbias=None, beta=0, stream=None):
    """haste_fwd_bce with the library's own per-device scratch (no workspace, allocates nothing)."""
    _check(lib.haste_fwd_bce_static(ctypes.byref(desc), _ptr(X), _ptr(idx), _ptr(W), _ptr(bias), _ptr(pos),
                                    _npos(pos), _ptr(dY), _ptr(dW), _ptr(dbias), int(beta), _stream(stream)))


def haste_fwd_bce_static_max_bytes() -> int:
    return int(lib.haste_fwd_bce_static_max_bytes())


def haste_tail_step(desc, X, idx, W, bias, pos, dY, dW, dbias, beta, dX, beta_dx, ws=None, stream=None):
    """haste_fwd_bce followed by haste_bwd_x on its dY (pos: [B, P] int32 tensor or None)."""
    p, n = _ws(ws)
    _check(lib.haste_tail_step(ctypes.byref(desc), _ptr(X), _ptr(idx), _ptr(W), _ptr(bias), _ptr(pos), _npos(pos),
                               _ptr(dY), _ptr(dW), _ptr(dbias), int(beta), _ptr(dX), int(beta_dx), p, n,
                               _stream(stream)))


def haste_tail_step_sgd(desc, X, idx, W, bias, pos, dY, dbias, opt, m, W_next, dX, beta_dx, ws=None, stream=None):
    """haste_fwd_bce_sgd followed by haste_bwd_x on its dY with the step's W."""
    p, n = _ws(ws)
    _check(lib.haste_tail_step_sgd(ctypes.byref(desc), _ptr(X), _ptr(idx), _ptr(W), _ptr(bias), _ptr(pos), _npos(pos),
                                   _ptr(dY), _ptr(dbias), ctypes.byref(opt), _ptr(m), _ptr(W_next), _ptr(dX),
                                   int(beta_dx), p, n, _stream(stream)))


def sgd_opts(lr: float, momentum: float, weight_decay: float = 0.0) -> haste_sgd_t:
    return haste_sgd_t(lr, momentum, weight_decay, 0)


def haste_fwd_bce_sgd(desc, X, idx, W, bias, pos, dY, opt, m, W_next, dbias=None, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib.haste_fwd_bce_sgd(ctypes.byref(desc), _ptr(X), _ptr(idx), _ptr(W), _ptr(bias), _ptr(pos), _npos(pos),
                                 _ptr(dY), _ptr(dbias), ctypes.byref(opt), _ptr(m), _ptr(W_next), p, n,
                                 _stream(stream)))


def haste_sgd_momentum(n, dtype, W, grad, m, opt, W_next, stream=None):
    _check(lib.haste_sgd_momentum(int(n), dtype, _ptr(W), _ptr(grad), _ptr(m), ctypes.byref(opt), _ptr(W_next),
                                  _stream(stream)))


def haste_rewire(desc, idx, W, m, rho, init_random, seed, ws=None, stream=None) -> int:
    """Rewires in place; returns the number of pruned slots."""
    p, n = _ws(ws)
    npr = ctypes.c_int64(0)
    _check(lib.haste_rewire(ctypes.byref(desc), _ptr(idx), _ptr(W), _ptr(m), float(rho), int(init_random),
                            int(seed) & ((1 << 64) - 1), ctypes.byref(npr), p, n, _stream(stream)))
    return int(npr.value)


def group_opts(G: int, beta: int, iters: int, seed: int) -> haste_group_opts_t:
    return haste_group_opts_t(G, beta, iters, seed & ((1 << 64) - 1))


def haste_group_workspace_bytes(N, D, opts) -> int:
    return int(lib.haste_group_workspace_bytes(N, D, ctypes.byref(opts)))


def haste_group_labels(E, opts, order, gsize, n_groups, cluster=None, ws=None, stream=None):
    """E: [N, D] int8 device tensor; n_groups: a 1-element int64 device tensor."""
    p, n = _ws(ws)
    N, D = E.shape
    _check(lib.haste_group_labels(N, D, _ptr(E), ctypes.byref(opts), _ptr(order), _ptr(gsize), _ptr(n_groups),
                                  _ptr(cluster), p, n, _stream(stream)))


def haste_bce_grad(B, N, dtype, Y, pos, dY, stream=None):
    _check(lib.haste_bce_grad(B, N, dtype, _ptr(Y), _ptr(pos), _npos(pos), _ptr(dY), _stream(stream)))


def haste_head_fwd(B, F_s, H, dtype, X, W_head, bias_h, Y_h, stream=None):
    _check(lib.haste_head_fwd(B, F_s, H, dtype, _ptr(X), _ptr(W_head), _ptr(bias_h), _ptr(Y_h), _stream(stream)))


def haste_head_fwd_bce(B, F_s, H, dtype, X, W_head, bias_h, pos, dY_h, stream=None):
    _check(lib.haste_head_fwd_bce(B, F_s, H, dtype, _ptr(X), _ptr(W_head), _ptr(bias_h), _ptr(pos), _npos(pos),
                                  _ptr(dY_h), _stream(stream)))


def haste_head_bwd(B, F_s, H, dtype, X, W_head, dY_h, dW_h, dX, beta_dx=0, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib.haste_head_bwd(B, F_s, H, dtype, _ptr(X), _ptr(W_head), _ptr(dY_h), _ptr(dW_h), _ptr(dX),
                              int(beta_dx), p, n, _stream(stream)))


_row_dtypes = {}


def _rows(t, B, F, dtype, name):
    """Address and row stride of a [B, F] tensor whose rows may lie apart."""
    if t is None:
        return None, F
    if not _row_dtypes:
        torch = _torch()
        _row_dtypes.update({HASTE_DTYPE_F32: (torch.float32, torch.int32),        # the values, or their bits
                            HASTE_DTYPE_BF16: (torch.bfloat16, torch.int16)})
    if t.shape != (B, F) or t.dtype not in _row_dtypes.get(dtype, ()):
        raise ValueError(f"{name} must be [{B}, {F}] of the dtype that the call names, got {tuple(t.shape)} {t.dtype}")
    ld, step = t.stride()
    if F > 1 and step != 1:
        raise ValueError(f"{name} must have the values of a row next to each other")
    if B > 1 and ld < F:
        raise ValueError(f"{name} must have rows that do not overlap")
    return t.data_ptr(), ld if B > 1 else F


def _vec(t, n, name, device):
    """Address of a contiguous fp32 vector of n values."""
    if t is None:
        return None
    if t.numel() != n or t.element_size() != 4 or not t.is_floating_point() or not t.is_contiguous():
        raise ValueError(f"{name} must be {n} contiguous fp32 values, got {tuple(t.shape)} {t.dtype}")
    if t.get_device() != device:
        _elsewhere(t, name)
    return t.data_ptr()


def _here(t, name):
    """The device of a tensor, which must be the current GPU."""
    if t is None:
        raise ValueError(f"{name} is missing")
    device = t.get_device()
    if device < 0 or device != _torch().cuda.current_device():
        _elsewhere(t, name)
    return device


def _elsewhere(t, name):
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    raise ValueError(f"{name} is on {t.device}, not on the current device cuda:{_torch().cuda.current_device()}")


def haste_layer_norm_workspace_bytes(B: int, F: int) -> int:
    return int(lib.haste_layer_norm_workspace_bytes(int(B), int(F)))


def haste_layer_norm_fwd(B, F, dtype_h, H, weight, bias, eps, dtype_x, X, mean=None, rstd=None, stream=None):
    """H and X: [B, F] tensors of dtype_h and dtype_x; their rows may lie apart (a view such as tokens[:, 0])."""
    (h, ldh), (x, ldx) = _rows(H, B, F, dtype_h, "H"), _rows(X, B, F, dtype_x, "X")
    on = _here(H, "H")
    if X is None:
        raise ValueError("X is missing")
    if X.get_device() != on:
        _elsewhere(X, "X")
    _check(lib.haste_layer_norm_fwd(B, F, dtype_h, h, ldh, _vec(weight, F, "weight", on), _vec(bias, F, "bias", on), eps,
                                    dtype_x, x, ldx, _vec(mean, B, "mean", on), _vec(rstd, B, "rstd", on),
                                    _stream(stream, on)))


def haste_layer_norm_bwd(B, F, dtype_h, H, weight, mean, rstd, dtype_dx, dX, dH=None, dweight=None, dbias=None, beta=0,
                         ws=None, stream=None):
    """dX and dH: [B, F] tensors of dtype_dx and dtype_h, rows apart or not; beta applies to dweight and dbias."""
    p, n = _ws(ws)
    (h, ldh), (dx, lddx) = _rows(H, B, F, dtype_h, "H"), _rows(dX, B, F, dtype_dx, "dX")
    dh, lddh = _rows(dH, B, F, dtype_h, "dH")
    on = _here(H, "H")
    for t, name in ((dX, "dX"), (dH, "dH")):
        if t is not None and t.get_device() != on:
            _elsewhere(t, name)
    _check(lib.haste_layer_norm_bwd(B, F, dtype_h, h, ldh, _vec(weight, F, "weight", on), _vec(mean, B, "mean", on),
                                    _vec(rstd, B, "rstd", on), dtype_dx, dx, lddx, dh, lddh,
                                    _vec(dweight, F, "dweight", on), _vec(dbias, F, "dbias", on), int(beta), p, n,
                                    _stream(stream, on)))


_codes = {}


def _dtype_of(t, name) -> int:
    if not _codes:
        _codes.update({_torch().float32: HASTE_DTYPE_F32, _torch().bfloat16: HASTE_DTYPE_BF16})
    code = _codes.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be torch.float32 or torch.bfloat16, got {t.dtype}")
    return code


_byte_types_of = []


def _byte_types():
    """The types of 8-bit moments and of their scales: bytes, or what they stand for."""
    if not _byte_types_of:
        torch = _torch()
        _byte_types_of.extend(({torch.uint8, torch.int8, torch.float8_e4m3fn}, {torch.uint8, torch.int8, torch.float8_e8m0fnu}))
    return _byte_types_of


def param(W=None, grad=None, m=None, v=None, scale=None, W32=None, lr_scale=1.0, weight_decay=0.0) -> haste_param_t:
    """One tensor of a list for haste_grad_norm (which needs grad alone) and haste_adamw.

    W (fp32 or bf16), grad (fp32 or bf16), and the moments m and v: fp32, or of one byte a value (uint8, or
    float8_e4m3fn) with scale, uint8 [ceil(n / 32), 2].  All contiguous, of n values each, on the current GPU.  The
    entry keeps the tensors alive."""
    if grad is None and W is None:
        raise ValueError("an entry needs grad, or W")
    first = grad if grad is not None else W
    n, device = first.numel(), _here(first, "grad" if grad is not None else "W")

    def at(t, name, count):
        if t is None:
            return None
        if t.numel() != count or not t.is_contiguous():
            raise ValueError(f"{name} must be {count} contiguous values, got {tuple(t.shape)}")
        if t.get_device() != device:
            _elsewhere(t, name)
        return t.data_ptr()

    bits = 32
    if m is not None and v is not None:
        if m.element_size() == 1 and v.element_size() == 1:
            bits = 8
            moments, exponents = _byte_types()
            if m.dtype not in moments or v.dtype not in moments:
                raise ValueError(f"8-bit moments must be uint8 or float8_e4m3fn, got {m.dtype} and {v.dtype}")
            if scale is None or scale.dtype not in exponents:
                raise ValueError(f"8-bit moments of {n} values need scale, uint8 [{(n + 31) // 32}, 2]")
        elif _dtype_of(m, "m") != HASTE_DTYPE_F32 or _dtype_of(v, "v") != HASTE_DTYPE_F32:
            raise ValueError("m and v must both be torch.float32, or both of one byte a value")
    if W32 is not None and _dtype_of(W32, "W32") != HASTE_DTYPE_F32:
        raise ValueError("W32 must be torch.float32")
    p = haste_param_t(at(W, "W", n), at(W32, "W32", n), at(grad, "grad", n), at(m, "m", n), at(v, "v", n),
                      at(scale, "scale", 2 * ((n + 31) // 32)), n, lr_scale, weight_decay,
                      0 if W is None else _dtype_of(W, "W"), 0 if grad is None else _dtype_of(grad, "grad"), bits, 0)
    p.keep, p.device = (W, grad, m, v, scale, W32), device
    return p


class _Entries:
    """The array of a list's entries.  One that is taken out of it or put into it brings its tensors and their device
    along: a ctypes array alone copies the addresses, and the tensors behind them could be freed."""

    def __getitem__(self, k):
        if isinstance(k, slice):
            return [self[i] for i in range(*k.indices(len(self)))]
        p = super().__getitem__(k)               # the entry in place: what is written to it, the list has
        p.keep = self.keep[k]
        p.device = None if p.keep is None else self.device
        return p

    def __setitem__(self, k, p):
        if isinstance(k, slice):
            raise TypeError("the entries of a list are set one by one")
        device = getattr(p, "device", None)
        if device is not None and self.device is not None and device != self.device:
            raise ValueError(f"the tensors of a list must be on one GPU, not on {sorted((device, self.device))}")
        super().__setitem__(k, p)
        self.keep[k] = getattr(p, "keep", None)
        self.device = device if self.device is None else self.device


_list_types = {}


def param_list(params):
    """The array of entries that haste_grad_norm and haste_adamw take; made once, it serves every step (set_grads points
    it at new gradients).  Entries may be taken out of one list and put into another, or replaced in place."""
    params = list(params)
    n = len(params)
    devices = {getattr(p, "device", None) for p in params} - {None}
    if len(devices) > 1:
        raise ValueError(f"the tensors of a list must be on one GPU, not on {sorted(devices)}")
    if n not in _list_types:
        _list_types[n] = type("param_list", (_Entries, haste_param_t * n), {})
    array = _list_types[n].from_buffer((haste_param_t * n)(*params)) if n else _list_types[n]()
    array.keep = [getattr(p, "keep", None) for p in params]
    array.device = devices.pop() if devices else None
    return array


def set_grads(params, grads):
    """Points a param_list at new gradients, in the order of its entries: contiguous, fp32 or bf16, of the entries' sizes,
    on the list's GPU; None leaves an entry's gradient as it is.  The list keeps the new tensors alive and no longer the
    old ones (which, as any tensor, must live on where a call on another stream still reads them); nothing is changed
    where one of them is refused.  A graph captured before holds the old addresses."""
    grads = list(grads)
    if len(grads) != len(params):
        raise ValueError(f"{len(grads)} gradients for a list of {len(params)} tensors")
    entries, dtypes = params[:], [None if g is None else _dtype_of(g, "grad") for g in grads]
    device = params.device
    for k, (p, g) in enumerate(zip(entries, grads)):
        if g is None:
            continue
        device = _here(g, "grad") if device is None else device
        if g.numel() != p.n or not g.is_contiguous():
            raise ValueError(f"grad of tensor {k} must be {p.n} contiguous values, got {tuple(g.shape)}")
        if g.get_device() != device:
            raise ValueError(f"grad of tensor {k} is on {g.device}, the list on cuda:{device}")
    for k, (p, g, dtype) in enumerate(zip(entries, grads, dtypes)):
        if g is not None:
            p.grad, p.grad_dtype = g.data_ptr(), dtype
            keep = params.keep[k] or (None,) * 6
            params.keep[k] = (keep[0], g, *keep[2:])
    params.device = device


def _still_here(params, opts=None):
    """Tensors that a list and options hold must be on the GPU that is current at the call, too; that GPU, if they hold any."""
    a, b = getattr(params, "device", None), getattr(opts, "device", None)
    if a is None and b is None:
        return None
    now = _torch().cuda.current_device()
    if (a is None or a == now) and (b is None or b == now):
        return now
    device, whose = (b, "options'") if a is None or a == now else (a, "list's")
    raise ValueError(f"the {whose} tensors are on cuda:{device}, not on the current device cuda:{now}")


def adamw_opts(lr, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0, lr_dev=None, step_dev=None,
               grad_scale=None) -> haste_adamw_opts_t:
    """Options of haste_adamw; the caller sets .step (and .lr) before each call.  lr_dev (fp32), step_dev (int64)
    and grad_scale (fp32, haste_grad_norm's out[1:]) are GPU tensors of one value, or None."""
    torch = _torch()
    o = haste_adamw_opts_t(lr=lr, beta1=beta1, beta2=beta2, eps=eps, step=step, seed=seed & ((1 << 64) - 1))
    o.keep = (lr_dev, step_dev, grad_scale)
    o.device = None
    for t, name, dtype in ((lr_dev, "lr_dev", torch.float32), (step_dev, "step_dev", torch.int64),
                           (grad_scale, "grad_scale", torch.float32)):
        if t is None:
            continue
        if t.numel() != 1 or t.dtype != dtype:
            raise ValueError(f"{name} must be one value of {dtype}")
        o.device = _here(t, name)
        setattr(o, name, t.data_ptr())
    return o


def haste_grad_norm_workspace_bytes(params) -> int:
    return int(lib.haste_grad_norm_workspace_bytes(params, len(params)))


def haste_grad_norm(params, max_norm, out, ws=None, stream=None):
    """params: a param_list; out: two fp32 values on the GPU, the norm and the factor that clips it to max_norm."""
    on = _still_here(params)
    p, n = _ws(ws)
    _check(lib.haste_grad_norm(params, len(params), max_norm, _vec(out, 2, "out", _here(out, "out")), p, n,
                               _stream(stream, on)))


def haste_adamw(params, opts, stream=None):
    """One AdamW step over a param_list, in place."""
    on = _still_here(params, opts)
    _check(lib.haste_adamw(params, len(params), ctypes.byref(opts), _stream(stream, on)))


def haste_validate_idx(desc, idx, n_bad_rows, stream=None):
    _check(lib.haste_validate_idx(ctypes.byref(desc), _ptr(idx), _ptr(n_bad_rows), _stream(stream)))


def haste_debug_gather(desc, X, idx, k0, nk, out, stream=None):
    _check(lib.haste_debug_gather(ctypes.byref(desc), _ptr(X), _ptr(idx), int(k0), int(nk), _ptr(out),
                                  _stream(stream)))
