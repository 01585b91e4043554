"""ctypes binding of libhdet.so: the same names and arguments as include/hdet.h.

Argument marshalling only -- every step of the path runs in the library's HIP kernels.
PyTorch tensors are accepted where the C ABI takes device pointers (their data_ptr() is
passed); PyTorch is used for device memory and streams, nothing else.  There is no CPU
fallback: loading fails loudly if libhdet.so has not been built.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

HDET_MAX_REPLICAS = 64
HDET_MAX_CH = 8
HDET_MAX_GROUPS = 4
HDET_MAX_LAYERS = 16

HDET_OK, HDET_EINVAL, HDET_ESTATE, HDET_EHIP, HDET_ENONFINITE = 0, -1, -2, -3, -4
HDET_SGDM, HDET_ADAMW = 0, 1
HDET_GRAD_SHARED, HDET_GRAD_PER_REPLICA = 0, 1
HDET_FP32, HDET_BF16_GEMM_FP32_MASTER = 0, 1
HDET_FLAT, HDET_MLP, HDET_TRANSFORMER = 0, 1, 2
HDET_CH_LR, HDET_CH_DROPOUT, HDET_CH_WD, HDET_CH_LABEL_SMOOTH, HDET_CH_ATTN_TEMP = 0, 1, 2, 3, 4
HDET_FUSE_CONVERGE = 1
HDET_TYPE_F32, HDET_TYPE_BF16 = 0, 1
HDET_MAX_NORM_WIDTH, HDET_MAX_CODES_WIDTH = 32768, 131056
HDET_VOCAB_NO_DW, HDET_VOCAB_LOSSES = -1, -2

EXPORTS = [
    "hdet_workspace_bytes", "hdet_create", "hdet_warm_init", "hdet_warm_init_noalloc", "hdet_forward_backward", "hdet_fanout_step", "hdet_train_step",
    "hdet_converge", "hdet_autolr_update", "hdet_get_state", "hdet_set_state",
    "hdet_set_launch_shape", "hdet_last_error", "hdet_destroy",
    "hdet_rmsnorm", "hdet_rmsnorm_backward_workspace", "hdet_rmsnorm_backward", "hdet_quantise_rows", "hdet_restore_rows",
    "hdet_quantised_linear", "hdet_quantised_linear_backward_workspace", "hdet_quantised_linear_backward",
    "hdet_vocab_loss_workspace", "hdet_vocab_loss",
]


class hdet_channel(C.Structure):
    _fields_ = [("kind", C.c_int32), ("reserved", C.c_int32), ("base", C.c_double),
                ("alpha", C.c_double), ("lambda_", C.c_double), ("lo", C.c_double),
                ("hi", C.c_double)]


class hdet_model_dims(C.Structure):
    _fields_ = [("n_params", C.c_int64), ("n_layers", C.c_int32),
                ("widths", C.c_int32 * (HDET_MAX_LAYERS + 1)), ("batch", C.c_int32),
                ("n_blocks", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("d_ff", C.c_int32), ("seq_len", C.c_int32), ("vocab", C.c_int32)]


class hdet_config(C.Structure):
    _fields_ = [
        ("n_replicas", C.c_int32), ("sync_interval", C.c_int32),
        ("total_steps", C.c_int64), ("warm_steps", C.c_int64),
        ("lr_max", C.c_double), ("f_div", C.c_double), ("f_final", C.c_double),
        ("pct_start", C.c_double),
        ("constant_lr", C.c_int32), ("autolr_enabled", C.c_int32),
        ("alpha", C.c_double), ("beta", C.c_double), ("sigma", C.c_double),
        ("lambda_", C.c_double), ("gamma_override", C.c_double),
        ("optimizer", C.c_int32), ("grad_mode", C.c_int32),
        ("shared_opt_state", C.c_int32), ("reshuffle_every_sync", C.c_int32),
        ("momentum", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double),
        ("eps", C.c_double), ("weight_decay", C.c_double),
        ("precision", C.c_int32), ("model_kind", C.c_int32),
        ("dims", hdet_model_dims),
        ("n_extra_channels", C.c_int32), ("n_groups", C.c_int32),
        ("group_end", C.c_int64 * HDET_MAX_GROUPS),
        ("extra", hdet_channel * (HDET_MAX_CH - 1)),
        ("seed", C.c_uint64), ("stream", C.c_void_p),
    ]


class hdet_buffers(C.Structure):
    _fields_ = [("params_dev", C.c_void_p), ("grads_dev", C.c_void_p), ("opt_m_dev", C.c_void_p),
                ("opt_v_dev", C.c_void_p), ("params_bf16_dev", C.c_void_p),
                ("workspace_dev", C.c_void_p), ("workspace_bytes", C.c_size_t),
                ("plane_stride", C.c_int64)]


class hdet_state(C.Structure):
    _fields_ = [
        ("t", C.c_int64), ("k", C.c_int64), ("controller_active", C.c_int32),
        ("nonfinite", C.c_int32), ("n_replicas", C.c_int32), ("n_channels", C.c_int32),
        ("autolr_done", C.c_int32), ("reserved", C.c_int32),
        ("gamma", C.c_double),
        ("base", C.c_double * HDET_MAX_CH), ("vel", C.c_double * HDET_MAX_CH),
        ("delta", C.c_double * HDET_MAX_CH),
        ("w", C.c_double * HDET_MAX_REPLICAS), ("l_acc", C.c_double * HDET_MAX_REPLICAS),
        ("l_last", C.c_double * HDET_MAX_REPLICAS), ("l_step", C.c_float * HDET_MAX_REPLICAS),
        ("lr", C.c_float * HDET_MAX_REPLICAS),
        ("rho", (C.c_double * HDET_MAX_REPLICAS) * HDET_MAX_CH),
        ("perm", (C.c_int32 * HDET_MAX_REPLICAS) * HDET_MAX_CH),
    ]


class hdet_rows(C.Structure):
    _fields_ = [("dev", C.c_void_p), ("row_stride", C.c_int64), ("replica_stride", C.c_int64)]


class hdet_norm_args(C.Structure):
    _fields_ = [("n_replicas", C.c_int32), ("dtype", C.c_int32), ("rows", C.c_int64), ("width", C.c_int32), ("reserved", C.c_int32),
                ("eps", C.c_double), ("x", hdet_rows), ("resid", hdet_rows), ("total", hdet_rows), ("y", hdet_rows), ("codes", hdet_rows),
                ("scale_dev", C.c_void_p), ("rstd_dev", C.c_void_p), ("gain_dev", C.c_void_p), ("gain_stride", C.c_int64)]


class hdet_norm_grad_args(C.Structure):
    _fields_ = [("n_replicas", C.c_int32), ("dtype", C.c_int32), ("rows", C.c_int64), ("width", C.c_int32), ("reserved", C.c_int32),
                ("total", hdet_rows), ("dy", hdet_rows), ("dtotal", hdet_rows), ("dx", hdet_rows),
                ("rstd_dev", C.c_void_p), ("gain_dev", C.c_void_p), ("gain_stride", C.c_int64), ("dgain_dev", C.c_void_p),
                ("dgain_stride", C.c_int64), ("workspace_dev", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class hdet_codes_args(C.Structure):
    _fields_ = [("n_replicas", C.c_int32), ("dtype", C.c_int32), ("rows", C.c_int64), ("width", C.c_int32), ("reserved", C.c_int32),
                ("values", hdet_rows), ("codes", hdet_rows), ("scale_dev", C.c_void_p)]


class hdet_linear_args(C.Structure):
    _fields_ = [("n_replicas", C.c_int32), ("y_dtype", C.c_int32), ("rows", C.c_int64), ("d_in", C.c_int32), ("d_out", C.c_int32),
                ("codes", hdet_rows), ("w_codes", hdet_rows), ("scale_dev", C.c_void_p), ("w_scale_dev", C.c_void_p),
                ("bias_dev", C.c_void_p), ("bias_stride", C.c_int64), ("y", hdet_rows)]


class hdet_linear_grad_args(C.Structure):
    _fields_ = [("n_replicas", C.c_int32), ("reserved", C.c_int32), ("rows", C.c_int64), ("d_in", C.c_int32), ("d_out", C.c_int32),
                ("dy", hdet_rows), ("codes", hdet_rows), ("w_codes", hdet_rows), ("scale_dev", C.c_void_p), ("w_scale_dev", C.c_void_p),
                ("dx", hdet_rows), ("dw", hdet_rows), ("db_dev", C.c_void_p), ("db_stride", C.c_int64),
                ("workspace_dev", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class hdet_vocab_args(C.Structure):
    _fields_ = [("n_replicas", C.c_int32), ("dw_dtype", C.c_int32), ("rows", C.c_int64), ("width", C.c_int32), ("classes", C.c_int32),
                ("piece", C.c_int32), ("reserved", C.c_int32), ("h", hdet_rows), ("w", hdet_rows), ("bias_dev", C.c_void_p),
                ("bias_stride", C.c_int64), ("labels_dev", C.c_void_p), ("row_loss_dev", C.c_void_p), ("mean_loss_dev", C.c_void_p),
                ("dh", hdet_rows), ("dw", hdet_rows), ("db_dev", C.c_void_p), ("db_stride", C.c_int64),
                ("workspace_dev", C.c_void_p), ("workspace_bytes", C.c_size_t)]


LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libhdet.so")
_lib = None


class HdetError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"hdet error {code}: {message}")
        self.code = code


def load_library(path: Optional[str] = None):
    """Loads libhdet.so (built by paper_2604_24708_amd.build) and declares the prototypes."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} is missing: build it with `python -m paper_2604_24708_amd.build` "
                           "(there is no CPU fallback)")
    # One HIP runtime per process: PyTorch ships its own libamdhip64 and must be the one that
    # libhdet.so binds to, or the library and the tensors it is handed would live in two
    # runtimes (the second one finds no device).  Importing torch first loads that copy.
    import torch
    global _F32, _BF16, _I8, _I32, _CODE
    _F32, _BF16, _I8, _I32 = torch.float32, torch.bfloat16, torch.int8, torch.int32
    _CODE = {_F32: HDET_TYPE_F32, _BF16: HDET_TYPE_BF16}
    lib = C.CDLL(p)
    vp = C.c_void_p
    lib.hdet_workspace_bytes.argtypes = [C.POINTER(hdet_config), C.c_int64, C.POINTER(C.c_size_t),
                                         C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
    lib.hdet_create.argtypes = [C.POINTER(hdet_config), C.POINTER(hdet_buffers), C.POINTER(vp)]
    lib.hdet_warm_init.argtypes = [vp, vp, C.c_double, C.c_uint64]
    lib.hdet_warm_init_noalloc.argtypes = [vp, vp, vp, C.c_int64, C.c_int64, C.c_int32, C.c_double, C.c_uint64, vp]
    lib.hdet_forward_backward.argtypes = [vp, vp, vp, C.POINTER(C.c_float)]
    lib.hdet_fanout_step.argtypes = [vp, vp, C.c_uint32]
    lib.hdet_train_step.argtypes = [vp, vp, vp, C.c_uint32, C.POINTER(C.c_float)]
    lib.hdet_converge.argtypes = [vp]
    lib.hdet_autolr_update.argtypes = [vp, C.POINTER(C.c_double)]
    lib.hdet_get_state.argtypes = [vp, C.POINTER(hdet_state)]
    lib.hdet_set_state.argtypes = [vp, C.POINTER(hdet_state)]
    lib.hdet_set_launch_shape.argtypes = [vp, C.c_int32, C.c_int32]
    lib.hdet_last_error.argtypes = [vp]
    lib.hdet_last_error.restype = C.c_char_p
    lib.hdet_destroy.argtypes = [vp]
    for name, args in (("hdet_rmsnorm", hdet_norm_args), ("hdet_rmsnorm_backward", hdet_norm_grad_args), ("hdet_quantise_rows", hdet_codes_args),
                       ("hdet_restore_rows", hdet_codes_args), ("hdet_quantised_linear", hdet_linear_args),
                       ("hdet_quantised_linear_backward", hdet_linear_grad_args), ("hdet_vocab_loss", hdet_vocab_args)):
        getattr(lib, name).argtypes = [C.POINTER(args), vp]
    size = C.POINTER(C.c_size_t)
    lib.hdet_rmsnorm_backward_workspace.argtypes = [C.c_int32, C.c_int64, C.c_int32, size]
    lib.hdet_quantised_linear_backward_workspace.argtypes = [C.c_int32, C.c_int64, C.c_int32, C.c_int32, size]
    lib.hdet_vocab_loss_workspace.argtypes = [C.c_int32, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_int32, size]
    for name in EXPORTS:
        if name != "hdet_last_error":
            getattr(lib, name).restype = C.c_int
    if path is None:
        _lib = lib
    return lib


def _ptr(x) -> Optional[int]:
    """Device pointer of a torch tensor (or an int / None passed through)."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _check(rc: int, handle=None):
    if rc != HDET_OK:
        msg = load_library().hdet_last_error(handle)
        raise HdetError(rc, msg.decode() if msg else "")


def make_config(**kw) -> hdet_config:
    """hdet_config with the paper's controller constants (beta 0.9, sigma 0.1, lambda 0.5)
    and the usual one-cycle factors as defaults; keyword names are the C field names
    (`lambda_` for lambda; `widths` and `extra` as Python sequences)."""
    cfg = hdet_config()
    cfg.f_div, cfg.f_final, cfg.pct_start = 25.0, 1e4, 0.3
    cfg.beta, cfg.sigma, cfg.lambda_ = 0.9, 0.1, 0.5
    cfg.gamma_override = -1.0
    cfg.momentum, cfg.beta1, cfg.beta2, cfg.eps = 0.9, 0.9, 0.999, 1e-8
    cfg.optimizer, cfg.grad_mode = HDET_ADAMW, HDET_GRAD_PER_REPLICA
    cfg.seed = 7
    widths = kw.pop("widths", None)
    extra = kw.pop("extra", None)
    group_end = kw.pop("group_end", None)
    for key in ("n_params", "batch", "n_blocks", "d_model", "n_heads", "d_ff", "seq_len", "vocab"):
        if key in kw:
            setattr(cfg.dims, key, kw.pop(key))
    if widths is not None:
        cfg.dims.n_layers = len(widths) - 1
        for i, wd in enumerate(widths):
            cfg.dims.widths[i] = wd
    if group_end is not None:
        cfg.n_groups = len(group_end)
        for g, end in enumerate(group_end):
            cfg.group_end[g] = end
    if extra is not None:
        cfg.n_extra_channels = len(extra)
        for j, ch in enumerate(extra):
            kind, base, alpha, lam, lo, hi = ch
            cfg.extra[j].kind, cfg.extra[j].base, cfg.extra[j].alpha = kind, base, alpha
            cfg.extra[j].lambda_, cfg.extra[j].lo, cfg.extra[j].hi = lam, lo, hi
    for key, val in kw.items():
        if not hasattr(cfg, key):
            raise TypeError(f"unknown hdet_config field {key}")
        setattr(cfg, key, val)
    return cfg


def hdet_workspace_bytes(cfg: hdet_config, plane_stride: int):
    a, b, c = C.c_size_t(), C.c_size_t(), C.c_size_t()
    _check(load_library().hdet_workspace_bytes(C.byref(cfg), plane_stride, C.byref(a), C.byref(b),
                                               C.byref(c)))
    return a.value, b.value, c.value


def hdet_create(cfg: hdet_config, params, opt_m, opt_v=None, grads=None, params_bf16=None,
                workspace=None, plane_stride: Optional[int] = None):
    """Returns an opaque handle.  Tensors are [N, plane_stride] device tensors kept alive by
    the caller for the lifetime of the handle."""
    buf = hdet_buffers()
    buf.params_dev, buf.grads_dev = _ptr(params), _ptr(grads)
    buf.opt_m_dev, buf.opt_v_dev = _ptr(opt_m), _ptr(opt_v)
    buf.params_bf16_dev = _ptr(params_bf16)
    buf.workspace_dev = _ptr(workspace)
    buf.workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    buf.plane_stride = plane_stride if plane_stride is not None else params.stride(0)
    h = C.c_void_p()
    _check(load_library().hdet_create(C.byref(cfg), C.byref(buf), C.byref(h)))
    return h


def hdet_warm_init(h, theta0, nu: float, seed: int):
    _check(load_library().hdet_warm_init(h, _ptr(theta0), nu, seed), h)


def hdet_warm_init_noalloc(theta0, params, params_bf16, n_params: int, plane_stride: int, n_replicas: int,
                           nu: float, seed: int, stream: Optional[int] = None):
    _check(load_library().hdet_warm_init_noalloc(_ptr(theta0), _ptr(params), _ptr(params_bf16), n_params, plane_stride,
                                                 n_replicas, nu, seed, stream))


def hdet_forward_backward(h, x, y, want_losses: bool = False):
    n = HDET_MAX_REPLICAS
    out = (C.c_float * n)() if want_losses else None
    _check(load_library().hdet_forward_backward(h, _ptr(x), _ptr(y), out), h)
    return out


def hdet_fanout_step(h, grads=None, flags: int = 0):
    _check(load_library().hdet_fanout_step(h, _ptr(grads), flags), h)


def hdet_train_step(h, x, y, flags: int = 0, want_losses: bool = False):
    out = (C.c_float * HDET_MAX_REPLICAS)() if want_losses else None
    _check(load_library().hdet_train_step(h, _ptr(x), _ptr(y), flags, out), h)
    return out


def hdet_converge(h):
    _check(load_library().hdet_converge(h), h)


def hdet_autolr_update(h, interval_losses: Optional[Sequence[float]] = None, n_replicas: Optional[int] = None):
    """`interval_losses`: None (the device-accumulated losses) or exactly N values; the C call reads
    N doubles, so the length is checked here against `n_replicas` or, if that is not given, against
    the handle's own count (one state query)."""
    arr = None
    if interval_losses is not None:
        n = n_replicas if n_replicas is not None else hdet_get_state(h).n_replicas
        if len(interval_losses) != n:
            raise ValueError(f"interval_losses has {len(interval_losses)} values, the handle has {n} replicas")
        arr = (C.c_double * n)(*[float(x) for x in interval_losses])
    _check(load_library().hdet_autolr_update(h, arr), h)


def hdet_get_state(h) -> hdet_state:
    st = hdet_state()
    _check(load_library().hdet_get_state(h, C.byref(st)), h)
    return st


def hdet_set_state(h, st: hdet_state):
    _check(load_library().hdet_set_state(h, C.byref(st)), h)


def hdet_set_launch_shape(h, variant: int = 0, blocks: int = 0):
    _check(load_library().hdet_set_launch_shape(h, variant, blocks), h)


def hdet_last_error(h=None) -> str:
    msg = load_library().hdet_last_error(h)
    return msg.decode() if msg else ""


def hdet_destroy(h):
    _check(load_library().hdet_destroy(h))


# ---------------------------------------------------------------------------------------
# Operators of language models.  Matrices are device tensors [N, rows, columns] whose columns are next to each other (any strides
# between rows and replicas); vectors a replica are [N, columns]; row scalars [N, rows] are contiguous.  `stream`: a hipStream_t as
# an integer, None for the default stream.  Tensors are borrowed until the work on that stream is done.
# ---------------------------------------------------------------------------------------
_F32 = _BF16 = _I8 = _I32 = _CODE = None       # torch's types, from load_library on


def _refuse(name, t, shape, dtype, contiguous=False):
    """Says what is wrong with a tensor that is not of this shape and type, on a GPU, with the last dimension's elements next to each other."""
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, {tuple(shape)} is wanted")
    if t.dtype != dtype:
        raise ValueError(f"{name} is {t.dtype}, {dtype} is wanted")
    if not t.is_cuda:
        raise ValueError(f"{name} is on {t.device}: device memory is wanted")
    raise ValueError(f"{name} must be contiguous" if contiguous else f"{name}: the last dimension's elements must be next to each other")


def _dtype_code(name, t) -> int:
    code = _CODE.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} is {t.dtype}: float32 or bfloat16 is wanted")
    return code


# The helpers below return what a field of the C structures is made from: (pointer, row stride, replica stride) of a matrix, a pointer, or a
# pointer and a stride.  (A call of a few microseconds notices every attribute that is asked twice.)
_ABSENT = (None, 0, 0)


def _rows_of(name, t, shape, dtype):
    if t is None:
        return _ABSENT
    s = t.stride()
    if t.shape != shape or t.dtype is not dtype or not t.is_cuda or (s[2] != 1 and shape[2] > 1):
        _refuse(name, t, shape, dtype)
    return (t.data_ptr(), s[1], s[0])


def _codes_of(name, t, shape):
    """int8 codes; the strides of dimensions of size 1 say nothing and are made to fit."""
    if t is None:
        return _ABSENT
    s = t.stride()
    if t.shape != shape or t.dtype is not _I8 or not t.is_cuda or (s[2] != 1 and shape[2] > 1):
        _refuse(name, t, shape, _I8)
    n, rows, width = shape
    wide = (width + 15) // 16 * 16
    row = s[1] if rows > 1 else max(wide, s[1] // 16 * 16)
    rep = s[0] if n > 1 else row * max(rows, 1)
    if width % 16 and n and rows and t.storage_offset() + (n - 1) * rep + (rows - 1) * row + wide > t.untyped_storage().nbytes():
        raise ValueError(f"{name}: rows of codes end with zeros up to a multiple of 16 columns, which this tensor's memory does not hold")
    return (t.data_ptr(), row, rep)


def _vector(name, t, shape):
    """fp32 vectors [N, columns]"""
    if t is None:
        return None, 0
    s = t.stride()
    if t.shape != shape or t.dtype is not _F32 or not t.is_cuda or (s[1] != 1 and shape[1] > 1):
        _refuse(name, t, shape, _F32)
    return t.data_ptr(), s[0] if shape[0] > 1 else max(s[0], shape[1])


def _scalars(name, t, shape, dtype=None):
    """contiguous row scalars"""
    if t is None:
        return None
    dtype = dtype or _F32
    if t.shape != shape or t.dtype is not dtype or not t.is_cuda or not t.is_contiguous():
        _refuse(name, t, shape, dtype, contiguous=True)
    return t.data_ptr()


def _work_of(t):
    """scratch memory: the kernels write as many bytes from its start on as the tensor has"""
    if t is None:
        return None, 0
    if not t.is_cuda or not t.is_contiguous():
        _refuse("workspace", t, t.shape, t.dtype, contiguous=True)
    return t.data_ptr(), t.numel() * t.element_size()


def _size_of(name, *args) -> int:
    n = C.c_size_t()
    _check(getattr(load_library(), name)(*args, C.byref(n)))
    return n.value


def hdet_codes_empty(n_replicas: int, rows: int, width: int, device="cuda"):
    """int8 codes [N, rows, width] in memory whose rows are padded with zeros to a multiple of 16 columns."""
    import torch
    return torch.zeros(n_replicas, rows, (width + 15) // 16 * 16, dtype=torch.int8, device=device)[..., :width]


def hdet_rmsnorm(x, gain, resid=None, total=None, y=None, codes=None, scale=None, rstd=None, eps: float = 1e-5, stream: Optional[int] = None):
    """total = x + resid; y = total / rms(total) * gain; codes and scale: y in 8 bits; rstd = 1 / rms.  Writes those of the four that are given."""
    lib = _lib or load_library()
    shape, dt = x.shape, x.dtype
    n, rows, width = shape
    a = hdet_norm_args(n, _dtype_code("x", x), rows, width, 0, eps, _rows_of("x", x, shape, dt), _rows_of("resid", resid, shape, dt),
                       _rows_of("total", total, shape, dt), _rows_of("y", y, shape, dt), _codes_of("codes", codes, shape),
                       _scalars("scale", scale, (n, rows)), _scalars("rstd", rstd, (n, rows)), *_vector("gain", gain, (n, width)))
    rc = lib.hdet_rmsnorm(C.byref(a), stream)
    if rc:
        _check(rc)


def hdet_rmsnorm_backward_workspace(n_replicas: int, rows: int, width: int) -> int:
    return _size_of("hdet_rmsnorm_backward_workspace", n_replicas, rows, width)


def hdet_rmsnorm_backward(total, gain, rstd, dy, dx, dtotal=None, dgain=None, workspace=None, stream: Optional[int] = None):
    """dx (of x and of resid) and dgain from the gradients at y (dy) and at total (dtotal)."""
    lib = _lib or load_library()
    shape, dt = total.shape, total.dtype
    n, rows, width = shape
    a = hdet_norm_grad_args(n, _dtype_code("total", total), rows, width, 0, _rows_of("total", total, shape, dt), _rows_of("dy", dy, shape, dt),
                            _rows_of("dtotal", dtotal, shape, dt), _rows_of("dx", dx, shape, dt), _scalars("rstd", rstd, (n, rows)),
                            *_vector("gain", gain, (n, width)), *_vector("dgain", dgain, (n, width)), *_work_of(workspace))
    rc = lib.hdet_rmsnorm_backward(C.byref(a), stream)
    if rc:
        _check(rc)


def _codes_args(values, codes, scale):
    shape = values.shape
    n, rows, width = shape
    return C.byref(hdet_codes_args(n, _dtype_code("values", values), rows, width, 0, _rows_of("values", values, shape, values.dtype),
                                   _codes_of("codes", codes, shape), _scalars("scale", scale, (n, rows))))


def hdet_quantise_rows(values, codes, scale, stream: Optional[int] = None):
    """codes, scale <- values, a power of two as each row's scale."""
    lib = _lib or load_library()
    rc = lib.hdet_quantise_rows(_codes_args(values, codes, scale), stream)
    if rc:
        _check(rc)


def hdet_restore_rows(codes, scale, values, stream: Optional[int] = None):
    """values <- codes * scale."""
    lib = _lib or load_library()
    rc = lib.hdet_restore_rows(_codes_args(values, codes, scale), stream)
    if rc:
        _check(rc)


def hdet_quantised_linear(codes, scale, w_codes, w_scale, y, bias=None, stream: Optional[int] = None):
    """y [N, rows, d_out] <- (codes * scale) (w_codes * w_scale)^T + bias."""
    lib = _lib or load_library()
    shape = codes.shape
    n, rows, d_in = shape
    d_out = w_codes.shape[1]
    a = hdet_linear_args(n, _dtype_code("y", y), rows, d_in, d_out, _codes_of("codes", codes, shape), _codes_of("w_codes", w_codes, (n, d_out, d_in)),
                         _scalars("scale", scale, (n, rows)), _scalars("w_scale", w_scale, (n, d_out)), *_vector("bias", bias, (n, d_out)),
                         _rows_of("y", y, (n, rows, d_out), y.dtype))
    rc = lib.hdet_quantised_linear(C.byref(a), stream)
    if rc:
        _check(rc)


def hdet_quantised_linear_backward_workspace(n_replicas: int, rows: int, d_in: int, d_out: int) -> int:
    return _size_of("hdet_quantised_linear_backward_workspace", n_replicas, rows, d_in, d_out)


def hdet_quantised_linear_backward(dy, codes, scale, w_codes, w_scale, dx=None, dw=None, db=None, workspace=None, stream: Optional[int] = None):
    """dx = dy W (bfloat16), dw = dy^T X (fp32), db = the rows' sum of dy (fp32), from the 8-bit copies; those that are given."""
    lib = _lib or load_library()
    shape = dy.shape
    n, rows, d_out = shape
    d_in = codes.shape[2]
    a = hdet_linear_grad_args(n, 0, rows, d_in, d_out, _rows_of("dy", dy, shape, _BF16), _codes_of("codes", codes, (n, rows, d_in)),
                              _codes_of("w_codes", w_codes, (n, d_out, d_in)), _scalars("scale", scale, (n, rows)), _scalars("w_scale", w_scale, (n, d_out)),
                              _rows_of("dx", dx, (n, rows, d_in), _BF16), _rows_of("dw", dw, (n, d_out, d_in), _F32),
                              *_vector("db", db, (n, d_out)), *_work_of(workspace))
    rc = lib.hdet_quantised_linear_backward(C.byref(a), stream)
    if rc:
        _check(rc)


def hdet_vocab_loss_workspace(n_replicas: int, rows: int, width: int, classes: int, dw=None, piece: int = 0) -> int:
    """`dw`: the dtype of the weight gradient, HDET_VOCAB_NO_DW for calls without one or HDET_VOCAB_LOSSES for the losses alone; None: float32.  What is enough with a dw of
    either type is enough without."""
    load_library()
    kind = dw if isinstance(dw, int) else _CODE.get(_F32 if dw is None else dw)
    if kind is None:
        raise ValueError(f"dw is {dw}: float32 or bfloat16 is wanted")
    return _size_of("hdet_vocab_loss_workspace", n_replicas, rows, width, classes, kind, piece)


def hdet_vocab_loss(h, w, labels, row_loss, mean_loss, dh=None, dw=None, bias=None, db=None, piece: int = 0, workspace=None,
                    stream: Optional[int] = None):
    """Cross-entropy of softmax(h w^T + bias) at `labels` (int32 [N, rows]; rows whose label is no class do not count), and its gradients."""
    lib = _lib or load_library()
    shape = h.shape
    n, rows, width = shape
    classes = w.shape[1]
    wide = (n, classes, width)
    a = hdet_vocab_args(n, 0 if dw is None else _dtype_code("dw", dw), rows, width, classes, piece, 0, _rows_of("h", h, shape, _BF16),
                        _rows_of("w", w, wide, _BF16), *_vector("bias", bias, (n, classes)), _scalars("labels", labels, (n, rows), _I32),
                        _scalars("row_loss", row_loss, (n, rows)), _scalars("mean_loss", mean_loss, (n,)), _rows_of("dh", dh, shape, _BF16),
                        _ABSENT if dw is None else _rows_of("dw", dw, wide, dw.dtype), *_vector("db", db, (n, classes)), *_work_of(workspace))
    rc = lib.hdet_vocab_loss(C.byref(a), stream)
    if rc:
        _check(rc)
