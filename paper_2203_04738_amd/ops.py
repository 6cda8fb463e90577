"""Binding of the operators around a gated linear recurrent layer (include/mgrit_ops.h): argument
marshalling only, as in binding.py, whose rules hold here too.

Sequences (gate, value, h and their gradients) are tensors [T,B,H] of any strides whose last one is 1:
halves of a product's rows, or batch-first storage as ``x.transpose(0, 1)``.  Rows of logits, x and y are
matrices whose last stride is 1.
"""
from __future__ import annotations

import ctypes

from .binding import MGRIT_BF16, MGRIT_F32, _check, lib as _base_lib

MGRIT_F16 = 4                             # dtype of the configurations below, beside MGRIT_F32 and MGRIT_BF16
GLR_MIX, GLR_DECAY = 0, 1
LOGPROBS_MAX_K, DISTILL_MAX_K = 64, 256
_ready = _torch = _TYPES = None


def _fields(c_type, names):
    return [(n, c_type) for n in names]


class GlrCfg(ctypes.Structure):
    """Mirror of ``glr_cfg``."""

    _fields_ = _fields(ctypes.c_int32, ("T", "B", "H", "form", "dtype"))

    def __init__(self, T, B, H, form=GLR_MIX, dtype=MGRIT_F32):
        super().__init__(T, B, H, form, dtype)


class GlrSeq(ctypes.Structure):
    """Mirror of ``glr_seq``."""

    _fields_ = [("data", ctypes.c_void_p)] + _fields(ctypes.c_int64, ("stride_t", "stride_b"))


class LogitsCfg(ctypes.Structure):
    """Mirror of ``logits_cfg``; a call passes the row strides of its tensors, in a copy."""

    _fields_ = (_fields(ctypes.c_int32, ("N", "V", "K", "dtype")) + [("temperature", ctypes.c_float)]
                + _fields(ctypes.c_int64, ("ld", "ld_grad")))

    def __init__(self, N, V, K, dtype=MGRIT_F32, temperature=1.0):
        super().__init__(N, V, K, dtype, temperature, V, V)


class Q8Cfg(ctypes.Structure):
    """Mirror of ``q8_cfg``; a call passes the row strides of its tensors, in a copy."""

    _fields_ = _fields(ctypes.c_int32, ("M", "N", "K", "dtype")) + _fields(ctypes.c_int64, ("ldx", "ldy"))

    def __init__(self, M, N, K, dtype=MGRIT_F32):
        super().__init__(M, N, K, dtype, K, N)


def _prototypes(L):
    """Argument types of the entry points in the library L."""
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    szp = ctypes.POINTER(sz)
    for name, cfg, args in (
            ("glr_workspace_bytes", GlrCfg, [szp]), ("glr_saved_bytes", GlrCfg, [szp]),
            ("glr_forward", GlrCfg, [vp] * 7 + [sz, vp, sz, vp]),
            ("glr_backward", GlrCfg, [vp] * 4 + [sz] + [vp] * 6 + [sz, vp]),
            ("glr_step", GlrCfg, [vp] * 3 + [i32] + [vp] * 5),
            ("logits_workspace_bytes", LogitsCfg, [szp]),
            ("token_logprobs", LogitsCfg, [vp] * 7 + [sz, vp]),
            ("distill_topk", LogitsCfg, [vp] * 8 + [sz, vp]),
            ("distill_topk_backward", LogitsCfg, [vp] * 7),
            ("q8_workspace_bytes", Q8Cfg, [szp]), ("q8_quantize", Q8Cfg, [vp] * 4),
            ("q8_linear", Q8Cfg, [vp] * 6 + [sz, vp])):
        fn = getattr(L, name)
        fn.argtypes = [ctypes.POINTER(cfg)] + args
        fn.restype = ctypes.c_int
    L.q8_row_bytes.argtypes = [i32]
    L.q8_row_bytes.restype = ctypes.c_int64
    return L


def _lib() -> ctypes.CDLL:
    global _ready, _torch, _TYPES
    if _ready is None:
        import torch
        _torch = torch
        _TYPES = {MGRIT_F32: torch.float32, MGRIT_BF16: torch.bfloat16, MGRIT_F16: torch.float16}
        _ready = _prototypes(_base_lib())
    return _ready


def _stream() -> int:
    """The current stream of the current device, as torch.cuda.current_stream().cuda_stream says."""
    return _torch._C._cuda_getCurrentRawStream(_torch._C._cuda_getDevice())


def _size(name, cfg) -> int:
    n = ctypes.c_size_t(0)
    _check(getattr(_lib(), name)(ctypes.byref(cfg), ctypes.byref(n)), name)
    return int(n.value)


# An argument is a plain value or (tensor, name, dtype, shape, kind): shape None: any; kind _DENSE:
# contiguous; _ROWS: the last stride is 1; _SEQ: the same, [T,B,H], passed as a pointer to a ``GlrSeq``;
# _STEP: the same, [B,H].
_DENSE, _ROWS, _SEQ, _STEP = 0, 1, 2, 3


def _unit_rows(t):
    return t.shape[-1] == 1 or t.stride(-1) == 1


def _explain(args):
    """Raises for the first argument that does not fit: all sizes first, then types, layouts and devices (as
    binding._marshal does).  Returns where every argument fits."""
    tensors = [a for a in args if type(a) is tuple and a[0] is not None]
    for t, name, _, shape, _ in tensors:
        if not isinstance(t, _torch.Tensor):
            raise TypeError(f"{name}: expected a CUDA tensor")
        if shape is not None and tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    for t, name, dtype, _, kind in tensors:
        if dtype is not None and t.dtype != dtype:
            raise TypeError(f"{name}: expected dtype {dtype}, got {t.dtype}")
        if kind == _DENSE and not t.is_contiguous():
            raise ValueError(f"{name}: tensor must be contiguous")
        if kind != _DENSE and not _unit_rows(t):
            raise ValueError(f"{name}: the last dimension must be contiguous")
        if not t.is_cuda:
            raise TypeError(f"{name}: expected a CUDA tensor")


def _call(name, cfg, *args) -> None:
    """Checks and marshals the arguments, then calls entry point `name` on the current stream.  (A call of a few
    microseconds' work is as long as this: one pass over the arguments, the reasons only where one does not fit.)"""
    L, tensor, out = _lib(), _torch.Tensor, []
    for a in args:
        if type(a) is not tuple:
            out.append(a)
            continue
        t, _, dtype, shape, kind = a
        if t is None:
            out.append(None)
            continue
        if not (isinstance(t, tensor) and (shape is None or t.shape == shape) and (dtype is None or t.dtype is dtype)
                and t.is_cuda and (t.is_contiguous() if kind == 0 else _unit_rows(t))):
            _explain(args)
            raise AssertionError(a[1])                # (not reached: _explain says what is wrong)
        if kind < 2:
            out.append(t.data_ptr())
        else:
            strides = t.stride()
            out.append(ctypes.byref(GlrSeq(t.data_ptr(), strides[0] if kind == 2 else 0, strides[-2])))
    rc = getattr(L, name)(ctypes.byref(cfg), *out, _stream())
    if rc:
        _check(rc, name)


def _bytes_of(t, name):
    """A workspace tensor and its size in bytes (the library compares the size with cfg)."""
    return (t, name, None, None, _DENSE), 0 if t is None else t.numel() * t.element_size()


def _dtype(cfg):
    _lib()
    return _TYPES.get(cfg.dtype)


def _f32(t, name, *shape):
    return t, name, _torch.float32, shape, _DENSE


# ---- gated linear recurrence
def glr_workspace_bytes(cfg: GlrCfg) -> int:
    return _size("glr_workspace_bytes", cfg)


def glr_saved_bytes(cfg: GlrCfg) -> int:
    return _size("glr_saved_bytes", cfg)


def _seq(cfg, t, name):
    return t, name, _dtype(cfg), (cfg.T, cfg.B, cfg.H), _SEQ


def _reset(t, *shape):
    return t, "reset", _torch.uint8, shape, _DENSE


def glr_forward(cfg, gate, value, h0, reset, h, h_last, saved, workspace) -> None:
    T, B, H = cfg.T, cfg.B, cfg.H
    _call("glr_forward", cfg, _seq(cfg, gate, "gate"), _seq(cfg, value, "value"), _f32(h0, "h0", B, H),
          _reset(reset, T, B), _seq(cfg, h, "h"), _f32(h_last, "h_last", B, H), *_bytes_of(saved, "saved"),
          *_bytes_of(workspace, "workspace"))


def glr_backward(cfg, gate, value, reset, saved, dh, dh_last, dgate, dvalue, dh0, workspace) -> None:
    T, B, H = cfg.T, cfg.B, cfg.H
    _call("glr_backward", cfg, _seq(cfg, gate, "gate"), _seq(cfg, value, "value"), _reset(reset, T, B),
          *_bytes_of(saved, "saved"), _seq(cfg, dh, "dh"), _f32(dh_last, "dh_last", B, H),
          _seq(cfg, dgate, "dgate"), _seq(cfg, dvalue, "dvalue"), _f32(dh0, "dh0", B, H),
          *_bytes_of(workspace, "workspace"))


def glr_step(cfg, gate, value, slots, reset, state_in, state_out, h) -> None:
    """gate, value, h: [B,H]; state_in, state_out: [n_slots,H]."""
    B, H, dtype = cfg.B, cfg.H, _dtype(cfg)
    n = state_in.shape[0] if isinstance(state_in, _torch.Tensor) and state_in.dim() == 2 else 0
    _call("glr_step", cfg, (gate, "gate", dtype, (B, H), _STEP), (value, "value", dtype, (B, H), _STEP),
          (slots, "slots", _torch.int32, (B,), _DENSE), n, _reset(reset, B), _f32(state_in, "state_in", n, H),
          _f32(state_out, "state_out", n, H), (h, "h", dtype, (B, H), _STEP))


# ---- rows of logits
def logits_workspace_bytes(cfg: LogitsCfg) -> int:
    return _size("logits_workspace_bytes", cfg)


def _matrix(cfg, t, name, rows, cols):
    return t, name, _dtype(cfg), (rows, cols), _ROWS


def _ld(t, cols):
    """Row stride of a matrix (one row: its width, whatever the tensor says)."""
    _lib()
    if not isinstance(t, _torch.Tensor) or t.dim() != 2 or t.shape[0] == 1:
        return cols
    return t.stride(0)


def _strided(cfg, **strides):
    """A copy of a configuration with the row strides of a call: the caller's own may be in another thread's call."""
    c = type(cfg).from_buffer_copy(cfg)
    for name, ld in strides.items():
        setattr(c, name, ld)
    return c


def _i64(t, name, *shape):
    return t, name, _torch.int64, shape, _DENSE


def token_logprobs(cfg, logits, tokens, logp, entropy, top_logp, top_ids, workspace) -> None:
    N, V, K = cfg.N, cfg.V, cfg.K
    cfg = _strided(cfg, ld=_ld(logits, V))
    _call("token_logprobs", cfg, _matrix(cfg, logits, "logits", N, V), _i64(tokens, "tokens", N),
          _f32(logp, "logp", N), _f32(entropy, "entropy", N), _f32(top_logp, "top_logp", N, K),
          _i64(top_ids, "top_ids", N, K), *_bytes_of(workspace, "workspace"))


def distill_topk(cfg, logits, ids, teacher, weight, loss, stats, dlogits, workspace) -> None:
    N, V, K = cfg.N, cfg.V, cfg.K
    cfg = _strided(cfg, ld=_ld(logits, V), ld_grad=_ld(dlogits, V))
    _call("distill_topk", cfg, _matrix(cfg, logits, "logits", N, V), _i64(ids, "ids", N, K),
          _f32(teacher, "teacher", N, K), _f32(weight, "weight", N), _f32(loss, "loss", N),
          _f32(stats, "stats", N, 2), _matrix(cfg, dlogits, "dlogits", N, V), *_bytes_of(workspace, "workspace"))


def distill_topk_backward(cfg, logits, ids, teacher, stats, dloss, dlogits) -> None:
    N, V, K = cfg.N, cfg.V, cfg.K
    cfg = _strided(cfg, ld=_ld(logits, V), ld_grad=_ld(dlogits, V))
    _call("distill_topk_backward", cfg, _matrix(cfg, logits, "logits", N, V), _i64(ids, "ids", N, K),
          _f32(teacher, "teacher", N, K), _f32(stats, "stats", N, 2), _f32(dloss, "dloss", N),
          _matrix(cfg, dlogits, "dlogits", N, V))


# ---- product in 8-bit integers
def q8_row_bytes(K: int) -> int:
    return (int(K) + 127) // 128 * 128


def q8_workspace_bytes(cfg: Q8Cfg) -> int:
    return _size("q8_workspace_bytes", cfg)


def q8_quantize(cfg, x, q, scale) -> None:
    """Rows x[M,K] -> q[M, q8_row_bytes(K)] int8, scale[M]."""
    M, K = cfg.M, cfg.K
    cfg = _strided(cfg, ldx=_ld(x, K))
    _call("q8_quantize", cfg, _matrix(cfg, x, "x", M, K), (q, "q", _torch.int8, (M, q8_row_bytes(K)), _DENSE),
          _f32(scale, "scale", M))


def q8_linear(cfg, x, w_q, w_scale, bias, y, workspace) -> None:
    M, N, K = cfg.M, cfg.N, cfg.K
    cfg = _strided(cfg, ldx=_ld(x, K), ldy=_ld(y, N))
    _call("q8_linear", cfg, _matrix(cfg, x, "x", M, K), (w_q, "w_q", _torch.int8, (N, q8_row_bytes(K)), _DENSE),
          _f32(w_scale, "w_scale", N), _f32(bias, "bias", N), _matrix(cfg, y, "y", M, N),
          *_bytes_of(workspace, "workspace"))
