"""Binding of the operators around a gated linear recurrent layer (include/mgrit_ops.h): argument
marshalling only, as in binding.py, whose rules hold here too.

Sequences (gate, value, h and their gradients) are tensors [T,B,H] of any strides whose last one is 1:
halves of a product's rows, or batch-first storage as ``x.transpose(0, 1)``.  Rows of logits, x and y are
matrices whose last stride is 1.
"""
from __future__ import annotations

import ctypes

from .binding import MGRIT_BF16, MGRIT_F32, _Arg, _check, _marshal, _stream, lib as _base_lib

MGRIT_F16 = 4                             # dtype of the configurations below, beside MGRIT_F32 and MGRIT_BF16
GLR_MIX, GLR_DECAY = 0, 1
LOGPROBS_MAX_K, DISTILL_MAX_K = 64, 256
_ready = None


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
    """Mirror of ``logits_cfg``; the row strides are filled in from the tensors of a call."""

    _fields_ = (_fields(ctypes.c_int32, ("N", "V", "K", "dtype")) + [("temperature", ctypes.c_float)]
                + _fields(ctypes.c_int64, ("ld", "ld_grad")))

    def __init__(self, N, V, K, dtype=MGRIT_F32, temperature=1.0):
        super().__init__(N, V, K, dtype, temperature, V, V)


class Q8Cfg(ctypes.Structure):
    """Mirror of ``q8_cfg``; the row strides are filled in from the tensors of a call."""

    _fields_ = _fields(ctypes.c_int32, ("M", "N", "K", "dtype")) + _fields(ctypes.c_int64, ("ldx", "ldy"))

    def __init__(self, M, N, K, dtype=MGRIT_F32):
        super().__init__(M, N, K, dtype, K, N)


def _lib() -> ctypes.CDLL:
    global _ready
    if _ready is None:
        L, vp, sz, i32 = _base_lib(), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
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
        _ready = L
    return _ready


def _size(name, cfg) -> int:
    n = ctypes.c_size_t(0)
    _check(getattr(_lib(), name)(ctypes.byref(cfg), ctypes.byref(n)), name)
    return int(n.value)


def _dtype(cfg):
    import torch
    return {MGRIT_F32: torch.float32, MGRIT_BF16: torch.bfloat16, MGRIT_F16: torch.float16}.get(cfg.dtype)


class _Strided(_Arg):
    """A tensor argument of the configuration's dtype whose last stride is 1."""


def _call(name, cfg, *args) -> None:
    """Like binding._call; sequences go as pointers to ``GlrSeq``, matrices as their data pointers."""
    import torch
    plain = [a for a in args if isinstance(a, _Arg) and not isinstance(a, _Strided)]
    strided = [a for a in args if isinstance(a, _Strided) and a.t is not None]
    for a in strided:
        if not isinstance(a.t, torch.Tensor):
            raise TypeError(f"{a.name}: expected a CUDA tensor")
        if tuple(a.t.shape) != tuple(a.shape):
            raise ValueError(f"{a.name}: expected shape {tuple(a.shape)}, got {tuple(a.t.shape)}")
    pointers = dict(zip(map(id, plain), _marshal(plain)))
    for a in strided:
        if a.dtype is not None and a.t.dtype != a.dtype:
            raise TypeError(f"{a.name}: expected dtype {a.dtype}, got {a.t.dtype}")
        if a.t.shape[-1] > 1 and a.t.stride(-1) != 1:
            raise ValueError(f"{a.name}: the last dimension must be contiguous")
        if not a.t.is_cuda:
            raise TypeError(f"{a.name}: expected a CUDA tensor")
        if a.t.dim() == 3:
            pointers[id(a)] = ctypes.byref(GlrSeq(a.t.data_ptr(), a.t.stride(0), a.t.stride(1)))
        else:
            pointers[id(a)] = a.t.data_ptr()
    out = [pointers.get(id(a)) if isinstance(a, _Arg) else a for a in args]
    _check(getattr(_lib(), name)(ctypes.byref(cfg), *out, _stream()), name)


def _bytes_of(t, name):
    """A workspace tensor and its size in bytes (the library compares the size with cfg)."""
    return _Arg(t, name), ctypes.c_size_t(0 if t is None else t.numel() * t.element_size())


def _f32(t, name, *shape):
    import torch
    return _Arg(t, name, torch.float32, shape)


# ---- gated linear recurrence
def glr_workspace_bytes(cfg: GlrCfg) -> int:
    return _size("glr_workspace_bytes", cfg)


def glr_saved_bytes(cfg: GlrCfg) -> int:
    return _size("glr_saved_bytes", cfg)


def _seq(cfg, t, name):
    return _Strided(t, name, _dtype(cfg), (cfg.T, cfg.B, cfg.H))


def _reset(cfg, t, *shape):
    import torch
    return _Arg(t, "reset", torch.uint8, shape)


def glr_forward(cfg, gate, value, h0, reset, h, h_last, saved, workspace) -> None:
    T, B, H = cfg.T, cfg.B, cfg.H
    _call("glr_forward", cfg, _seq(cfg, gate, "gate"), _seq(cfg, value, "value"), _f32(h0, "h0", B, H),
          _reset(cfg, reset, T, B), _seq(cfg, h, "h"), _f32(h_last, "h_last", B, H), *_bytes_of(saved, "saved"),
          *_bytes_of(workspace, "workspace"))


def glr_backward(cfg, gate, value, reset, saved, dh, dh_last, dgate, dvalue, dh0, workspace) -> None:
    T, B, H = cfg.T, cfg.B, cfg.H
    _call("glr_backward", cfg, _seq(cfg, gate, "gate"), _seq(cfg, value, "value"), _reset(cfg, reset, T, B),
          *_bytes_of(saved, "saved"), _seq(cfg, dh, "dh"), _f32(dh_last, "dh_last", B, H),
          _seq(cfg, dgate, "dgate"), _seq(cfg, dvalue, "dvalue"), _f32(dh0, "dh0", B, H),
          *_bytes_of(workspace, "workspace"))


def glr_step(cfg, gate, value, slots, reset, state_in, state_out, h) -> None:
    """gate, value, h: [B,H]; state_in, state_out: [n_slots,H]."""
    import torch
    B, H = cfg.B, cfg.H
    for t, name in ((gate, "gate"), (value, "value"), (h, "h"), (state_in, "state_in"), (state_out, "state_out")):
        if isinstance(t, torch.Tensor) and t.dim() != 2:
            raise ValueError(f"{name}: expected two dimensions, got shape {tuple(t.shape)}")
    one = lambda t: t[None] if isinstance(t, torch.Tensor) else t  # noqa: E731
    n = state_in.shape[0] if isinstance(state_in, torch.Tensor) else 0
    _call("glr_step", cfg, _seq(cfg, one(gate), "gate"), _seq(cfg, one(value), "value"),
          _Arg(slots, "slots", torch.int32, (B,)), ctypes.c_int32(n), _reset(cfg, reset, B),
          _f32(state_in, "state_in", n, H), _f32(state_out, "state_out", n, H), _seq(cfg, one(h), "h"))


# ---- rows of logits
def logits_workspace_bytes(cfg: LogitsCfg) -> int:
    return _size("logits_workspace_bytes", cfg)


def _matrix(cfg, t, name, rows, cols):
    return _Strided(t, name, _dtype(cfg), (rows, cols))


def _ld(t, cols):
    """Row stride of a matrix (one row: its width, whatever the tensor says)."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dim() != 2 or t.shape[0] == 1:
        return cols
    return t.stride(0)


def _with_strides(cfg, **strides):
    c = type(cfg).from_buffer_copy(cfg)
    for k, v in strides.items():
        setattr(c, k, v)
    return c


def _i64(t, name, *shape):
    import torch
    return _Arg(t, name, torch.int64, shape)


def token_logprobs(cfg, logits, tokens, logp, entropy, top_logp, top_ids, workspace) -> None:
    N, V, K = cfg.N, cfg.V, cfg.K
    c = _with_strides(cfg, ld=_ld(logits, V))
    _call("token_logprobs", c, _matrix(cfg, logits, "logits", N, V), _i64(tokens, "tokens", N),
          _f32(logp, "logp", N), _f32(entropy, "entropy", N), _f32(top_logp, "top_logp", N, K),
          _i64(top_ids, "top_ids", N, K), *_bytes_of(workspace, "workspace"))


def distill_topk(cfg, logits, ids, teacher, weight, loss, stats, dlogits, workspace) -> None:
    N, V, K = cfg.N, cfg.V, cfg.K
    c = _with_strides(cfg, ld=_ld(logits, V), ld_grad=_ld(dlogits, V))
    _call("distill_topk", c, _matrix(cfg, logits, "logits", N, V), _i64(ids, "ids", N, K),
          _f32(teacher, "teacher", N, K), _f32(weight, "weight", N), _f32(loss, "loss", N),
          _f32(stats, "stats", N, 2), _matrix(cfg, dlogits, "dlogits", N, V), *_bytes_of(workspace, "workspace"))


def distill_topk_backward(cfg, logits, ids, teacher, stats, dloss, dlogits) -> None:
    N, V, K = cfg.N, cfg.V, cfg.K
    c = _with_strides(cfg, ld=_ld(logits, V), ld_grad=_ld(dlogits, V))
    _call("distill_topk_backward", c, _matrix(cfg, logits, "logits", N, V), _i64(ids, "ids", N, K),
          _f32(teacher, "teacher", N, K), _f32(stats, "stats", N, 2), _f32(dloss, "dloss", N),
          _matrix(cfg, dlogits, "dlogits", N, V))


# ---- product in 8-bit integers
def q8_row_bytes(K: int) -> int:
    return int(_lib().q8_row_bytes(int(K)))


def q8_workspace_bytes(cfg: Q8Cfg) -> int:
    return _size("q8_workspace_bytes", cfg)


def q8_quantize(cfg, x, q, scale) -> None:
    """Rows x[M,K] -> q[M, q8_row_bytes(K)] int8, scale[M]."""
    import torch
    M, K = cfg.M, cfg.K
    c = _with_strides(cfg, ldx=_ld(x, K))
    _call("q8_quantize", c, _matrix(cfg, x, "x", M, K), _Arg(q, "q", torch.int8, (M, q8_row_bytes(K))),
          _f32(scale, "scale", M))


def q8_linear(cfg, x, w_q, w_scale, bias, y, workspace) -> None:
    import torch
    M, N, K = cfg.M, cfg.N, cfg.K
    c = _with_strides(cfg, ldx=_ld(x, K), ldy=_ld(y, N))
    _call("q8_linear", c, _matrix(cfg, x, "x", M, K), _Arg(w_q, "w_q", torch.int8, (N, q8_row_bytes(K))),
          _f32(w_scale, "w_scale", N), _f32(bias, "bias", N), _matrix(cfg, y, "y", M, N),
          *_bytes_of(workspace, "workspace"))
