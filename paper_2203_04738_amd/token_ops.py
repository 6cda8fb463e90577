"""Binding of the operators of a recurrent student over tokens (include/mgrit_tokens.h): argument marshalling only, as in
ops.py, whose rules hold here too.

Sequences are tensors [T,B,H] (b and c of the scan: [T,B,S]) of any strides whose last one is 1; rows of tables, logits
and embeddings are matrices whose last stride is 1.  All tensors of a call are on the current device, and the work is
enqueued on its current stream.
"""
from __future__ import annotations

import ctypes
import struct

from . import ops as _o
from .binding import MGRIT_F32, _check
from .ops import GlrSeq, _DENSE, _SEQ, _STEP, _bytes_of, _dtype, _f32, _fields, _i64, _ld, _matrix, _reset, _strided

CONV_LINEAR, CONV_SILU = 0, 1
CONV_MAX_W, SSM_MAX_S = 8, 64
_ready = None


class EmbedCfg(ctypes.Structure):
    """Mirror of ``embed_cfg``; a call passes the row strides of its tensors, in a copy."""

    _fields_ = (_fields(ctypes.c_int32, ("N", "V", "D", "dtype")) + [("scale", ctypes.c_float)]
                + _fields(ctypes.c_int64, ("ld_table", "ld_out")))

    def __init__(self, N, V, D, dtype=MGRIT_F32, scale=1.0):
        super().__init__(N, V, D, dtype, scale, D, D)


class ConvCfg(ctypes.Structure):
    """Mirror of ``conv_cfg``."""

    _fields_ = _fields(ctypes.c_int32, ("T", "B", "H", "W", "act", "dtype"))

    def __init__(self, T, B, H, W, act=CONV_SILU, dtype=MGRIT_F32):
        super().__init__(T, B, H, W, act, dtype)


class SsmCfg(ctypes.Structure):
    """Mirror of ``ssm_cfg``."""

    _fields_ = _fields(ctypes.c_int32, ("T", "B", "H", "S", "dtype"))

    def __init__(self, T, B, H, S, dtype=MGRIT_F32):
        super().__init__(T, B, H, S, dtype)


class SsmInputs(ctypes.Structure):
    """Mirror of ``ssm_inputs``."""

    _fields_ = ([(n, GlrSeq) for n in ("x", "dt", "b", "c", "z")]
                + _fields(ctypes.c_void_p, ("a", "skip", "bias")))


class SsmGrads(ctypes.Structure):
    """Mirror of ``ssm_grads``."""

    _fields_ = ([(n, GlrSeq) for n in ("dx", "ddt", "db", "dc", "dz")]
                + _fields(ctypes.c_void_p, ("da", "dskip", "dbias", "dh0")))


class PolicyCfg(ctypes.Structure):
    """Mirror of ``policy_cfg``."""

    _fields_ = _fields(ctypes.c_float, ("clip_low", "clip_high", "kl"))

    def __init__(self, clip_low=0.2, clip_high=0.2, kl=0.0):
        super().__init__(clip_low, clip_high, kl)


def _prototypes(L):
    """Argument types of the entry points in the library L."""
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    szp = ctypes.POINTER(sz)
    for name, cfg, args in (
            ("embed_lookup", EmbedCfg, [vp] * 4), ("embed_workspace_bytes", EmbedCfg, [szp]),
            ("embed_backward", EmbedCfg, [vp] * 4 + [sz, vp]),
            ("causal_conv_forward", ConvCfg, [vp] * 8), ("causal_conv_workspace_bytes", ConvCfg, [szp]),
            ("causal_conv_backward", ConvCfg, [vp] * 12 + [sz, vp]),
            ("causal_conv_step", ConvCfg, [vp] * 4 + [i32] + [vp] * 5),
            ("ssm_workspace_bytes", SsmCfg, [szp]), ("ssm_saved_bytes", SsmCfg, [szp]),
            ("ssm_forward", SsmCfg, [vp] * 6 + [sz, vp, sz, vp]),
            ("ssm_backward", SsmCfg, [vp] * 3 + [sz] + [vp] * 4 + [sz, vp]),
            ("ssm_step", SsmCfg, [vp] * 2 + [i32] + [vp] * 5),
            ("policy_workspace_bytes", _o.LogitsCfg, [szp]),
            ("policy_loss", _o.LogitsCfg, [vp] * 14 + [sz, vp]),
            ("policy_loss_backward", _o.LogitsCfg, [vp] * 10)):
        fn = getattr(L, name)
        fn.argtypes = [ctypes.POINTER(cfg)] + args
        fn.restype = ctypes.c_int
    return L


def _lib() -> ctypes.CDLL:
    global _ready
    if _ready is None:
        _ready = _prototypes(_o._lib())
    return _ready


def _size(name, cfg) -> int:
    n = ctypes.c_size_t(0)
    _check(getattr(_lib(), name)(ctypes.byref(cfg), ctypes.byref(n)), name)
    return int(n.value)


class _Group(tuple):
    """Arguments that one C structure holds, sequences and pointers: a tuple of them."""


_SEQS = {n: struct.Struct(f"{n}q") for n in range(1, 24)}
_NULL, _NO_SEQ = (0,), (0, 0, 0)


def _explain(args, device):
    flat = [b for a in args for b in (a if type(a) is _Group else (a,))]
    _o._explain(flat)
    for a in flat:
        if type(a) is tuple and a[0] is not None and a[0].get_device() != device:
            raise ValueError(f"{a[1]}: tensor on cuda:{a[0].get_device()}, the current device is cuda:{device}")


def _call(name, cfg, *args) -> None:
    """Checks and marshals the arguments, then calls entry point `name` on the current stream (ops._call, with
    structures of arguments, and all tensors on the current device)."""
    L, torch = _lib(), _o._torch
    tensor, device = torch.Tensor, torch._C._cuda_getDevice() if torch.cuda.is_initialized() else -2
    out = []
    for a in args:
        kind = type(a)
        if kind is tuple:
            group = (a,)
        elif kind is _Group:
            group = a
        else:
            out.append(ctypes.byref(a) if isinstance(a, ctypes.Structure) else a)
            continue
        words = []
        for t, _, dtype, shape, layout in group:
            if t is None:
                words += _NO_SEQ if layout >= _SEQ and kind is _Group else _NULL
                continue
            if not (isinstance(t, tensor) and (shape is None or t.shape == shape) and (dtype is None or t.dtype is dtype)
                    and t.get_device() == device):
                _refuse(args, device)
            if layout == _DENSE:
                if not t.is_contiguous():
                    _refuse(args, device)
                words.append(t.data_ptr())
                continue
            strides = t.stride()
            if strides[-1] != 1 and t.shape[-1] != 1:
                _refuse(args, device)
            if layout >= _SEQ:
                words += (t.data_ptr(), strides[0] if layout == _SEQ else 0, strides[-2])
            else:
                words.append(t.data_ptr())
        n = len(words)
        out.append(_SEQS[n].pack(*words) if n > 1 else words[0] or None)
    rc = getattr(L, name)(ctypes.byref(cfg), *out, _o._stream())
    if rc:
        _check(rc, name)


def _refuse(args, device):
    _explain(args, device)
    raise AssertionError("an argument that fits was refused")


# ---- embedding
def embed_workspace_bytes(cfg: EmbedCfg) -> int:
    return _size("embed_workspace_bytes", cfg)


def embed_lookup(cfg, tokens, table, out) -> None:
    N, V, D = cfg.N, cfg.V, cfg.D
    cfg = _strided(cfg, ld_table=_ld(table, D), ld_out=_ld(out, D))
    _call("embed_lookup", cfg, _i64(tokens, "tokens", N), _matrix(cfg, table, "table", V, D),
          _matrix(cfg, out, "out", N, D))


def embed_backward(cfg, tokens, dout, dtable, workspace) -> None:
    N, V, D = cfg.N, cfg.V, cfg.D
    cfg = _strided(cfg, ld_table=_ld(dtable, D), ld_out=_ld(dout, D))
    _call("embed_backward", cfg, _i64(tokens, "tokens", N), _matrix(cfg, dout, "dout", N, D),
          _matrix(cfg, dtable, "dtable", V, D), *_bytes_of(workspace, "workspace"))


# ---- causal convolution
def causal_conv_workspace_bytes(cfg: ConvCfg) -> int:
    return _size("causal_conv_workspace_bytes", cfg)


def _seq(cfg, t, name):
    return t, name, _dtype(cfg), (cfg.T, cfg.B, cfg.H), _SEQ


def _row(cfg, t, name):
    return t, name, _dtype(cfg), (cfg.B, cfg.H), _STEP


def _taps(cfg, weight, bias):
    return _f32(weight, "weight", cfg.H, cfg.W), _f32(bias, "bias", cfg.H)


def causal_conv_forward(cfg, x, weight, bias, past, reset, y, last) -> None:
    T, B, H, W = cfg.T, cfg.B, cfg.H, cfg.W
    _call("causal_conv_forward", cfg, _seq(cfg, x, "x"), *_taps(cfg, weight, bias), _f32(past, "past", B, W - 1, H),
          _reset(reset, T, B), _seq(cfg, y, "y"), _f32(last, "last", B, W - 1, H))


def causal_conv_backward(cfg, x, weight, bias, past, reset, dy, dlast, dx, dweight, dbias, dpast, workspace) -> None:
    T, B, H, W = cfg.T, cfg.B, cfg.H, cfg.W
    _call("causal_conv_backward", cfg, _seq(cfg, x, "x"), *_taps(cfg, weight, bias), _f32(past, "past", B, W - 1, H),
          _reset(reset, T, B), _seq(cfg, dy, "dy"), _f32(dlast, "dlast", B, W - 1, H), _seq(cfg, dx, "dx"),
          _f32(dweight, "dweight", H, W), _f32(dbias, "dbias", H), _f32(dpast, "dpast", B, W - 1, H),
          *_bytes_of(workspace, "workspace"))


def _slots(t):
    """Rows of a pool."""
    _lib()
    return t.shape[0] if isinstance(t, _o._torch.Tensor) and t.dim() == 3 else 0


def causal_conv_step(cfg, x, weight, bias, slots, reset, past_in, past_out, y) -> None:
    """x, y: [B,H]; past_in, past_out: [n_slots,W-1,H].  (W = 1: or None, then any slot that is not negative is one.)"""
    B, H, W, n = cfg.B, cfg.H, cfg.W, _slots(past_in)
    if W == 1 and past_in is None:
        n = 2 ** 31 - 1 if past_out is None else _slots(past_out)
    _call("causal_conv_step", cfg, _row(cfg, x, "x"), *_taps(cfg, weight, bias),
          (slots, "slots", _o._torch.int32, (B,), _DENSE), n, _reset(reset, B), _f32(past_in, "past_in", n, W - 1, H),
          _f32(past_out, "past_out", n, W - 1, H), _row(cfg, y, "y"))


# ---- selective state space scan
def ssm_workspace_bytes(cfg: SsmCfg) -> int:
    return _size("ssm_workspace_bytes", cfg)


def ssm_saved_bytes(cfg: SsmCfg) -> int:
    return _size("ssm_saved_bytes", cfg)


def _ssm_inputs(cfg, rows, layout, x, dt, b, c, z, a, skip, bias):
    """rows: what the shapes of sequences begin with."""
    H, S, dtype = cfg.H, cfg.S, _dtype(cfg)
    wide, narrow = rows + (H,), rows + (S,)
    return _Group(((x, "x", dtype, wide, layout), (dt, "dt", dtype, wide, layout), (b, "b", dtype, narrow, layout),
                   (c, "c", dtype, narrow, layout), (z, "z", dtype, wide, layout), _f32(a, "a", H, S),
                   _f32(skip, "skip", H), _f32(bias, "bias", H)))                                  # (SsmInputs)


def ssm_forward(cfg, x, dt, b, c, z, a, skip, bias, h0, reset, y, h_last, saved, workspace) -> None:
    """x, dt, z (or None), y: [T,B,H]; b, c: [T,B,S]; a: [H,S]; skip, bias: [H] or None; h0, h_last: [B,H,S] or None."""
    T, B, H, S = cfg.T, cfg.B, cfg.H, cfg.S
    _call("ssm_forward", cfg, _ssm_inputs(cfg, (T, B), _SEQ, x, dt, b, c, z, a, skip, bias), _f32(h0, "h0", B, H, S),
          _reset(reset, T, B), _seq(cfg, y, "y"), _f32(h_last, "h_last", B, H, S), *_bytes_of(saved, "saved"),
          *_bytes_of(workspace, "workspace"))


def ssm_backward(cfg, x, dt, b, c, z, a, skip, bias, reset, saved, dy, dh_last, dx, ddt, db, dc, dz, da, dskip, dbias,
                 dh0, workspace) -> None:
    T, B, H, S = cfg.T, cfg.B, cfg.H, cfg.S
    dtype, wide, narrow = _dtype(cfg), (T, B, H), (T, B, S)
    grads = _Group(((dx, "dx", dtype, wide, _SEQ), (ddt, "ddt", dtype, wide, _SEQ), (db, "db", dtype, narrow, _SEQ),
                    (dc, "dc", dtype, narrow, _SEQ), (dz, "dz", dtype, wide, _SEQ), _f32(da, "da", H, S),
                    _f32(dskip, "dskip", H), _f32(dbias, "dbias", H), _f32(dh0, "dh0", B, H, S)))    # (SsmGrads)
    _call("ssm_backward", cfg, _ssm_inputs(cfg, (T, B), _SEQ, x, dt, b, c, z, a, skip, bias), _reset(reset, T, B),
          *_bytes_of(saved, "saved"), _seq(cfg, dy, "dy"), _f32(dh_last, "dh_last", B, H, S), grads,
          *_bytes_of(workspace, "workspace"))


def ssm_step(cfg, x, dt, b, c, z, a, skip, bias, slots, reset, state_in, state_out, y) -> None:
    """x, dt, z (or None), y: [B,H]; b, c: [B,S]; state_in, state_out: [n_slots,H,S]."""
    B, H, S, n = cfg.B, cfg.H, cfg.S, _slots(state_in)
    _call("ssm_step", cfg, _ssm_inputs(cfg, (B,), _STEP, x, dt, b, c, z, a, skip, bias),
          (slots, "slots", _o._torch.int32, (B,), _DENSE), n, _reset(reset, B), _f32(state_in, "state_in", n, H, S),
          _f32(state_out, "state_out", n, H, S), _row(cfg, y, "y"))


# ---- policy loss
def policy_workspace_bytes(cfg) -> int:
    """cfg: a ``LogitsCfg`` (its K is not looked at)."""
    return _size("policy_workspace_bytes", cfg)


def _policy(cfg, logits, tokens, old_logp, ref_logp, advantage):
    N = cfg.N
    return (_matrix(cfg, logits, "logits", N, cfg.V), _i64(tokens, "tokens", N), _f32(old_logp, "old_logp", N),
            _f32(ref_logp, "ref_logp", N), _f32(advantage, "advantage", N))


def policy_loss(cfg, rule, logits, tokens, old_logp, ref_logp, advantage, weight, loss, logp, ratio, kl, stats, dlogits,
                workspace) -> None:
    N, V = cfg.N, cfg.V
    cfg = _strided(cfg, ld=_ld(logits, V), ld_grad=_ld(dlogits, V))
    _call("policy_loss", cfg, rule, *_policy(cfg, logits, tokens, old_logp, ref_logp, advantage),
          _f32(weight, "weight", N), _f32(loss, "loss", N), _f32(logp, "logp", N), _f32(ratio, "ratio", N),
          _f32(kl, "kl", N), _f32(stats, "stats", N, 2), _matrix(cfg, dlogits, "dlogits", N, V),
          *_bytes_of(workspace, "workspace"))


def policy_loss_backward(cfg, rule, logits, tokens, old_logp, ref_logp, advantage, stats, dloss, dlogits) -> None:
    N, V = cfg.N, cfg.V
    cfg = _strided(cfg, ld=_ld(logits, V), ld_grad=_ld(dlogits, V))
    _call("policy_loss_backward", cfg, rule, *_policy(cfg, logits, tokens, old_logp, ref_logp, advantage),
          _f32(stats, "stats", N, 2), _f32(dloss, "dloss", N), _matrix(cfg, dlogits, "dlogits", N, V))
