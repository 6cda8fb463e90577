"""The operators of a recurrent student over tokens in plain numpy, float64, from their definitions.

Test infrastructure only; inputs are float64 arrays (holding whatever the device arrays hold).
"""
from __future__ import annotations

import numpy as np


def sigmoid(v):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-v))


# ---- embedding
def embed_lookup(tokens, table, scale):
    out = np.zeros((len(tokens), table.shape[1]))
    for n, t in enumerate(tokens):
        if t >= len(table):
            out[n] = np.nan
        elif t >= 0:
            out[n] = scale * table[t]
    return out


def embed_backward(tokens, dout, V, scale):
    grad = np.zeros((V, dout.shape[1]))
    for n, t in enumerate(tokens):
        if 0 <= t < V:
            grad[t] += scale * dout[n]
    return grad


# ---- causal convolution; x[T,B,H], weight[H,W], past[B,W-1,H]
def _visible(reset, s, t, b):
    """Whether step t of batch row b sees input s."""
    return reset is None or not np.any(reset[max(s + 1, 0):t + 1, b])


def _input(x, past, s, b):
    return x[s, b] if s >= 0 else past[b, s + past.shape[1]]


def conv_forward(x, weight, bias, past=None, reset=None, silu=True):
    """(y, last, p)"""
    T, B, H = x.shape
    W = weight.shape[1]
    past = np.zeros((B, W - 1, H)) if past is None else past
    p = np.zeros((T, B, H)) + (0 if bias is None else bias)
    for t in range(T):
        for b in range(B):
            for k in range(W):
                s = t - W + 1 + k
                if _visible(reset, s, t, b):
                    p[t, b] += weight[:, k] * _input(x, past, s, b)
    last = np.zeros((B, W - 1, H))
    for b in range(B):
        for j in range(W - 1):
            s = T - (W - 1) + j
            if _visible(reset, s, T - 1, b):
                last[b, j] = _input(x, past, s, b)
    return (p * sigmoid(p) if silu else p.copy()), last, p


def conv_backward(x, weight, bias, dy, past=None, reset=None, silu=True, dlast=None):
    """(dx, dweight, dbias, dpast) for the loss sum(dy * y) + sum(dlast * last)."""
    T, B, H = x.shape
    W = weight.shape[1]
    first = np.zeros((B, W - 1, H)) if past is None else past
    _, _, p = conv_forward(x, weight, bias, past, reset, silu)
    s_ = sigmoid(p)
    dp = dy * (s_ + p * s_ * sigmoid(-p)) if silu else dy
    dx, dw, dpast = np.zeros_like(x), np.zeros_like(weight), np.zeros((B, W - 1, H))

    def to(s, b, v):
        if s >= 0:
            dx[s, b] += v
        else:
            dpast[b, s + W - 1] += v

    for b in range(B):
        for t in range(T):
            for k in range(W):
                s = t - W + 1 + k
                if _visible(reset, s, t, b):
                    to(s, b, weight[:, k] * dp[t, b])
                    dw[:, k] += dp[t, b] * _input(x, first, s, b)
        for j in range(W - 1):
            s = T - (W - 1) + j
            if dlast is not None and _visible(reset, s, T - 1, b):
                to(s, b, dlast[b, j])
    return dx, dw, dp.sum((0, 1)), dpast


# ---- selective state space scan; x, dt, z: [T,B,H], b, c: [T,B,S], a: [H,S]
def _d(dt, bias):
    v = dt + (0 if bias is None else bias)
    return np.logaddexp(v, 0), sigmoid(v)


def ssm_forward(x, dt, b, c, z, a, skip=None, bias=None, h0=None, reset=None):
    """(y, states [T,B,H,S], sums before the gate)"""
    T, B, H = x.shape
    S = a.shape[1]
    d, _ = _d(dt, bias)
    h = np.zeros((B, H, S)) if h0 is None else np.array(h0)
    states, s = np.empty((T, B, H, S)), np.empty((T, B, H))
    for t in range(T):
        with np.errstate(invalid="ignore"):
            past = np.exp(d[t][..., None] * a) * h
        if reset is not None:
            past = np.where(reset[t][:, None, None] != 0, 0.0, past)
        h = past + (d[t] * x[t])[..., None] * b[t][:, None, :]
        states[t] = h
        s[t] = (h * c[t][:, None, :]).sum(-1) + (0 if skip is None else skip * x[t])
    return (s if z is None else s * z * sigmoid(z)), states, s


def ssm_backward(x, dt, b, c, z, a, dy, skip=None, bias=None, h0=None, reset=None, dh_last=None):
    """A dict of the gradients of sum(dy * y) + sum(dh_last * h_T)."""
    T, B, H = x.shape
    S = a.shape[1]
    _, states, s = ssm_forward(x, dt, b, c, z, a, skip, bias, h0, reset)
    first = np.zeros((B, H, S)) if h0 is None else h0
    d, slope = _d(dt, bias)
    g = {k: np.zeros_like(v) for k, v in (("dx", x), ("ddt", dt), ("db", b), ("dc", c), ("da", a))}
    ds = dy
    if z is not None:
        sz = sigmoid(z)
        ds = dy * z * sz
        g["dz"] = dy * s * (sz + z * sz * sigmoid(-z))
    lam = np.zeros((B, H, S)) if dh_last is None else np.array(dh_last)
    for t in range(T - 1, -1, -1):
        past = states[t - 1] if t else first
        keep = np.exp(d[t][..., None] * a)
        lam = lam + ds[t][..., None] * c[t][:, None, :]
        g["dc"][t] = (ds[t][..., None] * states[t]).sum(1)
        g["db"][t] = ((d[t] * x[t])[..., None] * lam).sum(1)
        lb = (lam * b[t][:, None, :]).sum(-1)
        with np.errstate(invalid="ignore"):
            inner, lam = lam * keep * past, lam * keep
        if reset is not None:
            cut = reset[t][:, None, None] != 0
            inner, lam = np.where(cut, 0.0, inner), np.where(cut, 0.0, lam)
        g["da"] += (inner * d[t][..., None]).sum(0)
        g["ddt"][t] = (lb * x[t] + (inner * a).sum(-1)) * slope[t]
        g["dx"][t] = lb * d[t] + ds[t] * (0 if skip is None else skip)
    g["dskip"], g["dbias"], g["dh0"] = (ds * x).sum((0, 1)), g["ddt"].sum((0, 1)), lam
    return g


# ---- policy loss
def policy_loss(logits, tokens, old, ref, advantage, weight, t, low, high, beta):
    """(loss, logp, ratio, kl, dlogits), rows one by one."""
    N, V = logits.shape
    out = [np.zeros(N) for _ in range(4)] + [np.zeros((N, V))]
    with np.errstate(all="ignore"):
        for n in range(N):
            tok, w = tokens[n], 1.0 if weight is None else weight[n]
            if tok < 0:
                continue
            if tok >= V:
                for o in out[:4]:
                    o[n] = np.nan
                if w != 0:
                    out[4][n] = np.nan
                continue
            x = logits[n]
            m = x.max()
            e = np.exp((x - (0.0 if np.isneginf(m) else m)) / t)
            lp = -np.inf if x[tok] == -np.inf else (x[tok] - m) / t - np.log(e.sum())
            if np.isnan(x).any() or np.isposinf(x).any():
                lp = np.nan
            p = e / e.sum() if e.sum() != 0 else e
            r = np.exp(lp - old[n])
            A = advantage[n]
            gain, clipped = r * A, np.clip(r, 1 - low, 1 + high) * A
            loss, slope = (-clipped, 0.0) if gain > clipped else (-gain, -gain)
            k = 0.0
            if ref is not None:
                d = ref[n] - lp
                k = np.expm1(d) - d if np.isfinite(d) else np.inf if d == np.inf else np.nan
                if beta:
                    loss, slope = loss + beta * k, slope - beta * np.expm1(d)
            out[0][n], out[1][n], out[2][n], out[3][n] = loss, lp, r, k
            if w != 0 and slope != 0:
                g = -w * slope / t * p
                g[tok] += w * slope / t
                out[4][n] = g
    return out
