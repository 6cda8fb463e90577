"""The operators around a gated linear recurrent layer in plain numpy, float64, from their definitions.

Test infrastructure only; inputs are float64 arrays (holding whatever the device arrays hold).
"""
from __future__ import annotations

import numpy as np


# ---- gated linear recurrence: h_t = a_t h_{t-1} + b_t
def _coeffs(gate, value, form):
    if form == "mix":
        with np.errstate(over="ignore"):
            return 1 / (1 + np.exp(-gate)), 1 / (1 + np.exp(gate))
    return np.exp(gate), np.ones_like(gate)


def glr_forward(gate, value, h0=None, reset=None, form="mix"):
    """States [T,B,H] after every step."""
    a, nb = _coeffs(gate, value, form)
    h = np.zeros(gate.shape[1:]) if h0 is None else np.array(h0, dtype=np.float64)
    out = np.empty(gate.shape)
    for t in range(gate.shape[0]):
        past = a[t] * h
        if reset is not None:
            past = np.where(reset[t][:, None] != 0, 0.0, past)
        h = past + nb[t] * value[t]
        out[t] = h
    return out


def glr_backward(gate, value, h, dh, h0=None, reset=None, dh_last=None, form="mix"):
    """(dgate, dvalue, dh0) for the loss sum(dh * h) + sum(dh_last * h[T-1])."""
    a, nb = _coeffs(gate, value, form)
    T = gate.shape[0]
    first = np.zeros(gate.shape[1:]) if h0 is None else np.array(h0, dtype=np.float64)
    carry = np.zeros(gate.shape[1:]) if dh_last is None else np.array(dh_last, dtype=np.float64)
    dgate, dvalue = np.empty(gate.shape), np.empty(gate.shape)
    for t in range(T - 1, -1, -1):
        lam = dh[t] + carry
        past = h[t - 1] if t else first
        carry = a[t] * lam
        if reset is not None:
            cut = reset[t][:, None] != 0
            past, carry = np.where(cut, 0.0, past), np.where(cut, 0.0, carry)
        if form == "mix":
            dgate[t] = lam * a[t] * nb[t] * (past - value[t])
        else:
            dgate[t] = lam * a[t] * past
        dvalue[t] = lam * nb[t]
    return dgate, dvalue, carry


# ---- rows of logits
def _log_softmax(x):
    """Row by row; a row of nothing but -inf stays that, a NaN or +inf makes its row NaN."""
    with np.errstate(invalid="ignore", divide="ignore"):
        m = np.max(np.where(np.isnan(x), -np.inf, x), axis=1, keepdims=True)
        d = x - np.where(np.isneginf(m), 0.0, m)
        s = np.exp(d).sum(1, keepdims=True)
        out = d - np.log(s)
    out[s[:, 0] == 0] = -np.inf
    return out


def token_logprobs(x, tokens, K, temperature=1.0):
    """(logp, entropy, top_logp, top_ids)"""
    lp = _log_softmax(x / temperature)
    p = np.exp(lp)
    with np.errstate(invalid="ignore"):
        entropy = -np.where(p > 0, p * lp, np.where(np.isnan(p), np.nan, 0.0)).sum(1)
    n = np.arange(len(x))
    logp = np.where(tokens < 0, 0.0, np.where(tokens >= x.shape[1], np.nan,
                                              lp[n, np.clip(tokens, 0, x.shape[1] - 1)]))
    key = np.where(np.isnan(x), np.inf, x)                 # NaN above all, +inf next: the same rank is not tested
    ids = np.argsort(-key, axis=1, kind="stable")[:, :K]
    return logp, entropy + 0.0, np.take_along_axis(lp, ids, 1), ids


def distill(x, ids, teacher, weight, temperature=1.0):
    """(loss, dlogits)"""
    N, V = x.shape
    lp = _log_softmax(x / temperature)
    p = np.exp(lp)
    loss, grad = np.zeros(N), np.zeros((N, V))
    for n in range(N):
        t = np.where(ids[n] < 0, -np.inf, teacher[n] / temperature)
        if np.all(np.isneginf(t)):
            continue
        if np.any(ids[n] >= V):
            loss[n] = np.nan
            grad[n] = np.nan if weight[n] != 0 else 0.0
            continue
        q = np.exp(t - t.max())
        q /= q.sum()
        on = q > 0
        loss[n] = np.sum(q[on] * (np.log(q[on]) - lp[n, ids[n][on]]))
        if weight[n] == 0:
            continue
        g = p[n].copy()
        np.add.at(g, ids[n][on], -q[on])
        grad[n] = g * weight[n] / temperature
    return loss, grad


# ---- product in 8-bit integers
def q8_quantize(x):
    """(q, scale) of rows of float32 values; both quotients are rounded to float32 by definition."""
    x = np.asarray(x, dtype=np.float32)
    finite = np.isfinite(x).all(1, keepdims=True)
    clean = np.where(finite, x, np.float32(0))
    amax = np.abs(clean).max(1, keepdims=True)
    scale = np.maximum(amax / np.float32(127), np.float32(2.0 ** -126))
    q = np.rint(clean / scale)
    return q.astype(np.int8), np.where(finite, scale, np.float32(np.nan))[:, 0]


def q8_linear(x, w_q, w_scale, bias=None):
    q, scale = q8_quantize(x)
    y = q.astype(np.float64) @ w_q.astype(np.float64).T
    y = y * scale.astype(np.float64)[:, None] * np.asarray(w_scale, dtype=np.float64)
    return y if bias is None else y + bias
