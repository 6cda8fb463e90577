"""The float64 oracle of the operators over tokens against torch: autograd through plain step-by-step forms, and differences."""
import numpy as np
import pytest
import torch

from oracle import token_ops_oracle as orc


def r(rng, *s):
    return rng.standard_normal(s)


def test_embedding():
    rng = np.random.default_rng(0)
    tok, table, dout = np.array([3, -1, 0, 3, 7, 9]), r(rng, 8, 5), r(rng, 6, 5)
    out = orc.embed_lookup(tok, table, 2.5)
    t = torch.from_numpy(table).requires_grad_(True)
    ref = 2.5 * t[torch.tensor([3, 0, 3, 7])]
    assert np.array_equal(out[[0, 2, 3, 4]], ref.detach().numpy())
    assert (out[1] == 0).all() and np.isnan(out[5]).all()
    (ref * torch.from_numpy(dout[[0, 2, 3, 4]])).sum().backward()
    assert np.allclose(orc.embed_backward(tok, dout, 8, 2.5), t.grad.numpy(), atol=1e-14)


@pytest.mark.parametrize("T,W,silu,resets", [(7, 4, True, False), (2, 5, True, False), (6, 1, False, False), (9, 3, True, True)])
def test_convolution(T, W, silu, resets):
    rng = np.random.default_rng(T)
    B, H = 2, 3
    x, w, bias, past = r(rng, T, B, H), r(rng, H, W), r(rng, H), r(rng, B, W - 1, H)
    dy, dlast = r(rng, T, B, H), r(rng, B, W - 1, H)
    reset = (rng.random((T, B)) < 0.3).astype(np.uint8) if resets else None
    tx, tw, tb, tp = (torch.from_numpy(v).requires_grad_(True) for v in (x, w, bias, past))
    ys, lasts = [], []
    for b in range(B):
        window = [tp[b, j] for j in range(W - 1)]
        for t in range(T):
            if resets and reset[t, b]:
                window = [torch.zeros(H, dtype=torch.float64)] * (W - 1)
            window = window + [tx[t, b]]
            p = tb + sum(tw[:, k] * window[k] for k in range(W))
            ys.append(p * torch.sigmoid(p) if silu else p)
            window = window[1:]
        lasts += window
    y = torch.stack(ys).view(B, T, H).transpose(0, 1)
    last = torch.stack(lasts).view(B, W - 1, H) if W > 1 else torch.zeros(B, 0, H, dtype=torch.float64)
    got, got_last, _ = orc.conv_forward(x, w, bias, past, reset, silu)
    assert np.allclose(got, y.detach().numpy(), atol=1e-13) and np.allclose(got_last, last.detach().numpy(), atol=1e-14)
    ((y * torch.from_numpy(dy)).sum() + (last * torch.from_numpy(dlast)).sum()).backward()
    for a, b in zip(orc.conv_backward(x, w, bias, dy, past, reset, silu, dlast), (tx, tw, tb, tp)):
        ref = b.grad if b.grad is not None else torch.zeros_like(b)
        assert np.allclose(a, ref.numpy(), atol=1e-12)


@pytest.mark.parametrize("gated,resets,full", [(True, False, True), (False, True, True), (True, True, False)])
def test_selective_scan(gated, resets, full):
    rng = np.random.default_rng(5)
    T, B, H, S = 7, 2, 3, 4
    v = {k: r(rng, T, B, H) for k in ("x", "dt", "z")}
    v.update(b=r(rng, T, B, S), c=r(rng, T, B, S), a=-np.exp(r(rng, H, S)))
    if full:
        v.update(skip=r(rng, H), bias=r(rng, H), h0=r(rng, B, H, S))
    if not gated:
        v["z"] = None
    reset = (rng.random((T, B)) < 0.3).astype(np.uint8) if resets else None
    dy, dh = r(rng, T, B, H), r(rng, B, H, S)
    t = {k: torch.from_numpy(a).requires_grad_(True) for k, a in v.items() if a is not None}
    h = t.get("h0", torch.zeros(B, H, S, dtype=torch.float64))
    loss = 0
    ys = []
    for i in range(T):
        d = torch.nn.functional.softplus(t["dt"][i] + t.get("bias", 0), threshold=1e9)
        if resets:
            h = torch.where(torch.from_numpy(reset[i] != 0)[:, None, None], torch.zeros_like(h), h)
        h = torch.exp(d[..., None] * t["a"]) * h + (d * t["x"][i])[..., None] * t["b"][i][:, None]
        y = (h * t["c"][i][:, None]).sum(-1) + t.get("skip", 0) * t["x"][i]
        ys.append(y * torch.nn.functional.silu(t["z"][i]) if gated else y)
        loss = loss + (ys[-1] * torch.from_numpy(dy[i])).sum()
    (loss + (h * torch.from_numpy(dh)).sum()).backward()
    got, states, _ = orc.ssm_forward(reset=reset, **v)
    assert np.allclose(got, torch.stack(ys).detach().numpy(), atol=1e-13)
    assert np.allclose(states[-1], h.detach().numpy(), atol=1e-13)
    g = orc.ssm_backward(reset=reset, dy=dy, dh_last=dh, **v)
    for k, a in t.items():
        name = {"skip": "dskip", "bias": "dbias", "h0": "dh0"}.get(k, "d" + k)
        assert np.allclose(g[name], a.grad.numpy(), atol=1e-11), k


@pytest.mark.parametrize("beta,t", [(0.0, 1.0), (0.3, 0.7)])
def test_policy_loss(beta, t):
    rng = np.random.default_rng(7)
    N, V, low, high = 40, 6, 0.2, 0.3
    x, tok = 2 * r(rng, N, V), rng.integers(-1, V, N)
    lx = torch.from_numpy(x).requires_grad_(True)
    lp = torch.log_softmax(lx / t, 1).gather(1, torch.from_numpy(tok).clamp(min=0)[:, None])[:, 0]
    old, ref = lp.detach().numpy() + 0.4 * r(rng, N), lp.detach().numpy() + 0.4 * r(rng, N)
    A, w = r(rng, N), rng.random(N)
    ratio = torch.exp(lp - torch.from_numpy(old))
    ta = torch.from_numpy(A)
    loss = -torch.minimum(ratio * ta, ratio.clamp(1 - low, 1 + high) * ta)
    d = torch.from_numpy(ref) - lp
    loss = loss + beta * (torch.exp(d) - d - 1)
    some = torch.from_numpy(tok >= 0)
    (loss * torch.from_numpy(w))[some].sum().backward()
    got = orc.policy_loss(x, tok, old, ref if beta else None, A, w, t, low, high, beta)
    want = [torch.where(some, v, 0.0).detach().numpy() for v in (loss, lp, ratio, torch.exp(d) - d - 1)]
    for k in range(4 if beta else 3):
        assert np.allclose(got[k], want[k], atol=1e-13), k
    assert np.allclose(got[4], lx.grad.numpy(), atol=1e-13)
    assert ((got[2] > 1 + high) & (A > 0)).any() and ((got[2] < 1 - low) & (got[2] > 0) & (A < 0)).any()
