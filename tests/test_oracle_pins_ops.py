"""The oracle of the operators around a gated linear recurrent layer against torch in float64 on the CPU."""
import numpy as np
import pytest
import torch

from oracle import ops_oracle as orc


@pytest.mark.parametrize("form", ["mix", "decay"])
def test_recurrence_and_its_adjoint_are_torchs(form):
    rng = np.random.default_rng(0)
    T, B, H = 30, 3, 5
    gate = rng.standard_normal((T, B, H)) if form == "mix" else -rng.random((T, B, H))
    value, h0, dh, dh_last = (rng.standard_normal(s) for s in ((T, B, H), (B, H), (T, B, H), (B, H)))
    reset = (rng.random((T, B)) < 0.1).astype(np.uint8)
    g, v, s0 = (torch.from_numpy(a).requires_grad_(True) for a in (gate, value, h0))
    s, out = s0, []
    for t in range(T):
        a = torch.sigmoid(g[t]) if form == "mix" else torch.exp(g[t])
        b = (1 - a) * v[t] if form == "mix" else v[t]
        s = a * s * torch.from_numpy(1.0 - reset[t])[:, None] + b
        out.append(s)
    out = torch.stack(out)
    ((out * torch.from_numpy(dh)).sum() + (out[-1] * torch.from_numpy(dh_last)).sum()).backward()
    h = orc.glr_forward(gate, value, h0, reset, form)
    grads = orc.glr_backward(gate, value, h, dh, h0, reset, dh_last, form)
    assert np.allclose(h, out.detach().numpy(), rtol=0, atol=1e-12)
    for mine, ref in zip(grads, (g.grad, v.grad, s0.grad)):
        assert np.allclose(mine, ref.numpy(), rtol=0, atol=1e-11)


def test_log_probabilities_entropy_and_alternatives():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 17))
    x[1, 3], x[2, :] = -np.inf, 0.25
    tokens = np.array([0, 4, -1, 16, 17])
    logp, entropy, top, ids = orc.token_logprobs(x, tokens, 4, 0.7)
    lp = torch.log_softmax(torch.from_numpy(x) / 0.7, 1)
    assert np.allclose(logp[[0, 1, 3]], lp[[0, 1, 3], [0, 4, 16]].numpy(), atol=1e-12)
    assert logp[2] == 0 and np.isnan(logp[4])
    assert np.allclose(entropy, torch.special.entr(lp.exp()).sum(1).numpy(), atol=1e-12)
    assert np.allclose(top, torch.topk(lp, 4, 1).values.numpy(), atol=1e-12)
    assert np.array_equal(ids[2], [0, 1, 2, 3])                  # ties: the lowest indices
    none = orc.token_logprobs(np.full((1, 3), -np.inf), np.array([1]), 2)
    assert none[0][0] == -np.inf and none[1][0] == 0 and np.array_equal(none[3], [[0, 1]])


def test_distillation_is_the_divergence_on_the_teachers_entries():
    rng = np.random.default_rng(2)
    N, V, K, tau = 6, 23, 4, 1.7
    x, t, w = rng.standard_normal((N, V)), rng.standard_normal((N, K)), rng.random(N)
    ids = np.stack([rng.choice(V, K, replace=False) for _ in range(N)])
    ids[1, 2:] = -1
    ids[2] = -1
    ids[3, 1] = ids[3, 0]
    y = torch.from_numpy(x).requires_grad_(True)
    lp = torch.log_softmax(y / tau, 1)
    q = torch.softmax(torch.from_numpy(np.where(ids < 0, -np.inf, t / tau)), 1).nan_to_num(0.0)
    i = torch.from_numpy(ids).clamp(min=0)
    loss = (torch.special.xlogy(q, q) - q * lp.gather(1, i)).sum(1)
    (loss * torch.from_numpy(w)).sum().backward()
    mine, grad = orc.distill(x, ids, t, w, tau)
    assert np.allclose(mine, loss.detach().numpy(), atol=1e-12)
    assert np.allclose(grad, y.grad.numpy(), atol=1e-12)


def test_quantised_rows_and_products():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((4, 9)).astype(np.float32)
    x[1] = 0
    x[2, 3] = np.nan
    q, scale = orc.q8_quantize(x)
    assert np.array_equal(np.abs(q[[0, 3]]).max(1), [127, 127]) and not q[[1, 2]].any()
    assert np.isnan(scale[2]) and scale[1] == np.float32(2.0 ** -126)
    assert np.all(np.abs(q[0] * scale[0] - x[0]) <= 0.5001 * scale[0])
    w = rng.integers(-128, 128, (5, 9)).astype(np.int8)
    ws, b = rng.random(5).astype(np.float32), rng.standard_normal(5).astype(np.float32)
    y = orc.q8_linear(x, w, ws, b)
    assert np.allclose(y[0], (q[0].astype(int) @ w.astype(int).T) * (scale[0].astype(float) * ws) + b, rtol=1e-12)
    assert np.isnan(y[2]).all() and np.allclose(y[1], b)
