"""The path that uses the operators together: a student taught by a GRU from its top logits, then served in 8 bits."""
import numpy as np
import pytest
import torch

import paper_2203_04738_amd as mg
from paper_2203_04738_amd.student import LinearStudent, Served, example, teacher_top

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def small(seed=0, T=20, B=3, D=5, H=70, V=40, K=6, lr=1e-3):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g).to(DEV)  # noqa: E731
    params = [[r(2 * H, n) / n ** 0.5, 0.1 * r(2 * H)] for n in (D, H)]
    student = LinearStudent(T, B, params, [r(V, H) / H ** 0.5, 0.1 * r(V)], K=K, temperature=1.5, lr=lr)
    x = r(T, B, D)
    ids, top = teacher_top(2 * r(T * B, V), K)
    ids[::5] = -1
    return student, x, ids, top


def test_training_step_has_the_gradients_of_torch():
    # the same network, loss and gradients in float64 torch autograd on the CPU
    student, x, ids, top = small()
    T, B, H, V, tau = 20, 3, 70, 40, 1.5
    ps = [p.detach().double().cpu().requires_grad_(True) for layer in student.params for p in layer]
    ho = [p.detach().double().cpu().requires_grad_(True) for p in student.head]
    h = x.double().cpu()
    for W, b in (ps[:2], ps[2:]):
        gv = h @ W.t() + b
        a, out, s = torch.sigmoid(gv[..., :H]), [], torch.zeros(B, H, dtype=torch.float64)
        for t in range(T):
            s = a[t] * s + (1 - a[t]) * gv[t, :, H:]
            out.append(s)
        h = torch.stack(out)
    lp = torch.log_softmax((h.reshape(T * B, H) @ ho[0].t() + ho[1]) / tau, 1)
    i, rows = ids.cpu(), (ids.cpu() >= 0).all(1)
    q = torch.softmax(top.double().cpu() / tau, 1)
    each = (q * (torch.log(q) - lp.gather(1, i.clamp(min=0)))).sum(1)
    loss = each[rows].mean()
    loss.backward()
    got = student.step(x, ids, top)
    assert abs(got - float(loss)) <= 1e-5 * max(1.0, float(loss))
    mine = [p.grad for layer in student.params for p in layer] + [p.grad for p in student.head]
    for m, ref in zip(mine, ps + ho):
        # (gradients are sums of 60 products of values known to about 1e-6 each, in float)
        err = (m.double().cpu() - ref.grad).abs().max() / ref.grad.abs().max()
        assert err <= 2e-5, float(err)


def test_teaching_lowers_the_loss_and_serving_agrees_with_training():
    first, last, by_token, to_own = example(T=128, B=16, steps=40, say=lambda *_: None)
    assert last < 0.7 * first
    # read at once or token by token: the same 8-bit products, states summed in another order (1e-6), which may move
    # a value of the next layer across a rounding to 8 bits (a step of 1/127 of its row's largest, of many)
    assert by_token <= 0.1
    # 8-bit weights and tokens in three products: each within 1/254 of a row's largest value
    assert to_own <= 0.15


def test_served_sequences_do_not_touch_each_other():
    student, x, _, _ = small(seed=3)
    served = Served(student, slots=6)
    slots = torch.tensor([4, 1, 2], dtype=torch.int32, device=DEV)
    served.read(x, slots)
    before = [s.clone() for s in served.state]
    served.next(x[0, :2], slots[:2])
    for s, b in zip(served.state, before):
        assert torch.equal(s[[0, 2, 3, 5]], b[[0, 2, 3, 5]]) and not torch.equal(s[[4, 1]], b[[4, 1]])
    logits = served.next(x[1], slots)
    logp, entropy, top, ids = served.alternatives(logits, 4, torch.tensor([0, 5, -1], device=DEV))
    lp = torch.log_softmax(logits.double(), 1)
    assert torch.allclose(top.double(), torch.topk(lp, 4, dim=1).values, atol=1e-5)
    assert abs(float(logp[1]) - float(lp[1, 5])) <= 1e-5 and float(logp[2]) == 0
    assert np.allclose(entropy.cpu().numpy(), -(lp.exp() * lp).sum(1).cpu().numpy(), atol=1e-5)
