"""Operators over tokens whose arrays reach beyond 32-bit offsets: the same bits as for the same values close together."""
import pytest
import torch

import paper_2203_04738_amd as mg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def far(t, stride):
    """A copy of t[T,B,C] whose steps are `stride` elements apart (nothing else of the memory is touched)."""
    out = torch.empty((t.shape[0] - 1) * stride + t[0].numel(), dtype=t.dtype, device=DEV)
    v = torch.as_strided(out, t.shape, (stride, t.shape[2], 1))
    v.copy_(t)
    return v


def test_sequences_with_far_steps():
    T, B, H, S, W, stride = 70, 1, 66, 16, 4, 1 << 25           # 70 x 2^25 elements of 2 bytes: 4.7 GB an array
    g = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=g).to(DEV)  # noqa: E731
    x, dt, z, dy, b, c = (r(T, B, n).to(BF) for n in (H, H, H, H, S, S))
    w, bias, a = r(H, W), r(H), -r(H, S).exp()
    ccfg, scfg = mg.ConvCfg(T, B, H, W, mg.CONV_SILU, mg.MGRIT_BF16), mg.SsmCfg(T, B, H, S, mg.MGRIT_BF16)
    byte = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)  # noqa: E731
    ws = byte(max(mg.causal_conv_workspace_bytes(ccfg), mg.ssm_workspace_bytes(scfg)))
    saved = byte(mg.ssm_saved_bytes(scfg))

    def run(place):
        px, pdt, pz, pdy, pb, pc = (place(t) for t in (x, dt, z, dy, b, c))
        y, dx = place(torch.zeros_like(x)), place(torch.zeros_like(x))
        dw, db = torch.empty(H, W, device=DEV), torch.empty(H, device=DEV)
        mg.causal_conv_forward(ccfg, px, w, bias, None, None, y, None)
        mg.causal_conv_backward(ccfg, px, w, bias, None, None, pdy, None, dx, dw, db, None, ws)
        out = [y.clone(), dx.clone(), dw, db]
        da = torch.empty(H, S, device=DEV)
        mg.ssm_forward(scfg, px, pdt, pb, pc, pz, a, bias, None, None, None, y, None, saved, ws)
        grads = [dx] + [place(torch.zeros_like(t)) for t in (dt, b, c, z)]
        mg.ssm_backward(scfg, px, pdt, pb, pc, pz, a, bias, None, None, saved, pdy, None, *grads, da, None, None, None, ws)
        return out + [y.clone(), da] + [t.clone() for t in grads]

    close = run(lambda t: t.clone())
    for p, q in zip(close, run(lambda t: far(t, stride))):
        assert torch.equal(p, q) and float(p.abs().max()) > 0


def test_a_table_with_far_rows():
    N, V, D, ld = 40, 33000, 64, 1 << 17                         # 33000 x 2^17 elements of 2 bytes: 8.7 GB
    g = torch.Generator().manual_seed(1)
    tok = torch.randint(0, V, (N,), generator=g)
    tok[:2] = torch.tensor([V - 1, 0])
    tok = tok.to(DEV)
    buf = torch.empty((V - 1) * ld + D, dtype=BF, device=DEV)
    table = torch.as_strided(buf, (V, D), (ld, 1))
    small = torch.randn(V, D, generator=g).to(DEV, BF)
    table.copy_(small)
    cfg = mg.EmbedCfg(N, V, D, mg.MGRIT_BF16, 2.0)
    out, want = (torch.empty(N, D, dtype=BF, device=DEV) for _ in range(2))
    mg.embed_lookup(cfg, tok, table, out)
    mg.embed_lookup(cfg, tok, small, want)
    assert torch.equal(out, want) and torch.equal(out, 2 * small[tok])
    ws = torch.empty(mg.embed_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)
    grad = torch.empty_like(small)
    table.fill_(7)
    mg.embed_backward(cfg, tok, out, table, ws)
    mg.embed_backward(cfg, tok, out, grad, ws)
    assert torch.equal(table, grad) and float(grad.abs().max()) > 0
