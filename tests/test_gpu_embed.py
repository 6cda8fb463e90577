"""Embedding and the gradient of its table on the GPU against the float64 oracle."""
import numpy as np
import pytest
import torch

import paper_2203_04738_amd as mg
from oracle import token_ops_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": (mg.MGRIT_F32, torch.float32, 2.0 ** -24), "bf16": (mg.MGRIT_BF16, torch.bfloat16, 2.0 ** -8),
         "f16": (mg.MGRIT_F16, torch.float16, 2.0 ** -11)}


def padded(rows, cols, dtype, pad, fill=float("nan")):
    """(a buffer full of a mark, its matrix [rows, cols])"""
    buf = torch.full((rows, cols + pad), fill, dtype=dtype, device=DEV)
    return buf, buf[:, :cols]


def run(tokens, V, D, dtype, scale, pad=0, seed=0):
    code, dt, unit = TYPES[dtype]
    g = torch.Generator().manual_seed(seed)
    N = len(tokens)
    _, table = padded(V, D, dt, pad)
    _, dout = padded(N, D, dt, pad)
    table.copy_(torch.randn(V, D, generator=g))
    dout.copy_(torch.randn(N, D, generator=g))
    (obuf, out), (gbuf, grad) = padded(N, D, dt, pad, 77.0), padded(V, D, dt, pad, 77.0)
    tok = torch.as_tensor(tokens, dtype=torch.int64).to(DEV)
    cfg = mg.EmbedCfg(N, V, D, code, scale)
    ws = torch.full((mg.embed_workspace_bytes(cfg),), 255, dtype=torch.uint8, device=DEV)
    mg.embed_lookup(cfg, tok, table, out)
    mg.embed_backward(cfg, tok, dout, grad, ws)
    torch.cuda.synchronize()
    if pad:
        assert (obuf[:, D:] == 77).all() and (gbuf[:, D:] == 77).all()
    t, d = table.double().cpu().numpy(), dout.double().cpu().numpy()
    tokens = np.asarray(tokens)
    want = orc.embed_lookup(tokens, t, scale)
    assert np.array_equal(np.isnan(want), np.isnan(out.double().cpu().numpy()))
    # one product in float, then the type's rounding (half a step), subnormal results to a step of 2^-24
    err = np.abs(out.double().cpu().numpy() - want)
    assert (err <= (unit + 2.0 ** -24) * np.abs(want) + 2.0 ** -24 * scale)[~np.isnan(want)].all()
    ref = orc.embed_backward(tokens, d, V, scale)
    size = orc.embed_backward(tokens, np.abs(d), V, scale)
    # a sum of n floats: at most n roundings of 2^-24 of a partial sum, that is of the sum of magnitudes; the longest way of
    # any term is through the 8 or (of more than 4096 tokens) 32 of its block, then through the blocks of a part, then some more
    per = 8 if N <= 4096 else 32
    n = min(N, per) + N // per / 4 + 4
    err = np.abs(grad.double().cpu().numpy() - ref)
    assert (err <= unit * np.abs(ref) + n * 2.0 ** -24 * size + 2.0 ** -24 * scale * (size > 0)).all()
    return grad


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("N,V,D,pad", [(1, 1, 1, 0), (1, 5, 8, 0), (33, 7, 64, 0), (100, 300, 520, 8), (257, 130, 51, 3),
                                       (1000, 40000, 24, 0), (64, 70000, 16, 0), (31, 300000, 8, 0), (5000, 1000, 32, 0)])
def test_lookup_and_gradient(dtype, N, V, D, pad):
    rng = np.random.default_rng(N)
    tokens = np.minimum((V * rng.random(N) ** 3).astype(np.int64), V - 1)
    run(tokens, V, D, dtype, 2.5, pad)


@pytest.mark.parametrize("N,V", [(8193, 1000), (30000, 20000), (40000, 129), (40000, 70000), (140001, 3000), (70000, 600000)])
def test_parts_of_many_tokens(N, V):
    """Several workgroups place the tokens of a range; the last part is short, or has waves with nothing."""
    rng = np.random.default_rng(N)
    tokens = np.minimum((V * rng.random(N) ** 3).astype(np.int64), V - 1)
    tokens[rng.random(N) < 0.1] = -1
    run(tokens, V, 3, "f32", 1.0, seed=N)


@pytest.mark.parametrize("kind", ["same", "padding", "beyond", "last", "two", "rising", "falling"])
@pytest.mark.parametrize("N", [1, 8, 9, 32, 33, 700, 4096, 4097, 9000])
def test_tokens_of_every_kind(kind, N):
    V, n = 200, np.arange(N)
    tokens = {"same": np.full(N, 3), "padding": np.full(N, -1), "beyond": np.where(n % 3, V + 5 * n, n % V),
              "last": np.full(N, V - 1), "two": np.where(n < N // 2, 199, 0), "rising": n % V,
              "falling": V - 1 - n % V}[kind]
    tokens = np.where(n % 7 == 6, -1 - n, tokens)
    run(tokens, V, 40, "f32", 1.0)


def test_extreme_tokens_are_neither_read_nor_written():
    t = [2 ** 62, -2 ** 63, 2 ** 31, 2 ** 32 + 1, -2 ** 31, 4]
    grad = run(t, 5, 16, "bf16", 1.0)
    assert (grad[:4] == 0).all()


def test_a_sum_has_the_same_bits_in_every_run():
    rng = np.random.default_rng(1)
    tokens = np.minimum((500 * rng.random(20000) ** 4).astype(np.int64), 499)
    first = run(tokens, 500, 64, "f32", 1.0)
    for _ in range(3):
        assert torch.equal(first, run(tokens, 500, 64, "f32", 1.0))


def test_captured_and_replayed():
    code, dt, _ = TYPES["bf16"]
    cfg = mg.EmbedCfg(300, 90, 64, code, 3.0)
    g = torch.Generator().manual_seed(3)
    table, dout = (torch.randn(n, 64, generator=g).to(DEV, dt) for n in (90, 300))
    tok = torch.randint(-2, 90, (300,), generator=g).to(DEV)
    out, grad = torch.empty(300, 64, dtype=dt, device=DEV), torch.empty(90, 64, dtype=dt, device=DEV)
    ws = torch.empty(mg.embed_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)

    def call(o, d):
        mg.embed_lookup(cfg, tok, table, o)
        mg.embed_backward(cfg, tok, dout, d, ws)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call(out, grad)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, grad)
    for i in range(3):
        tok.copy_(torch.randint(-2, 90, (300,), generator=g))
        out.fill_(9)
        grad.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        o, d = torch.empty_like(out), torch.empty_like(grad)
        call(o, d)
        assert torch.equal(out, o) and torch.equal(grad, d)
