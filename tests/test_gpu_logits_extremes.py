"""Rows of logits at the ends of the types' ranges: long rows of which a mask leaves whole segments, masks of the type's
lowest value beside -inf, teachers as far apart, at temperatures that carry any of it beyond a float."""
import numpy as np
import pytest
import torch

import paper_2203_04738_amd as mg
from oracle import ops_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": (mg.MGRIT_F32, torch.float32), "bf16": (mg.MGRIT_BF16, torch.bfloat16),
         "f16": (mg.MGRIT_F16, torch.float16)}
# log p = (x - max) / t - log s: three roundings to 2^-24 of values up to some 40, and sums of exponentials, each to
# (40 log2 e + 3) 2^-24 = 4e-6 of itself
TOL = 1.2e-5
UNIT = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8, "f16": 2.0 ** -10}
INF = float("inf")


def rows(seed, N, V, dtype):
    x = 2 * np.random.default_rng(seed).standard_normal((N, V))
    return torch.from_numpy(x).to(DEV).to(TYPES[dtype][1])


def space(cfg):
    return torch.empty(mg.logits_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)


def as_float(r):
    """What a float can say of a value of 64 bits."""
    return np.where(np.abs(r) > np.finfo(np.float32).max, np.sign(r) * INF, r)


def check_logprobs(x, tokens, K, dtype, temperature):
    N, V = x.shape
    cfg = mg.LogitsCfg(N, V, K, TYPES[dtype][0], temperature)
    logp, entropy, top = (torch.full(s, 9.0, device=DEV) for s in ((N,), (N,), (N, K)))
    ids = torch.full((N, K), -9, dtype=torch.int64, device=DEV)
    mg.token_logprobs(cfg, x, torch.from_numpy(tokens).to(DEV), logp, entropy, top, ids, space(cfg))
    torch.cuda.synchronize()
    ref = orc.token_logprobs(x.double().cpu().numpy(), tokens, K, float(np.float32(temperature)))
    for name, g, r in zip(("logp", "entropy", "top"), (logp, entropy, top), ref):
        g = g.cpu().numpy()
        with np.errstate(invalid="ignore"):
            r = np.where(np.isneginf(r), r, as_float(r))
        assert np.array_equal(np.isnan(g), np.isnan(r)), (name, g, r)
        assert np.array_equal(np.isneginf(g), np.isneginf(r)), (name, g, r)
        on = np.isfinite(r)
        bound = TOL / min(1.0, temperature) * np.maximum(1.0, np.abs(r[on]) / 40)
        assert np.all(np.abs(g[on] - r[on]) <= bound), (name, np.abs(g[on] - r[on]).max())
    assert np.array_equal(ids.cpu().numpy(), ref[3])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [40, 5000, 20000, 70001])
def test_masked_entries_beside_the_lowest_value(V, dtype):
    # -inf where the row's largest value is the lowest of its type, at a temperature that takes that beyond a float
    x = rows(V, 4, V, dtype)
    low = torch.finfo(TYPES[dtype][1]).min
    x[0], x[0, ::2] = low, -INF
    x[1], x[1, 1:] = low, -INF
    x[2, ::2] = -INF
    x[3, ::2] = low
    for temperature in (0.5, 1e-3, 1.0):
        check_logprobs(x, np.array([0, V - 1, 0, 1]), min(V, 12), dtype, temperature)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 20000, 70001])
@pytest.mark.parametrize("temperature", [0.1, 1e-30, 1.0, 1e30])
def test_differences_beyond_a_float(V, temperature, dtype):
    x = rows(V, 4, V, dtype)
    n = torch.arange(V, device=DEV)
    info = torch.finfo(TYPES[dtype][1])
    x[0] = torch.where(n % 3 == 0, 3e38, 1e38)               # all of one sign, far apart
    x[1] = torch.where(n % 3 == 0, -3e38, -1e38)
    x[2] = torch.where(n % 3 == 0, info.max, info.min)
    x[3] = torch.where(n % 5 == 0, info.min, -1.0)
    x[3, 1] = -INF
    check_logprobs(x, np.array([0, 1, 2, 3]), min(V, 12), dtype, temperature)
    check_logprobs(x, np.array([1, 0, 1, 1]), 3, dtype, temperature)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [7, 400])                      # held by teams, and streamed
@pytest.mark.parametrize("temperature", [1.0, 0.5])
def test_whole_segments_at_the_lowest_value(N, temperature, dtype):
    V = 70001                                                # three segments
    x = rows(N, N, V, dtype)
    low = torch.finfo(TYPES[dtype][1]).min
    x[0, 20000:] = low                                       # what a mask leaves lies in the first segment, in the last,
    x[1, :60000] = low                                       # in the middle,
    x[2, :30000], x[2, 40000:] = low, low
    x[3] = low                                               # nowhere
    x[4, :], x[4, 50000] = low, 3.0
    x[5, :40000], x[5, 40000:] = -INF, low                   # and beside segments that hold nothing at all
    check_logprobs(x, np.arange(N) * 997 % V, 9, dtype, temperature)


def distill(x, ids, t, w, dtype, temperature, apart):
    N, V = x.shape
    cfg = mg.LogitsCfg(N, V, ids.shape[1], TYPES[dtype][0], temperature)
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    loss, stats, grad = torch.full((N,), 9.0, device=DEV), torch.full((N, 2), 9.0, device=DEV), torch.full_like(x, 9.0)
    if apart:
        mg.distill_topk(cfg, x, d(ids), d(t), None, loss, stats, None, space(cfg))
        mg.distill_topk_backward(cfg, x, d(ids), d(t), stats, d(w), grad)
    else:
        mg.distill_topk(cfg, x, d(ids), d(t), d(w), loss, None, grad, space(cfg))
    torch.cuda.synchronize()
    return loss.double().cpu().numpy(), grad.double().cpu().numpy()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [50, 3000, 20000, 70001])
@pytest.mark.parametrize("temperature", [0.5, 0.01, 1.0, 50.0])
def test_teachers_at_the_ends_of_the_range(V, temperature, dtype):
    N, K = 7, 4
    x = rows(V, N, V, dtype)
    info = np.finfo(np.float32)
    ids = np.stack([np.random.default_rng(n).choice(V, K, replace=False) for n in range(N)]).astype(np.int64)
    t = np.random.default_rng(1).standard_normal((N, K)).astype(np.float32)
    t[0] = info.min                                          # all alike: a quarter each
    t[1], t[1, 2] = info.min, 1.0
    t[2] = info.max
    t[3] = info.min, info.max, info.max, -INF
    t[4] = 3e37, 3e37, -INF, 1.0
    t[5] = info.min, -INF, -INF, info.min
    w = np.linspace(0.5, 1.5, N).astype(np.float32)
    tau = float(np.float32(temperature))
    for apart in (False, True):
        loss, grad = distill(x, ids, t, w, dtype, temperature, apart)
        ref = orc.distill(x.double().cpu().numpy(), ids, t.astype(np.float64), w.astype(np.float64), tau)
        scale = 1 / min(1.0, tau)
        assert np.all(np.abs(loss - ref[0]) <= 2 * TOL * scale * np.maximum(1.0, np.abs(ref[0]) / 20)), (loss, ref[0])
        bound = UNIT[dtype] * np.abs(ref[1]) + 2 * TOL * scale * w[:, None] / tau + (2.0 ** -25 if dtype == "f16" else 0)
        assert np.all(np.abs(grad - ref[1]) <= bound)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [50, 20000, 70001])
def test_an_id_that_does_not_exist_makes_a_masked_row_nan_too(V, dtype):
    x = rows(V, 2, V, dtype)
    x[0] = -INF
    ids = np.array([[1, V], [1, 2]], np.int64)
    for apart in (False, True):
        loss, grad = distill(x, ids, np.zeros((2, 2), np.float32), np.ones(2, np.float32), dtype, 1.0, apart)
        assert np.isnan(loss[0]) and np.all(np.isnan(grad[0])) and np.all(np.isfinite(grad[1]))
