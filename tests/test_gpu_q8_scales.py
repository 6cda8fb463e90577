"""Scales of the product in 8-bit integers: a row's largest magnitude over 127, rounded once, and products of scales at the
ends of the range."""
import numpy as np
import pytest
import torch

import paper_2203_04738_amd as mg
from oracle import ops_oracle as orc

DEV = "cuda:0"
TYPES = {"f32": (mg.MGRIT_F32, torch.float32), "bf16": (mg.MGRIT_BF16, torch.bfloat16),
         "f16": (mg.MGRIT_F16, torch.float16)}


def halves():
    """A row for every bf16 significand: its largest value, half of that (a tie, but for the scale's rounding), others."""
    top = (128 + np.arange(128)).astype(np.float32)[:, None]
    return np.concatenate([top, top / 2, -top / 2, top / 4, -top / 8, np.zeros_like(top)], 1) / 256


def test_the_oracles_scale_is_the_quotient_rounded_once():
    x = np.concatenate([halves(), np.random.default_rng(0).standard_normal((500, 6)).astype(np.float32)])
    q, scale = orc.q8_quantize(x)
    top = np.abs(x).max(1)
    # the float nearest to top / 127: the quotient in 64 bits is nowhere near half way between two floats
    assert np.array_equal(scale, (top.astype(np.float64) / 127).astype(np.float32))
    assert np.array_equal(q[:128], np.rint(x[:128] / scale[:128, None]))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,M", [(6, 128), (700, 128), (1500, 2176), (3000, 128), (9000, 128), (40000, 128)])
def test_quantised_ties(K, M, dtype):
    x = np.zeros((M, K), np.float32)
    x[:, K - 6:] = np.tile(halves(), (M // 128, 1))
    d = torch.from_numpy(x).to(DEV).to(TYPES[dtype][1])
    assert np.array_equal(d.float().cpu().numpy(), x)
    q, scale = torch.empty(M, mg.q8_row_bytes(K), dtype=torch.int8, device=DEV), torch.empty(M, device=DEV)
    mg.q8_quantize(mg.Q8Cfg(M, 1, K, TYPES[dtype][0]), d, q, scale)
    rs = (np.abs(x).max(1).astype(np.float64) / 127).astype(np.float32)
    assert np.array_equal(scale.cpu().numpy(), rs)
    assert np.array_equal(q[:, :K].cpu().numpy(), np.rint(x / rs[:, None]))


def product(x, q, scale, dtype="f32"):
    M, K = x.shape
    cfg = mg.Q8Cfg(M, len(q), K, TYPES[dtype][0])
    y = torch.empty(M, len(q), dtype=x.dtype, device=DEV)
    mg.q8_linear(cfg, x, torch.from_numpy(q).to(DEV), torch.from_numpy(scale).to(DEV), None, y,
                 torch.empty(mg.q8_workspace_bytes(cfg), dtype=torch.uint8, device=DEV))
    return y.double().cpu().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 40, 130, 3000])            # in one launch, few tokens, tiles
def test_ties_in_a_product(M):
    rng = np.random.default_rng(M)
    x = np.tile(halves(), (M // 128 + 1, 1))[rng.permutation(M) if M > 128 else rng.choice(128, M, replace=False)]
    x = np.concatenate([x, np.tile(x, (1, 5))], 1)
    q = rng.integers(-128, 128, (70, mg.q8_row_bytes(x.shape[1]))).astype(np.int8)
    scale = (rng.random(70) / 1000 + 1e-4).astype(np.float32)
    ref = orc.q8_linear(x, q[:, :x.shape[1]], scale)
    got = product(torch.from_numpy(x).to(DEV), q, scale)
    assert np.all(np.abs(got - ref) <= 4 * 2.0 ** -24 * np.abs(ref))    # an exact sum, rounded and multiplied twice


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 40, 130, 3000])
def test_large_tokens_and_small_weights(M):
    # tokens near a float's largest: sums times the token's scale alone would be beyond it
    rng = np.random.default_rng(M)
    K = 300
    x = (rng.uniform(-1, 1, (M, K)) * 3e38).astype(np.float32)
    q = rng.integers(-128, 128, (70, mg.q8_row_bytes(K))).astype(np.int8)
    scale = (rng.random(70) * 1e-9 + 1e-10).astype(np.float32)
    ref = orc.q8_linear(x, q[:, :K], scale)
    assert np.abs(ref / scale).max() > np.finfo(np.float32).max > np.abs(ref).max()
    got = product(torch.from_numpy(x).to(DEV), q, scale)
    assert np.all(np.abs(got - ref) <= 4 * 2.0 ** -24 * np.abs(ref))
