"""Product in 8-bit integers on the GPU: quantised rows equal to the definition's, sums exact, edges and strides."""
import numpy as np
import pytest
import torch

import paper_2203_04738_amd as mg
from oracle import ops_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": (mg.MGRIT_F32, torch.float32), "bf16": (mg.MGRIT_BF16, torch.bfloat16),
         "f16": (mg.MGRIT_F16, torch.float16)}
# an exact sum is rounded to float (2^-24), multiplied twice and a bias added: 4 roundings
TOL = 4 * 2.0 ** -24
UNIT = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -10}


def tokens(seed, M, K, dtype, offset=0, ld=None):
    rng = np.random.default_rng(seed)
    ld = ld or K
    mem = torch.full((offset + M * ld,), float("nan"), dtype=TYPES[dtype][1], device=DEV)
    x = mem[offset:offset + M * ld].view(M, ld)[:, :K]
    x.copy_(torch.from_numpy(rng.standard_normal((M, K)) * np.exp(rng.standard_normal((M, 1)))))
    return x


def weights(seed, N, K):
    rng = np.random.default_rng(seed)
    q = rng.integers(-128, 128, (N, mg.q8_row_bytes(K))).astype(np.int8)      # what lies beyond K does not matter
    scale = (rng.random(N) / 1000 + 1e-4).astype(np.float32)
    return q, scale, rng.standard_normal(N).astype(np.float32)


def linear(x, q, scale, bias, dtype, y=None):
    M, K = x.shape
    N = len(q)
    cfg = mg.Q8Cfg(M, N, K, TYPES[dtype][0])
    d = lambda a: None if a is None else torch.from_numpy(a).to(DEV)  # noqa: E731
    y = torch.full((M, N), float("nan"), dtype=x.dtype, device=DEV) if y is None else y
    ws = torch.empty(mg.q8_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)
    ws.fill_(77)
    mg.q8_linear(cfg, x, d(q), d(scale), d(bias), y, ws)
    torch.cuda.synchronize()
    return y.double().cpu().numpy()


def check(x, q, scale, bias, dtype, y=None):
    K = x.shape[1]
    v = x.float().cpu().numpy()
    ref = orc.q8_linear(v, q[:, :K], scale, bias)
    got = linear(x, q, scale, bias, dtype, y)
    b = 0.0 if bias is None else np.abs(bias)
    bound = TOL * (np.abs(ref) + 2 * b) + UNIT[dtype] * np.abs(ref) + (2.0 ** -25 if dtype == "f16" else 0)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    on = np.isfinite(ref)
    assert np.all(np.abs(got - ref)[on] <= bound[on]), np.max((np.abs(got - ref) - bound)[on])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K", [(1, 1), (3, 127), (5, 128), (17, 129), (4, 1000), (2, 5000), (1, 70000)])
def test_quantised_rows(M, K, dtype):
    for offset, ld in ((0, K), (1, K + 3)):
        x = tokens(K, M, K, dtype, offset, ld)
        q = torch.full((M, mg.q8_row_bytes(K)), 99, dtype=torch.int8, device=DEV)
        scale = torch.empty(M, device=DEV)
        mg.q8_quantize(mg.Q8Cfg(M, 1, K, TYPES[dtype][0]), x, q, scale)
        torch.cuda.synchronize()
        rq, rs = orc.q8_quantize(x.float().cpu().numpy())
        assert np.array_equal(scale.cpu().numpy(), rs)
        assert np.array_equal(q[:, :K].cpu().numpy(), rq)
        assert torch.all(q[:, K:] == 0)


def test_rows_of_odd_values():
    K = 300
    x = tokens(1, 8, K, "f32")
    x[0] = 0
    x[1, 5] = float("inf")
    x[2, 7] = float("nan")
    x[3] *= 1e-42                                    # below what a scale can be: 2^-126 serves
    x[4] *= 1e35
    x[5] = -2.5
    x[6, 1:] = 0
    x[7, 0] = -float("inf")
    q = torch.empty(8, mg.q8_row_bytes(K), dtype=torch.int8, device=DEV)
    scale = torch.empty(8, device=DEV)
    mg.q8_quantize(mg.Q8Cfg(8, 1, K), x, q, scale)
    rq, rs = orc.q8_quantize(x.cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), rs, equal_nan=True)
    assert np.array_equal(q[:, :K].cpu().numpy(), rq)
    w = weights(1, 70, K)
    x[3] = 1.0                                       # (products of such scales are below float's normal numbers)
    check(x, *w, "f32")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [1, 7, 16, 17, 33, 64, 65, 130, 300])
@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (50, 100), (129, 257), (500, 1030)])
def test_sizes(M, N, K, dtype):
    check(tokens(M + K, M, K, dtype), *weights(N, N, K), dtype)


@pytest.mark.parametrize("M,N,K", [(1, 4100, 4096), (9, 300, 20000), (513, 770, 640), (2048, 1024, 1024), (1025, 2100, 130),
                                   (48, 2048, 8192), (2100, 70, 1500), (8000, 2040, 200)])
def test_larger_sizes(M, N, K):
    check(tokens(M, M, K, "bf16"), *weights(N, N, K), "bf16")
    q, scale, _ = weights(N, N, K)
    check(tokens(M, M, K, "f32"), q, scale, None, "f32")


def test_the_largest_sums():
    # every product -128 * 127 over the longest rows: the sum is within 32 bits
    K = 131072
    x = torch.ones(2, K, device=DEV)
    q = np.full((20, K), -128, np.int8)
    got = linear(x, q, np.ones(20, np.float32), None, "f32")
    scale = np.float32(1) * (np.float32(1) / np.float32(127))
    assert np.all(np.abs(got + 128.0 * 127 * K * float(scale)) <= TOL * 128 * K)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [3, 40, 200])
def test_strides_and_what_lies_beside(M, dtype):
    N, K = 77, 210
    x = tokens(2, M, K, dtype, 3, K + 5)
    mem = torch.full((M * (N + 3) + 1,), 7.0, dtype=x.dtype, device=DEV)
    y = mem[1:].view(M, N + 3)[:, :N]
    check(x, *weights(2, N, K), dtype, y)
    assert torch.all(mem[1:].view(M, N + 3)[:, N:] == 7) and mem[0] == 7


@pytest.mark.parametrize("M", [3, 130])
def test_rows_beyond_32_bit_offsets(M):
    N, K = 70, 300
    ld = ((3 << 30) // M + 8) // 4 * 4                # bf16 rows over 6 GB in all, of tokens and of results
    x = torch.as_strided(torch.empty((M - 1) * ld + K, dtype=torch.bfloat16, device=DEV), (M, K), (ld, 1))
    x.copy_(tokens(1, M, K, "bf16"))
    y = torch.as_strided(torch.empty((M - 1) * ld + N, dtype=torch.bfloat16, device=DEV), (M, N), (ld, 1))
    check(x, *weights(1, N, K), "bf16", y)
