"""Token log probabilities and the distillation loss on the GPU against the float64 oracle: types, widths around the teams and
segments, rows that start anywhere, ties, masks that leave little or nothing, values that are not finite."""
import numpy as np
import pytest
import torch

import paper_2203_04738_amd as mg
from oracle import ops_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": (mg.MGRIT_F32, torch.float32), "bf16": (mg.MGRIT_BF16, torch.bfloat16),
         "f16": (mg.MGRIT_F16, torch.float16)}
# log p = (x - max) / t - log s: a difference of up to some 40, its product with 1/t and the logarithm, each rounded to 2^-24 of
# 40 or less: 3 * 40 * 2^-24 = 7e-6; sums of exponentials, each to (40 log2 e + 3) 2^-24 = 4e-6 of itself
TOL = 1.2e-5
UNIT = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8, "f16": 2.0 ** -10}
INF = float("inf")


def rows(seed, N, V, dtype, offset=0, ld=None):
    """(device view [N,V], its values): a view `offset` elements into its memory, rows `ld` apart."""
    rng = np.random.default_rng(seed)
    ld = ld or V
    mem = torch.full((offset + N * ld,), float("nan"), dtype=TYPES[dtype][1], device=DEV)   # nothing else may be read
    x = mem[offset:offset + N * ld].view(N, ld)[:, :V]
    x.copy_(torch.from_numpy(2 * rng.standard_normal((N, V))))
    return x, mem


def values(x):
    return x.double().cpu().numpy()


def space(cfg):
    return torch.empty(mg.logits_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)


def logprobs(x, tokens, K, dtype, temperature=1.0):
    N, V = x.shape
    cfg = mg.LogitsCfg(N, V, K, TYPES[dtype][0], temperature)
    logp, entropy = torch.full((N,), 9.0, device=DEV), torch.full((N,), 9.0, device=DEV)
    top = torch.full((N, K), 9.0, device=DEV) if K else None
    ids = torch.full((N, K), -9, dtype=torch.int64, device=DEV) if K else None
    mg.token_logprobs(cfg, x, torch.from_numpy(tokens).to(DEV), logp, entropy, top, ids, space(cfg))
    torch.cuda.synchronize()
    return [None if t is None else t.cpu().numpy() for t in (logp, entropy, top, ids)]


def check_logprobs(x, tokens, K, dtype, temperature=1.0, ids_too=True):
    got = logprobs(x, tokens, K, dtype, temperature)
    ref = orc.token_logprobs(values(x), tokens, K, temperature)
    for name, g, r in zip(("logp", "entropy", "top"), got, ref):
        if g is None:
            continue
        r = np.where(np.abs(r) > np.finfo(np.float32).max, np.sign(r) * INF, r)   # (what a float can say)
        assert np.array_equal(np.isnan(g), np.isnan(r)), name
        assert np.array_equal(np.isneginf(g), np.isneginf(r)), name
        on = np.isfinite(r)
        bound = TOL / min(1.0, temperature) * np.maximum(1.0, np.abs(r[on]) / 40)   # (TOL: log p down to -40)
        assert np.all(np.abs(g[on] - r[on]) <= bound), (name, np.abs(g[on] - r[on]).max())
    if K and ids_too:
        assert np.array_equal(got[3], ref[3])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,K", [(1, 1), (2, 2), (51, 5), (63, 63), (511, 64), (1024, 20), (1025, 20), (8192, 64), (8200, 1),
                                 (32768, 64), (32775, 33), (70001, 64)])
def test_widths(V, K, dtype):
    N = 5
    x, _ = rows(V, N, V, dtype)
    tokens = np.array([0, V - 1, V // 2, -1, V])
    check_logprobs(x, tokens, K, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset,pad", [(1, 0), (3, 5), (8, 3), (7, 1)])
@pytest.mark.parametrize("V", [9, 1020, 8190, 32766, 40000])
def test_rows_that_start_anywhere(V, offset, pad, dtype):
    x, _ = rows(V + offset, 4, V, dtype, offset, V + pad)
    check_logprobs(x, np.array([0, 1, V - 1, -5]), min(V, 10), dtype, temperature=0.7)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [40, 900, 5000, 20000, 100000])
def test_ties_and_masks(V, dtype):
    N, K = 9, 13
    x, _ = rows(1, N, V, dtype)
    low = torch.finfo(TYPES[dtype][1]).min
    x[0] = 1.5                                       # one value everywhere
    x[1] = -INF                                      # nothing left
    x[2] = low
    x[3] = -INF
    x[3, V - 3] = 0.25                               # one, near the end
    x[4] = torch.where(torch.arange(V, device=DEV) % 7 == 3, x[4], -INF)
    x[5] = torch.where(torch.arange(V, device=DEV) % 5 == 3, x[5], low)
    x[6] = x[6].round()                              # many ties
    x[7] = torch.where(x[7] > 0, 0.0, -0.0)          # zeros of both signs tie
    x[8, ::2] = -INF
    check_logprobs(x, np.array([0, V - 1, 3, V - 3, 3, 3, 1, 2, 0]), K, dtype)
    check_logprobs(x, np.full(N, V - 3), 0, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [40, 5000, 20000, 100000])
def test_rows_that_are_not_finite_stay_by_themselves(V, dtype):
    x, _ = rows(2, 5, V, dtype)
    x[1, V // 2] = float("nan")
    x[3, V - 1] = INF
    x[4] = float("nan")
    check_logprobs(x, np.array([1, 2, 3, 4, 5]), 7, dtype, ids_too=False)
    ids = logprobs(x, np.array([1, 2, 3, 4, 5]), 7, dtype)[3]
    assert ids[1, 0] == V // 2 and ids[3, 0] == V - 1 and np.array_equal(ids[4], np.arange(7))


def test_some_outputs_are_left_out():
    x, _ = rows(3, 4, 60000, "bf16")
    full = logprobs(x, np.array([1, 2, 3, 4]), 5, "bf16")
    cfg = mg.LogitsCfg(4, 60000, 5, mg.MGRIT_BF16)
    top, ids = torch.empty(4, 5, device=DEV), torch.empty(4, 5, dtype=torch.int64, device=DEV)
    mg.token_logprobs(cfg, x, None, None, None, top, ids, space(cfg))
    assert np.array_equal(top.cpu().numpy(), full[2]) and np.array_equal(ids.cpu().numpy(), full[3])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,offset,pad", [(800, 9000, 0, 0), (800, 8193, 3, 6), (400, 33001, 1, 2)])
def test_many_long_rows(N, V, offset, pad, dtype):
    x, _ = rows(N, N, V, dtype, offset, V + pad)
    low = torch.finfo(TYPES[dtype][1]).min
    x[0], x[1], x[2], x[3] = 0.5, -INF, low, -INF
    x[3, V - 2] = 2.0
    x[4, : V // 2] = -INF                            # whole pieces, also the first, that a mask leaves out
    x[5, : V // 2] = low
    x[6] = x[6].round()
    x[7, 3000:] += 60                                # the reference moves on the way
    x[8, :3000] += 60
    x[9, 5], x[10, 6] = float("nan"), INF
    tokens = np.arange(N) * 7 % V
    tokens[20:30] = -1
    check_logprobs(x, tokens, 20, dtype, temperature=0.7, ids_too=False)
    keep = [n for n in range(N) if n not in (9, 10)]
    ids = logprobs(x, tokens, 20, dtype, 0.7)[3]
    ref = orc.token_logprobs(values(x), tokens, 20, 0.7)[3]
    assert np.array_equal(ids[keep], ref[keep])
    assert ids[9, 0] == 5 and ids[10, 0] == 6


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [3, 800])
@pytest.mark.parametrize("temperature", [1.0, 4.0])
def test_values_of_the_types_whole_range(N, temperature, dtype):
    V = 9000
    x, _ = rows(N, N, V, dtype)
    info = torch.finfo(TYPES[dtype][1])
    x[0] = info.min
    x[1] = torch.where(torch.arange(V, device=DEV) % 3 == 0, info.max, info.min)
    x[2] = x[2] * 3000
    x[2, 77] = info.min
    check_logprobs(x, np.arange(N), 5, dtype, temperature)
    ids, t = teacher(1, N, V, 4)
    w = np.ones(N, np.float32)
    loss, grad = distill(x, ids, t, w, dtype, temperature)
    ref = orc.distill(values(x), ids, t.astype(np.float64), w.astype(np.float64), temperature)
    beyond = ref[0] > np.finfo(np.float32).max               # (what a float can say)
    assert np.all(loss[beyond] == INF)
    assert np.all((np.abs(loss - ref[0]) <= 2 * TOL * np.maximum(1.0, np.abs(ref[0]) / 20))[~beyond])
    assert np.all(np.abs(grad - ref[1]) <= UNIT[dtype] * np.abs(ref[1]) + 2 * TOL / temperature)


# ---------------------------------------------------------------------------
def teacher(seed, N, V, K):
    rng = np.random.default_rng(seed)
    ids = np.stack([rng.choice(V, K, replace=V < K) for _ in range(N)])
    return ids.astype(np.int64), (2 * rng.standard_normal((N, K))).astype(np.float32)


def distill(x, ids, t, w, dtype, temperature=1.0, apart=False, in_place=False, grad_mem=None):
    N, V = x.shape
    cfg = mg.LogitsCfg(N, V, ids.shape[1], TYPES[dtype][0], temperature)
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    loss, stats = torch.full((N,), 9.0, device=DEV), torch.full((N, 2), 9.0, device=DEV)
    grad = x if in_place else grad_mem if grad_mem is not None else torch.full_like(x, 9.0)
    if apart:
        mg.distill_topk(cfg, x, d(ids), d(t), None, loss, stats, None, space(cfg))
        mg.distill_topk_backward(cfg, x, d(ids), d(t), stats, d(w), grad)
    else:
        mg.distill_topk(cfg, x, d(ids), d(t), d(w), loss, None, grad, space(cfg))
    torch.cuda.synchronize()
    return loss.double().cpu().numpy(), values(grad)


def check_distill(x, ids, t, w, dtype, temperature=1.0, **kw):
    v = values(x)
    ref = orc.distill(v, ids, t.astype(np.float64), w.astype(np.float64), temperature)
    for apart in (False, True):
        y = x.clone() if kw.get("in_place") else x
        loss, grad = distill(y, ids, t, w, dtype, temperature, apart=apart, **kw)
        assert np.array_equal(np.isfinite(loss), np.isfinite(ref[0])) and np.array_equal(np.isnan(loss), np.isnan(ref[0]))
        on = np.isfinite(ref[0])
        assert np.all(np.abs(loss[on] - ref[0][on]) <= 2 * TOL / min(1.0, temperature))
        assert np.array_equal(np.isnan(grad), np.isnan(ref[1]))
        g, r = np.nan_to_num(grad), np.nan_to_num(ref[1])
        scale = (np.abs(w) / temperature)[:, None]
        # (16-bit fractions below the type's smallest normal number are rounded to its smallest step)
        tiny = 2.0 ** -25 if dtype == "f16" else 0.0
        # probabilities are at most 1, each known to TOL of itself (to more of it at a low temperature)
        bound = UNIT[dtype] * np.abs(r) + TOL / min(1.0, temperature) * np.maximum(np.abs(r), scale * 2.0 ** -23)
        bound = bound + TOL * scale * (np.abs(r) > 0) * 2.0 ** -3 + tiny
        assert np.all(np.abs(g - r) <= bound), (apart, np.max(np.abs(g - r) - bound))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,K", [(1, 1), (2, 2), (51, 5), (700, 256), (1025, 64), (8192, 1), (20000, 70), (32768, 64),
                                 (32775, 3), (70001, 200)])
def test_distillation_widths(V, K, dtype):
    N = 5
    x, _ = rows(V, N, V, dtype)
    ids, t = teacher(V, N, V, K)
    w = np.array([1.0, 0.5, -2.0, 0.0, 1e-3], np.float32)
    check_distill(x, ids, t, w, dtype, temperature=2.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [50, 3000, 32760, 50021])
def test_distillation_of_strided_rows_and_in_place(V, dtype):
    N, K = 4, 6
    x, mem = rows(8, N, V, dtype, 3, V + 5)
    ids, t = teacher(8, N, V, K)
    w = np.ones(N, np.float32)
    check_distill(x, ids, t, w, dtype)
    check_distill(x, ids, t, w, dtype, in_place=True)
    other = torch.full((N * (V + 2) + 1,), 7.0, dtype=x.dtype, device=DEV)       # rows that start elsewhere
    grad = other[1:].view(N, V + 2)[:, :V]
    check_distill(x, ids, t, w, dtype, grad_mem=grad)
    assert torch.all(other[1:].view(N, V + 2)[:, V:] == 7) and other[0] == 7     # and nothing besides
    assert torch.isnan(mem[:3]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [50, 3000, 20000, 70000])
def test_distillation_of_rows_with_little_in_them(V, dtype):
    N, K = 11, 5
    x, _ = rows(4, N, V, dtype)
    ids, t = teacher(4, N, V, K)
    ids[0] = -1                                      # no teacher
    ids[1, 2:] = -7                                  # a short list
    ids[2] = ids[2, 0]                               # one id five times
    ids[3, 3] = ids[3, 1]
    t[4] = -INF                                      # entries without weight
    t[5, 1:] = -INF
    x[6] = -INF                                      # a student with nothing left
    x[7, int(ids[7, 0])] = -INF                      # the student forbids what the teacher says
    t[8, 0] = -INF
    x[8, int(ids[8, 0])] = -INF                      # ... and where the teacher gives it no weight
    ids[9, 1] = V                                    # not an id
    x[10] = torch.finfo(TYPES[dtype][1]).min
    check_distill(x, ids, t, np.linspace(0.5, 1.5, N).astype(np.float32), dtype)
    # rows of weight zero have no gradient, whatever they hold
    x[1, 3], x[2, 0] = float("nan"), INF
    loss, grad = distill(x, ids, t, np.zeros(N, np.float32), dtype)
    assert np.all(grad == 0) and np.isnan(loss[[1, 2, 9]]).all()
    # without a teacher neither, also where the student is not finite
    x[0, 5] = float("nan")
    loss, grad = distill(x, ids, t, np.ones(N, np.float32), dtype)
    assert loss[0] == 0 and np.all(grad[0] == 0) and np.all(np.isnan(grad[1]))


def test_distillation_gradient_against_differences():
    # central differences of the float64 oracle's loss
    N, V, K, eps = 3, 300, 9, 1e-5
    x, _ = rows(6, N, V, "f32")
    ids, t = teacher(6, N, V, K)
    _, grad = distill(x, ids, t, np.ones(N, np.float32), "f32", 0.7)
    v = values(x)
    for n, j in [(0, int(ids[0, 0])), (0, 7), (1, int(ids[1, 3])), (2, 299)]:
        up, down = v.copy(), v.copy()
        up[n, j] += eps
        down[n, j] -= eps
        loss = lambda y: orc.distill(y, ids, t.astype(np.float64), np.ones(N), 0.7)[0][n]  # noqa: E731
        assert abs((loss(up) - loss(down)) / (2 * eps) - grad[n, j]) <= 1e-8 + 2 * TOL


def test_cross_entropy_is_one_teacher_entry():
    N, V = 6, 51
    x, _ = rows(7, N, V, "f32")
    labels = np.arange(N, dtype=np.int64)
    loss, grad = distill(x, labels[:, None], np.zeros((N, 1), np.float32), np.ones(N, np.float32), "f32")
    y = torch.from_numpy(values(x)).requires_grad_(True)
    ref = torch.nn.functional.cross_entropy(y, torch.from_numpy(labels), reduction="none")
    ref.sum().backward()
    assert np.all(np.abs(loss - ref.detach().numpy()) <= 2 * TOL)
    assert np.all(np.abs(grad - y.grad.numpy()) <= TOL)


def test_graph_replays_and_repeats_give_the_same_bits():
    N, V, K = 64, 70000, 16
    x, _ = rows(9, N, V, "bf16")
    ids, t = teacher(9, N, V, K)
    first = distill(x, ids, t, np.ones(N, np.float32), "bf16")
    tops = logprobs(x, np.arange(N), K, "bf16")
    cfg = mg.LogitsCfg(N, V, K, mg.MGRIT_BF16)
    ws, loss, grad = space(cfg), torch.empty(N, device=DEV), torch.empty_like(x)
    logp, top, top_ids = torch.empty(N, device=DEV), torch.empty(N, K, device=DEV), torch.empty(N, K, dtype=torch.int64, device=DEV)
    dids, dt, tok = torch.from_numpy(ids).to(DEV), torch.from_numpy(t).to(DEV), torch.arange(N, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mg.distill_topk(cfg, x, dids, dt, None, loss, None, grad, ws)
        mg.token_logprobs(cfg, x, tok, logp, None, top, top_ids, ws)
    for _ in range(3):
        for a in (loss, grad, logp, top):
            a.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(loss.double().cpu().numpy(), first[0]) and np.array_equal(values(grad), first[1])
        assert np.array_equal(logp.cpu().numpy(), tops[0]) and np.array_equal(top.cpu().numpy(), tops[2])
        assert np.array_equal(top_ids.cpu().numpy(), tops[3])
        grad.float().abs().sum().item()


def test_rows_beyond_32_bit_offsets():
    N, V, ld = 3, 9000, (1 << 30) + 3                 # bf16 rows 2 GB apart
    mem = torch.empty((N - 1) * ld + V, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(mem, (N, V), (ld, 1))
    x.copy_(rows(5, N, V, "bf16")[0])
    check_logprobs(x, np.array([0, V - 1, 77]), 9, "bf16")
    ids, t = teacher(5, N, V, 7)
    y = x.clone()
    loss, grad = distill(x, ids, t, np.ones(N, np.float32), "bf16", in_place=True)
    ref = distill(y, ids, t, np.ones(N, np.float32), "bf16")
    assert np.array_equal(loss, ref[0]) and np.array_equal(grad, ref[1])
