"""Causal convolution on the GPU against the float64 oracle: types, taps, lengths around the runs and segments, strides, resets,
the past handed on, gradients, one step at a time."""
import numpy as np
import pytest
import torch

import paper_2203_04738_amd as mg
from oracle import token_ops_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": (mg.MGRIT_F32, torch.float32, 2.0 ** -24), "bf16": (mg.MGRIT_BF16, torch.bfloat16, 2.0 ** -8),
         "f16": (mg.MGRIT_F16, torch.float16, 2.0 ** -11)}
# a sum of at most 9 products and a sigmoid known to some units of 2^-24, of terms that add up to some times the largest
# result: (9 + 8) 2^-24 times 5; gradients multiply two such values, and sums of them run through 64 steps of a segment and
# some levels: (64 + 20) 2^-24 times 5
TOL, GRAD_TOL = 5e-6, 2.5e-5


def close(got, want, unit, tol):
    got = got.double().cpu().numpy()
    assert got.shape == want.shape
    if want.size == 0:
        return
    err = np.abs(got - want)
    assert (err <= unit * np.abs(want) + tol * max(np.abs(want).max(), 1e-30)).all(), float(err.max() / np.abs(want).max())


def problem(seed, T, B, H, W, dtype, batch_first=False, resets=0.0, offset=0):
    rng = np.random.default_rng(seed)
    dt = TYPES[dtype][1]
    d, dev = {}, {}

    def seq(name, width, at):
        buf = torch.full((B, T, width) if batch_first else (T, B, width), float("nan"), dtype=dt, device=DEV)
        view = (buf.transpose(0, 1) if batch_first else buf)[..., at:at + H]
        view.copy_(torch.from_numpy(rng.standard_normal((T, B, H))))
        dev[name], d[name] = view, view.double().cpu().numpy()

    seq("x", 2 * H + offset, offset)
    seq("dy", H, 0)
    for name, shape in (("weight", (H, W)), ("bias", (H,)), ("past", (B, W - 1, H)), ("dlast", (B, W - 1, H))):
        v = rng.standard_normal(shape).astype(np.float32)
        d[name], dev[name] = v.astype(np.float64), torch.from_numpy(v).to(DEV)
    d["reset"] = (rng.random((T, B)) < resets).astype(np.uint8) if resets else None
    dev["reset"] = torch.from_numpy(d["reset"]).to(DEV) if resets else None
    return d, dev


def run(d, dev, T, B, H, W, dtype, silu=True, with_past=True, batch_first=False):
    code, dt, unit = TYPES[dtype]
    cfg = mg.ConvCfg(T, B, H, W, mg.CONV_SILU if silu else mg.CONV_LINEAR, code)
    nan = float("nan")
    seq = lambda: (lambda b: b.transpose(0, 1) if batch_first else b)(  # noqa: E731
        torch.full((B, T, H) if batch_first else (T, B, H), nan, dtype=dt, device=DEV))
    y, dx = seq(), seq()
    new = lambda *s: torch.full(s, nan, device=DEV)  # noqa: E731
    last, dw, db, dp = new(B, W - 1, H), new(H, W), new(H), new(B, W - 1, H)
    past, dlast = (dev["past"], dev["dlast"]) if with_past else (None, None)
    bias = dev["bias"] if with_past else None
    mg.causal_conv_forward(cfg, dev["x"], dev["weight"], bias, past, dev["reset"], y, last)
    ws = torch.full((mg.causal_conv_workspace_bytes(cfg),), 255, dtype=torch.uint8, device=DEV)
    mg.causal_conv_backward(cfg, dev["x"], dev["weight"], bias, past, dev["reset"], dev["dy"], dlast, dx, dw, db, dp, ws)
    torch.cuda.synchronize()
    np_past, np_dlast, np_bias = (d["past"], d["dlast"], d["bias"]) if with_past else (None, None, None)
    wy, wl, _ = orc.conv_forward(d["x"], d["weight"], np_bias, np_past, d["reset"], silu)
    g = orc.conv_backward(d["x"], d["weight"], np_bias, d["dy"], np_past, d["reset"], silu, np_dlast)
    close(y, wy, unit, TOL)
    close(last, wl, 0, 0)
    for got, want, u in zip((dx, dw, db, dp), g, (unit, 0, 0, 0)):
        close(got, want, u, GRAD_TOL)
    return y, last, dx, dw, db, dp


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("T,B,H,W", [(1, 1, 1, 1), (1, 2, 3, 4), (2, 1, 6, 5), (16, 2, 33, 2), (17, 1, 64, 3), (61, 2, 130, 4),
                                     (62, 1, 30, 4), (57, 3, 16, 8), (58, 1, 7, 7), (130, 2, 34, 6), (125, 1, 100, 4), (150, 2, 9, 1)])
def test_shapes(dtype, T, B, H, W):
    run(*problem(T * 7 + H, T, B, H, W, dtype), T, B, H, W, dtype)


@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("with_past", [True, False])
@pytest.mark.parametrize("resets", [0.0, 0.3, 1.0])
@pytest.mark.parametrize("T,W,batch_first,offset", [(70, 4, False, 0), (3, 6, True, 1), (140, 3, True, 0), (64, 1, False, 1)])
def test_options(silu, with_past, resets, T, W, batch_first, offset):
    B, H = 2, 20
    d, dev = problem(T + W, T, B, H, W, "f32", batch_first, resets, offset)
    run(d, dev, T, B, H, W, "f32", silu, with_past, batch_first)


def test_long_and_many_rows():
    # several segments of one thread, several groups of one channel tile
    run(*problem(5, 400, 40, 6, 4, "bf16", resets=0.02), 400, 40, 6, 4, "bf16")


@pytest.mark.parametrize("low", [-3e38, -1e30, -200.0])
def test_the_activation_of_the_lowest_values_is_0(low):
    """p sigmoid(p) and its slope are 0 to within 1e-36 from p = -89 on, whatever p."""
    d, dev = problem(31, 50, 2, 24, 4, "f32")
    dev["bias"][::3] = low
    d["bias"] = dev["bias"].double().cpu().numpy()
    y, _, dx, dw, db, _ = run(d, dev, 50, 2, 24, 4, "f32")
    assert (y[..., ::3].abs() <= 1e-30).all() and (dw[::3].abs() <= 1e-30).all() and (db[::3].abs() <= 1e-30).all()


def test_what_a_reset_forgets_may_be_anything():
    T, B, H, W = 40, 2, 10, 4
    d, dev = problem(9, T, B, H, W, "f32")
    dev["x"][:20] = float("nan")
    dev["past"].fill_(float("inf"))
    reset = torch.zeros(T, B, dtype=torch.uint8, device=DEV)
    reset[20] = 255
    cfg = mg.ConvCfg(T, B, H, W)
    y, last = torch.empty(T, B, H, device=DEV), torch.empty(B, W - 1, H, device=DEV)
    mg.causal_conv_forward(cfg, dev["x"], dev["weight"], dev["bias"], dev["past"], reset, y, last)
    want, _, _ = orc.conv_forward(d["x"][20:], d["weight"], d["bias"])
    close(y[20:], want, 2.0 ** -24, TOL)
    assert torch.isnan(y[:20]).all() and torch.isfinite(last).all()


def test_a_sequence_in_pieces():
    T, B, H, W = 50, 3, 18, 4
    d, dev = problem(11, T, B, H, W, "f32", resets=0.05)
    whole, last = torch.empty(T, B, H, device=DEV), torch.empty(B, W - 1, H, device=DEV)
    mg.causal_conv_forward(mg.ConvCfg(T, B, H, W), dev["x"], dev["weight"], dev["bias"], dev["past"], dev["reset"], whole, last)
    past, out, t = dev["past"], [], 0
    for n in (1, 2, 20, 1, 26):
        y, nxt = torch.empty(n, B, H, device=DEV), torch.empty(B, W - 1, H, device=DEV)
        mg.causal_conv_forward(mg.ConvCfg(n, B, H, W), dev["x"][t:t + n], dev["weight"], dev["bias"], past,
                               dev["reset"][t:t + n].contiguous(), y, nxt)
        past, t = nxt, t + n
        out.append(y)
    assert torch.equal(torch.cat(out), whole) and torch.equal(past, last)


@pytest.mark.parametrize("dtype,W,silu", [("f32", 4, True), ("bf16", 2, True), ("f16", 1, False), ("f32", 8, False)])
def test_steps_on_a_pool(dtype, W, silu):
    T, B, H, n = 12, 4, 50, 7
    code, dt, unit = TYPES[dtype]
    d, dev = problem(13, T, B, H, W, dtype, resets=0.2)
    cfg = mg.ConvCfg(1, B, H, W, mg.CONV_SILU if silu else mg.CONV_LINEAR, code)
    pool = torch.full((n, W - 1, H), 5.0, device=DEV)
    slots = torch.tensor([6, 0, 9, 2], dtype=torch.int32, device=DEV)
    for row in (0, 1, 3):
        pool[int(slots[row])] = dev["past"][row]
    out = []
    for t in range(T):
        y = torch.full((B, H), float("nan"), dtype=dt, device=DEV)
        mg.causal_conv_step(cfg, dev["x"][t], dev["weight"], dev["bias"], slots, dev["reset"][t], pool, pool, y)
        out.append(y)
    want, last, _ = orc.conv_forward(d["x"], d["weight"], d["bias"], d["past"], d["reset"], silu)
    live = [0, 1, 3]
    close(torch.stack(out)[:, live], want[:, live], unit, TOL)
    close(pool[slots[live].long()], last[live], 0, 0)
    assert (torch.stack(out)[:, 2] == 0).all() and (pool[[1, 3, 4, 5]] == 5).all()


def test_some_gradients_only_and_by_differences():
    T, B, H, W = 30, 2, 5, 4
    d, dev = problem(17, T, B, H, W, "f32", resets=0.1)
    cfg = mg.ConvCfg(T, B, H, W)
    ws = torch.empty(mg.causal_conv_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)
    dx, dw = torch.empty(T, B, H, device=DEV), torch.empty(H, W, device=DEV)
    mg.causal_conv_backward(cfg, dev["x"], dev["weight"], dev["bias"], None, dev["reset"], dev["dy"], None, dx, None, None, None,
                            ws)
    mg.causal_conv_backward(cfg, dev["x"], dev["weight"], dev["bias"], None, dev["reset"], dev["dy"], None, dx, dw, None, None,
                            ws)

    def loss(w):
        y = torch.empty(T, B, H, device=DEV)
        mg.causal_conv_forward(cfg, dev["x"], w, dev["bias"], None, dev["reset"], y, None)
        return float((y.double() * dev["dy"].double()).sum())

    # central differences of step 1e-2: its square times the third derivative (some units), and 600 values known to 1e-6 over
    # the step
    e = 1e-2
    for at in ((0, 0), (2, 3), (4, 1)):
        up, down = dev["weight"].clone(), dev["weight"].clone()
        up[at] += e
        down[at] -= e
        num = (loss(up) - loss(down)) / (float(up[at]) - float(down[at]))
        assert abs(num - float(dw[at])) <= 5e-3 * max(1.0, float(dw.abs().max()))


def test_the_same_bits_in_every_run_and_in_a_graph():
    T, B, H, W = 300, 3, 70, 4
    d, dev = problem(19, T, B, H, W, "bf16", resets=0.02)
    cfg = mg.ConvCfg(T, B, H, W, mg.CONV_SILU, mg.MGRIT_BF16)
    ws = torch.empty(mg.causal_conv_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)
    new = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device=DEV)  # noqa: E731
    bf = torch.bfloat16
    out = [new(T, B, H, dtype=bf), new(B, W - 1, H), new(T, B, H, dtype=bf), new(H, W), new(H), new(B, W - 1, H)]

    def both():
        given = (dev["x"], dev["weight"], dev["bias"], dev["past"], dev["reset"])
        mg.causal_conv_forward(cfg, *given, out[0], out[1])
        mg.causal_conv_backward(cfg, *given, dev["dy"], dev["dlast"], *out[2:], ws)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        dev["x"].mul_(-0.9)
        for t in out:
            t.zero_()
        both()
        eager = [t.clone() for t in out]
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, out):
            assert torch.equal(a, b) and float(a.abs().max()) > 0


@pytest.mark.parametrize("slots", [None, [2, -1, 0, 70000]])
def test_steps_of_one_tap_have_no_pool(slots):
    """W = 1: no past is looked at, so that none has to be there; without a pool only a negative slot is outside of it."""
    B, H = 4, 50
    d, dev = problem(14, 1, B, H, 1, "f32")
    cfg = mg.ConvCfg(1, B, H, 1)
    s = None if slots is None else torch.tensor(slots, dtype=torch.int32, device=DEV)
    want = orc.conv_forward(d["x"], d["weight"], d["bias"])[0][0]
    live = [b for b in range(B) if slots is None or slots[b] >= 0]
    y = torch.full((B, H), float("nan"), device=DEV)
    mg.causal_conv_step(cfg, dev["x"][0], dev["weight"], dev["bias"], s, None, None, None, y)
    close(y[live], want[live], 2.0 ** -24, TOL)
    assert (y[[b for b in range(B) if b not in live]] == 0).all()
    # with a pool its rows count as before
    pool = torch.empty(3 if slots else B, 0, H, device=DEV)
    live = [b for b in live if slots is None or slots[b] < 3]
    for pools in ((pool, pool), (None, pool), (pool, None)):
        again = torch.full((B, H), float("nan"), device=DEV)
        mg.causal_conv_step(cfg, dev["x"][0], dev["weight"], dev["bias"], s, None, *pools, again)
        close(again[live], want[live], 2.0 ** -24, TOL)
        assert (again[[b for b in range(B) if b not in live]] == 0).all()
