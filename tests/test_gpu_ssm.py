"""Selective state space scan on the GPU against the float64 oracle: types, states per channel, lengths around tiles and chunks,
widths around the lanes, strides, resets, states handed on, gradients by formula and by differences, one step at a time."""
import numpy as np
import pytest
import torch

import paper_2203_04738_amd as mg
from oracle import token_ops_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": (mg.MGRIT_F32, torch.float32, 2.0 ** -24), "bf16": (mg.MGRIT_BF16, torch.bfloat16, 2.0 ** -8),
         "f16": (mg.MGRIT_F16, torch.float16, 2.0 ** -11)}
# d a is between -0.02 and -8 or so: a state remembers at most some 50 steps, each rounded to 2^-24 of it, and an exponential is
# known to |d a| + 3 units of 2^-24, up to 11; sums over 64 states: (50 + 11 + 20) 2^-24 = 5e-6 of the largest value, doubled.
# Gradients multiply two such values, and are sums over the steps in chunks.
TOL, GRAD_TOL = 1e-5, 4e-5


def close(got, want, unit, tol, name=""):
    got = got.double().cpu().numpy()
    assert got.shape == want.shape, name
    err = np.abs(got - want)
    top = max(np.abs(want).max(), 1e-30)
    assert (err <= unit * np.abs(want) + tol * top).all(), (name, float(err.max() / top))


def problem(seed, T, B, H, S, dtype="f32", batch_first=False, resets=0.0, gated=True):
    rng = np.random.default_rng(seed)
    dt = TYPES[dtype][1]
    d, dev = {}, {}

    def rows(width):
        buf = torch.full((B, T, width) if batch_first else (T, B, width), float("nan"), dtype=dt, device=DEV)
        return buf.transpose(0, 1) if batch_first else buf

    def seq(name, view, values):
        view.copy_(torch.from_numpy(values))
        dev[name], d[name] = view, view.double().cpu().numpy()

    xz, dbc, dy = rows(2 * H), rows(H + 2 * S), rows(H)     # parts of two products' rows
    normal = rng.standard_normal
    seq("x", xz[..., :H], normal((T, B, H)))
    seq("z", xz[..., H:], 2 * normal((T, B, H)))
    seq("dt", dbc[..., :H], normal((T, B, H)) - 1)
    seq("b", dbc[..., H:H + S], normal((T, B, S)))
    seq("c", dbc[..., H + S:], normal((T, B, S)))
    seq("dy", dy, normal((T, B, H)))
    for name, v in (("a", -np.exp(rng.uniform(-1.5, 1, (H, S)))), ("skip", normal(H)), ("bias", 0.5 * normal(H)),
                    ("h0", normal((B, H, S))), ("dh_last", normal((B, H, S)))):
        v = v.astype(np.float32)
        d[name], dev[name] = v.astype(np.float64), torch.from_numpy(v).to(DEV)
    d["reset"] = (rng.random((T, B)) < resets).astype(np.uint8) if resets else None
    dev["reset"] = torch.from_numpy(d["reset"]).to(DEV) if resets else None
    if not gated:
        d["z"] = dev["z"] = None
    return d, dev


INPUTS = ("x", "dt", "b", "c", "z", "a", "skip", "bias")


def forward(dev, T, B, H, S, dtype="f32", batch_first=False, h0=True, train=True):
    code, dt, _ = TYPES[dtype]
    cfg = mg.SsmCfg(T, B, H, S, code)
    ws = torch.full((mg.ssm_workspace_bytes(cfg),), 255, dtype=torch.uint8, device=DEV)
    saved = torch.full((mg.ssm_saved_bytes(cfg),), 255, dtype=torch.uint8, device=DEV) if train else None
    y = torch.full((B, T, H) if batch_first else (T, B, H), float("nan"), dtype=dt, device=DEV)
    y = y.transpose(0, 1) if batch_first else y
    h_last = torch.full((B, H, S), float("nan"), device=DEV)
    mg.ssm_forward(cfg, *(dev[k] for k in INPUTS), dev["h0"] if h0 else None, dev["reset"], y, h_last, saved, ws)
    return cfg, ws, saved, y, h_last


def run(d, dev, T, B, H, S, dtype="f32", batch_first=False, full=True):
    if not full:
        for k in ("skip", "bias"):
            d[k] = dev[k] = None
    unit = TYPES[dtype][2]
    cfg, ws, saved, y, h_last = forward(dev, T, B, H, S, dtype, batch_first, full)
    gated, dt = dev["z"] is not None, TYPES[dtype][1]
    mark = 77.0
    shape = (B, T) if batch_first else (T, B)
    dxz = torch.full((*shape, 2 * H + 3), mark, dtype=dt, device=DEV)
    ddbc = torch.full((*shape, H + 2 * S + 1), mark, dtype=dt, device=DEV)
    v, w = (t.transpose(0, 1) if batch_first else t for t in (dxz, ddbc))
    nan = lambda *s: torch.full(s, float("nan"), device=DEV)  # noqa: E731
    g = {"dx": v[..., :H], "ddt": w[..., :H], "db": w[..., H:H + S], "dc": w[..., H + S:H + 2 * S],
         "dz": v[..., H:2 * H] if gated else None, "da": nan(H, S), "dskip": nan(H) if full else None,
         "dbias": nan(H) if full else None, "dh0": nan(B, H, S) if full else None}
    ws.fill_(255)
    mg.ssm_backward(cfg, *(dev[k] for k in INPUTS), dev["reset"], saved, dev["dy"], dev["dh_last"] if full else None,
                    *g.values(), ws)
    torch.cuda.synchronize()
    extra = dict(skip=d["skip"], bias=d["bias"], h0=d["h0"] if full else None, reset=d["reset"])
    args = [d[k] for k in INPUTS[:6]]
    wy, states, _ = orc.ssm_forward(*args, **extra)
    close(y, wy, unit, TOL, "y")
    close(h_last, states[-1], 0, TOL, "h_last")
    want = orc.ssm_backward(*args, d["dy"], dh_last=d["dh_last"] if full else None, **extra)
    for k, got in g.items():
        if got is not None:
            close(got, want[k], unit if k in ("dx", "ddt", "db", "dc", "dz") else 0, GRAD_TOL, k)
    assert (dxz[..., 2 * H:] == mark).all() and (ddbc[..., H + 2 * S:] == mark).all()
    if not gated:
        assert (dxz[..., H:] == mark).all()
    return y, h_last, g


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("T,B,H,S", [(1, 1, 1, 1), (3, 2, 5, 16), (15, 1, 16, 16), (16, 2, 17, 4), (17, 1, 63, 5), (32, 1, 64, 16),
                                     (33, 2, 65, 16), (50, 1, 20, 32), (49, 1, 33, 64), (130, 2, 40, 8)])
def test_shapes(dtype, T, B, H, S):
    run(*problem(T + H, T, B, H, S, dtype), T, B, H, S, dtype)


@pytest.mark.parametrize("S", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 47, 63, 64])
def test_states_of_a_channel(S):
    run(*problem(S, 37, 2, 18, S, resets=0.05), 37, 2, 18, S)


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("full", [True, False])
@pytest.mark.parametrize("resets", [0.0, 0.04, 1.0])
@pytest.mark.parametrize("batch_first", [False, True])
def test_options(gated, full, resets, batch_first):
    T, B, H, S = 90, 2, 24, 16
    run(*problem(3, T, B, H, S, "f32", batch_first, resets, gated), T, B, H, S, "f32", batch_first, full)


@pytest.mark.parametrize("T,B,H,S,resets", [(700, 1, 30, 16, 0.0), (700, 2, 100, 16, 0.01), (333, 3, 50, 64, 0.01),
                                            (1200, 1, 8, 2, 0.003), (2600, 1, 20, 16, 0.002)])
def test_many_chunks(T, B, H, S, resets):
    run(*problem(T, T, B, H, S, "f32", True, resets), T, B, H, S, "f32", True)


def test_many_rows_in_one_chunk():
    # more workgroups across than a card has: no chunks
    T, B, H, S = 20, 600, 6, 16
    run(*problem(2, T, B, H, S, "bf16"), T, B, H, S, "bf16")


def test_infinities_before_a_reset_stay_there():
    T, B, H, S = 80, 2, 20, 16
    d, dev = problem(8, T, B, H, S)
    dev["x"][10] = float("inf")
    dev["x"][11] = float("nan")
    dev["h0"].fill_(float("nan"))
    reset = torch.zeros(T, B, dtype=torch.uint8, device=DEV)
    reset[45] = 1
    dev["reset"] = reset
    cfg, ws, saved, y, h_last = forward(dev, T, B, H, S)
    assert torch.isnan(y[:45]).all()
    rest = {k: d[k][45:] if k in ("x", "dt", "b", "c", "z") else d[k] for k in INPUTS}
    want, states, _ = orc.ssm_forward(*(rest[k] for k in INPUTS[:6]), skip=d["skip"], bias=d["bias"])
    close(y[45:], want, 2.0 ** -24, TOL)
    close(h_last, states[-1], 0, TOL)
    # gradients behind it, and of b and c there
    new = lambda *s: torch.empty(*s, device=DEV)  # noqa: E731
    g = [new(T, B, H), new(T, B, H), new(T, B, S), new(T, B, S), new(T, B, H), new(H, S), None, None, None]
    mg.ssm_backward(cfg, *(dev[k] for k in INPUTS), reset, saved, dev["dy"], None, *g, ws)
    w = orc.ssm_backward(*(rest[k] for k in INPUTS[:6]), d["dy"][45:], skip=d["skip"], bias=d["bias"])
    for got, k in zip(g[:5], ("dx", "ddt", "db", "dc", "dz")):
        close(got[45:], w[k], 2.0 ** -24, GRAD_TOL, k)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_gates_of_the_lowest_value_are_closed(dtype):
    """z sigmoid(z) is 0 to within 1e-36 from z = -89 on, down to the type's lowest value, and so is its slope."""
    T, B, H, S = 40, 2, 20, 8
    d, dev = problem(22, T, B, H, S, dtype)
    low = torch.finfo(TYPES[dtype][1]).min
    for t, v in ((3, low), (4, low / 2), (11, -1000.0), (12, -120.0), (39, low)):
        dev["z"][t] = v
        d["z"][t] = dev["z"][t].double().cpu().numpy()
    with np.errstate(over="ignore"):
        y, _, g = run(d, dev, T, B, H, S, dtype)
    for t in (3, 4, 11, 12, 39):
        assert (y[t].abs() <= 1e-30).all() and (g["dz"][t].abs() <= 1e-30).all()


@pytest.mark.parametrize("T", [1, 15, 16, 17, 700])
def test_an_infinite_decay_forgets_at_every_step(T):
    d, dev = problem(21, T, 2, 20, 5)
    dev["a"][::2, ::2] = float("-inf")
    d["a"][::2, ::2] = -np.inf
    _, _, _, y, h_last = forward(dev, T, 2, 20, 5)
    want, states, _ = orc.ssm_forward(*(d[k] for k in INPUTS[:6]), skip=d["skip"], bias=d["bias"], h0=d["h0"])
    close(y, want, 2.0 ** -24, TOL, "y")
    close(h_last, states[-1], 0, TOL, "h_last")


def test_steps_so_large_or_small_that_exponentials_leave_the_floats():
    # d a down to -1e4 (a state that is forgotten at once) and to -1e-9 (one that stays), d down to e^-60
    T, B, H, S = 40, 1, 12, 16
    d, dev = problem(4, T, B, H, S)
    raw = np.linspace(-60, 60, T * H).reshape(T, 1, H)
    dev["dt"].copy_(torch.from_numpy(raw))
    a = -np.exp(np.linspace(-12, 5, H * S)).reshape(H, S).astype(np.float32)
    dev["a"], d["a"], d["dt"] = torch.from_numpy(a).to(DEV), a.astype(np.float64), dev["dt"].double().cpu().numpy()
    run(d, dev, T, B, H, S)


def test_softplus_and_its_slope_to_some_units():
    # one step from nothing: h = d b x, dL/ddt = slope b x c, with b = x = c = 1
    H = 4001
    raw = torch.linspace(-100, 100, H)
    one = lambda *s: torch.ones(*s, device=DEV)  # noqa: E731
    cfg = mg.SsmCfg(1, 1, H, 1)
    ws, saved = (torch.empty(f(cfg), dtype=torch.uint8, device=DEV) for f in (mg.ssm_workspace_bytes, mg.ssm_saved_bytes))
    dt, y = raw.view(1, 1, H).to(DEV), torch.empty(1, 1, H, device=DEV)
    inputs = (one(1, 1, H), dt, one(1, 1, 1), one(1, 1, 1), None, -one(H, 1), None, None)
    mg.ssm_forward(cfg, *inputs, None, None, y, None, saved, ws)
    ddt = torch.empty(1, 1, H, device=DEV)
    mg.ssm_backward(cfg, *inputs, None, saved, one(1, 1, H), None, torch.empty(1, 1, H, device=DEV), ddt, torch.empty(1, 1, 1,
                    device=DEV), torch.empty(1, 1, 1, device=DEV), None, torch.empty(H, 1, device=DEV), None, None, None, ws)
    v = raw.double().numpy()
    # an exponential known to 3 units, a reciprocal to 1, a series of 8 roundings: 2^-20 relative, where it is a normal float
    for got, want in ((y, np.logaddexp(v, 0)), (ddt, orc.sigmoid(v))):
        rel = np.abs(got.view(-1).double().cpu().numpy() - want) / want
        assert rel[v > -85].max() <= 2.0 ** -20, float(rel[v > -85].max())
        assert (got.view(-1).cpu().numpy()[v < -85] <= 2 * want[v < -85]).all()


def test_a_sequence_in_pieces():
    T, B, H, S = 120, 2, 30, 16
    d, dev = problem(6, T, B, H, S, resets=0.01)
    _, _, _, whole, last = forward(dev, T, B, H, S, train=False)
    parts, t = [], 0
    cur = dict(dev)
    for n in (1, 16, 40, 63):
        for k in ("x", "dt", "b", "c", "z"):
            cur[k] = dev[k][t:t + n]
        cur["reset"] = dev["reset"][t:t + n].contiguous()
        _, _, _, y, cur["h0"] = forward(cur, n, B, H, S, train=False)
        parts.append(y)
        t += n
    close(torch.cat(parts), whole.double().cpu().numpy(), 0, TOL)
    close(cur["h0"], last.double().cpu().numpy(), 0, TOL)


@pytest.mark.parametrize("dtype,S,gated", [("f32", 16, True), ("bf16", 5, False), ("f16", 64, True), ("bf16", 1, True)])
def test_steps_on_a_pool(dtype, S, gated):
    T, B, H, n = 10, 4, 21, 6
    code, dt, unit = TYPES[dtype]
    d, dev = problem(12, T, B, H, S, dtype, resets=0.2, gated=gated)
    cfg = mg.SsmCfg(1, B, H, S, code)
    slots = torch.tensor([5, 0, -1, 2], dtype=torch.int32, device=DEV)
    live = [0, 1, 3]
    pool = torch.full((n, H, S), 7.0, device=DEV)
    pool[slots[live].long()] = dev["h0"][live]
    out = []
    for t in range(T):
        y = torch.full((B, H), float("nan"), dtype=dt, device=DEV)
        mg.ssm_step(cfg, *(dev[k][t] if k in ("x", "dt", "b", "c", "z") and dev[k] is not None else dev[k] for k in INPUTS), slots,
                    dev["reset"][t], pool, pool, y)
        out.append(y)
    want, states, _ = orc.ssm_forward(*(d[k] for k in INPUTS[:6]), skip=d["skip"], bias=d["bias"], h0=d["h0"], reset=d["reset"])
    close(torch.stack(out)[:, live], want[:, live], unit, TOL)
    close(pool[slots[live].long()], states[-1][live], 0, TOL)
    assert (torch.stack(out)[:, 2] == 0).all() and (pool[[1, 3, 4]] == 7).all()


def test_gradients_by_differences():
    T, B, H, S = 40, 1, 6, 16
    d, dev = problem(14, T, B, H, S, resets=0.03)
    _, _, g = run(d, dev, T, B, H, S)

    def loss():
        _, _, _, y, h_last = forward(dev, T, B, H, S, train=False)
        return float((y.double() * dev["dy"].double()).sum() + (h_last.double() * dev["dh_last"].double()).sum())

    # central differences of step 1e-2 of a loss of some hundred values known to 1e-6 of some units: the square of the step times
    # a third derivative of some units of the largest gradient
    for name, grad, at in (("a", "da", (2, 5)), ("skip", "dskip", (3,)), ("bias", "dbias", (1,)), ("h0", "dh0", (0, 4, 7)),
                           ("x", "dx", (7, 0, 2)), ("dt", "ddt", (20, 0, 5)), ("b", "db", (11, 0, 9)), ("c", "dc", (30, 0, 0)),
                           ("z", "dz", (3, 0, 3))):
        v, e = dev[name], 1e-2
        old = float(v[at])
        v[at] = old + e
        up, hi = loss(), float(v[at])
        v[at] = old - e
        down, lo = loss(), float(v[at])
        v[at] = old
        top = float(g[grad].abs().max())
        assert abs((up - down) / (hi - lo) - float(g[grad][at])) <= 5e-3 * max(1.0, top), name


def test_the_same_bits_in_every_run_and_in_a_graph():
    T, B, H, S = 300, 2, 70, 16
    d, dev = problem(15, T, B, H, S, "bf16", resets=0.01)
    cfg, ws, saved, y, h_last = forward(dev, T, B, H, S, "bf16")
    new = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device=DEV)  # noqa: E731
    f32 = torch.float32
    g = [new(T, B, H), new(T, B, H), new(T, B, S), new(T, B, S), new(T, B, H), new(H, S, dtype=f32), new(H, dtype=f32),
         new(H, dtype=f32), new(B, H, S, dtype=f32)]
    inputs = [dev[k] for k in INPUTS]

    def both():
        mg.ssm_forward(cfg, *inputs, dev["h0"], dev["reset"], y, h_last, saved, ws)
        mg.ssm_backward(cfg, *inputs, dev["reset"], saved, dev["dy"], dev["dh_last"], *g, ws)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for i in range(3):
        dev["x"].mul_(-0.9)
        for t in [y, h_last] + g:
            t.zero_()
        both()
        eager = [t.clone() for t in [y, h_last] + g]
        for t in [y, h_last] + g:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, [y, h_last] + g):
            assert torch.equal(a, b) and float(a.abs().max()) > 0


@pytest.mark.parametrize("T", [1, 8, 15, 16, 17, 21, 33, 700])
@pytest.mark.parametrize("S", [5, 16, 64])
@pytest.mark.parametrize("full", [False, True])
def test_an_infinite_last_state_is_in_no_gradient_that_it_is_not_read_for(T, S, full):
    """The last input is infinite, and so is h_T.  da, dh0 and the gradients of the steps before do not read it, whether T is a
    multiple of a tile or not."""
    B, H, ch = 2, 20, 7
    d, dev = problem(23, T, B, H, S)
    dev["x"][T - 1, 1, ch] = float("inf")
    d["x"] = dev["x"].double().cpu().numpy()
    cfg, ws, saved, y, h_last = forward(dev, T, B, H, S, h0=full)
    new = lambda *s: torch.full(s, float("nan"), device=DEV)  # noqa: E731
    g = {"dx": new(T, B, H), "ddt": new(T, B, H), "db": new(T, B, S), "dc": new(T, B, S), "dz": new(T, B, H), "da": new(H, S),
         "dskip": new(H), "dbias": new(H), "dh0": new(B, H, S)}
    mg.ssm_backward(cfg, *(dev[k] for k in INPUTS), None, saved, dev["dy"], dev["dh_last"] if full else None, *g.values(), ws)
    with np.errstate(invalid="ignore"):
        want = orc.ssm_backward(*(d[k] for k in INPUTS[:6]), d["dy"], skip=d["skip"], bias=d["bias"], h0=d["h0"] if full else None,
                                dh_last=d["dh_last"] if full else None)
    assert torch.isinf(h_last[1, ch]).all() and torch.isfinite(h_last[0]).all()
    for k in ("da", "dh0", "dx"):
        assert np.isfinite(want[k]).all()
        close(g[k], want[k], 2.0 ** -24, GRAD_TOL, k)
    for k in ("ddt", "db", "dc", "dz"):
        close(g[k][:T - 1], want[k][:T - 1], 2.0 ** -24, GRAD_TOL, k) if T > 1 else None
    others = [i for i in range(H) if i != ch]
    for k in ("dskip", "dbias"):
        close(g[k][others], want[k][others], 0, GRAD_TOL, k)


@pytest.mark.parametrize("T", [1, 15, 16, 17, 90, 700])
@pytest.mark.parametrize("low", [-90.0, -110.0, -500.0])
def test_an_infinite_decay_forgets_where_the_step_is_too_small_for_a_float(T, low):
    """softplus(low) is above 0, if only by e^low: exp(d a) is 0 for a = -infinity, in sequences and single steps."""
    B, H, S = 2, 20, 5
    d, dev = problem(24, T, B, H, S)
    dev["a"][::2, ::2] = float("-inf")
    d["a"][::2, ::2] = -np.inf
    dev["dt"][::3] = low
    dev["dt"][:, 1] = low                                      # and nothing but such steps
    d["dt"] = dev["dt"].double().cpu().numpy()
    cfg, _, _, y, h_last = forward(dev, T, B, H, S)
    want, states, _ = orc.ssm_forward(*(d[k] for k in INPUTS[:6]), skip=d["skip"], bias=d["bias"], h0=d["h0"])
    close(y, want, 2.0 ** -24, TOL, "y")
    close(h_last, states[-1], 0, TOL, "h_last")
    pool, out = dev["h0"].clone(), []
    one = mg.SsmCfg(1, B, H, S)
    for t in range(min(T, 20)):
        out.append(torch.full((B, H), float("nan"), device=DEV))
        mg.ssm_step(one, *(dev[k][t] if k in ("x", "dt", "b", "c", "z") else dev[k] for k in INPUTS), None, None, pool, pool, out[-1])
    close(torch.stack(out), want[:20], 2.0 ** -24, TOL, "step")
    close(pool, states[len(out) - 1], 0, TOL, "pool")
