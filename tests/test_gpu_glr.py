"""Gated linear recurrence on the GPU against the float64 oracle: types, forms, lengths around the tiles, widths around
the lanes, strides, resets, states handed on, gradients by formula and by differences, and one step at a time."""
import numpy as np
import pytest
import torch

import paper_2203_04738_amd as mg
from oracle import ops_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": (mg.MGRIT_F32, torch.float32), "bf16": (mg.MGRIT_BF16, torch.bfloat16),
         "f16": (mg.MGRIT_F16, torch.float16)}
FORMS = {"mix": mg.GLR_MIX, "decay": mg.GLR_DECAY}
# |gate| <= 4: a state remembers at most 1 / (1 - sigmoid(4)) = 56 steps, each rounded to 2^-24 of it, and a gate is known to
# about 10 units of 2^-24: (56 + 10) 2^-24 = 4e-6 of the largest value, doubled.  Gradients multiply two such values.
TOL, GRAD_TOL = 8e-6, 2.5e-5
# a result stored in 16 bits is rounded to half a unit of its last place
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -10}


def problem(seed, T, B, H, dtype="f32", form="mix", batch_first=False, resets=0.0):
    rng = np.random.default_rng(seed)
    dt = TYPES[dtype][1]
    gate = rng.uniform(-4, 4, (T, B, H)) if form == "mix" else -np.exp(rng.uniform(-4, 1, (T, B, H)))
    d = {"gate": gate, "value": rng.standard_normal((T, B, H)), "dh": rng.standard_normal((T, B, H))}
    dev = {}
    gv = torch.empty((B, T, 2 * H) if batch_first else (T, B, 2 * H), dtype=dt, device=DEV)
    gv = gv.transpose(0, 1) if batch_first else gv
    dev["gate"], dev["value"] = gv[..., :H], gv[..., H:]      # halves of one product's rows
    dev["dh"] = torch.empty((T, B, H), dtype=dt, device=DEV)
    for k in ("gate", "value", "dh"):
        dev[k].copy_(torch.from_numpy(d[k]))
        d[k] = dev[k].double().cpu().numpy()                  # as rounded
    for k in ("h0", "dh_last"):
        dev[k] = torch.from_numpy(rng.standard_normal((B, H)).astype(np.float32)).to(DEV)
        d[k] = dev[k].double().cpu().numpy()
    d["reset"] = (rng.random((T, B)) < resets).astype(np.uint8) if resets else None
    dev["reset"] = torch.from_numpy(d["reset"]).to(DEV) if resets else None
    return d, dev


def space(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


def run(dev, T, B, H, dtype, form, batch_first=False, h0=True, train=True):
    code, dt = TYPES[dtype]
    cfg = mg.GlrCfg(T, B, H, FORMS[form], code)
    ws, saved = space(mg.glr_workspace_bytes(cfg)), space(mg.glr_saved_bytes(cfg)) if train else None
    nan = float("nan")
    new = lambda W: torch.full((B, T, W) if batch_first else (T, B, W), nan, dtype=dt, device=DEV)  # noqa: E731
    seq = lambda t: t.transpose(0, 1) if batch_first else t  # noqa: E731
    h, h_last = seq(new(H)), torch.full((B, H), nan, device=DEV)
    first = dev["h0"] if h0 else None
    mg.glr_forward(cfg, dev["gate"], dev["value"], first, dev["reset"], h, h_last, saved, ws)
    out = {"h": h, "h_last": h_last}
    if train:
        dgv, dh0 = seq(new(2 * H)), torch.full((B, H), nan, device=DEV)
        mg.glr_backward(cfg, dev["gate"], dev["value"], dev["reset"], saved, dev["dh"],
                        dev["dh_last"] if h0 else None, dgv[..., :H], dgv[..., H:], dh0, ws)
        out.update(dgate=dgv[..., :H], dvalue=dgv[..., H:], dh0=dh0)
    torch.cuda.synchronize()
    return {k: v.double().cpu().numpy() for k, v in out.items()}


def expected(d, form, h0=True):
    first, last = (d["h0"], d["dh_last"]) if h0 else (None, None)
    h = orc.glr_forward(d["gate"], d["value"], first, d["reset"], form)
    dgate, dvalue, dh0 = orc.glr_backward(d["gate"], d["value"], h, d["dh"], first, d["reset"], last, form)
    return {"h": h, "h_last": h[-1], "dgate": dgate, "dvalue": dvalue, "dh0": dh0}


def close(got, ref, dtype, what=""):
    for k, g in got.items():
        r = ref[k]
        unit = UNIT["f32"] if k in ("h_last", "dh0") else UNIT[dtype]
        tol = GRAD_TOL if k.startswith("d") else TOL
        err = np.abs(g - r) - unit * np.abs(r)
        assert np.all(np.isfinite(g)), (what, k)
        assert err.max() <= tol * max(1.0, np.abs(r).max()), (what, k, err.max(), np.abs(r).max())


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 127, 128, 129, 300])
@pytest.mark.parametrize("H", [1, 3, 32, 33, 64, 65, 130])
def test_lengths_and_widths(T, H):
    d, dev = problem(T * 1000 + H, T, 2, H, resets=0.02)
    close(run(dev, T, 2, H, "f32", "mix"), expected(d, "mix"), "f32", (T, H))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("batch_first,resets,H", [(False, 0.0, 96), (True, 0.01, 96), (True, 0.3, 37), (False, 1.0, 37)])
def test_types_forms_strides(dtype, form, batch_first, resets, H):
    T, B = 533, 3
    d, dev = problem(7, T, B, H, dtype, form, batch_first, resets)
    close(run(dev, T, B, H, dtype, form, batch_first), expected(d, form), dtype)
    d["reset"] = dev["reset"] = None
    close(run(dev, T, B, H, dtype, form, batch_first, h0=False), expected(d, form, False), dtype)


@pytest.mark.parametrize("T,B,H", [(4500, 1, 70), (20000, 1, 5), (9000, 5, 200)])
def test_sequences_of_more_tiles_than_are_looked_at_at_once(T, B, H):
    d, dev = problem(3, T, B, H, resets=0.0005)
    got = run(dev, T, B, H, "f32", "mix")
    close(got, expected(d, "mix"), "f32")
    again = run(dev, T, B, H, "f32", "mix")
    assert all(np.array_equal(got[k], again[k]) for k in got)    # the order in which tiles meet does not show


def test_memory_that_lasts_the_whole_sequence():
    # gates of one (to rounding): nothing decays, and every tile's state counts for the last
    T, B, H = 3000, 2, 130
    d, dev = problem(5, T, B, H, form="decay")
    dev["gate"].zero_()
    dev["value"].copy_(torch.randint(-4, 5, (T, B, H)))         # whole numbers: the sums are exact
    dev["h0"].copy_(torch.randint(-4, 5, (B, H)))
    dev["dh"].copy_(torch.randint(-4, 5, (T, B, H)))
    dev["dh_last"].zero_()
    got = run(dev, T, B, H, "f32", "decay")
    v, dh = dev["value"].double().cpu().numpy(), dev["dh"].double().cpu().numpy()
    assert np.array_equal(got["h"], dev["h0"].double().cpu().numpy() + np.cumsum(v, 0))
    assert np.array_equal(got["dvalue"], np.cumsum(dh[::-1], 0)[::-1])
    assert np.array_equal(got["dh0"], dh.sum(0))


@pytest.mark.parametrize("form", FORMS)
def test_a_reset_forgets_what_is_not_finite(form):
    T, B, H = 700, 2, 96
    d, dev = problem(11, T, B, H, form=form, resets=0.0)
    reset = np.zeros((T, B), np.uint8)
    reset[300], reset[301, 1] = 1, 1
    dev["reset"] = torch.from_numpy(reset).to(DEV)
    clean = run(dev, T, B, H, "f32", form)
    dev["h0"].fill_(float("nan"))
    dev["value"][100:120] = float("inf")
    dev["gate"][250:260] = float("nan")
    got = run(dev, T, B, H, "f32", form)
    assert np.all(np.isnan(got["h"][260:300])) and np.all(np.isnan(got["h"][0]))   # and it lasts until then
    assert np.array_equal(got["h"][300:], clean["h"][300:])
    for k in ("dgate", "dvalue"):
        assert np.array_equal(got[k][301:], clean[k][301:])
    # from the other end: a gradient that is not finite stops at the reset
    d, dev = problem(11, T, B, H, form=form, resets=0.0)
    dev["reset"] = torch.from_numpy(reset).to(DEV)
    dev["dh"][500:510] = float("nan")
    got = run(dev, T, B, H, "f32", form)
    assert np.all(np.isnan(got["dvalue"][301:500])) and np.all(np.isnan(got["dvalue"][300, 0]))
    for k in ("dgate", "dvalue"):
        assert np.array_equal(got[k][:300], clean[k][:300])
    assert np.array_equal(got["dh0"], clean["dh0"])


def test_a_nan_is_not_forgotten_where_nothing_resets():
    T, B, H = 2000, 1, 70
    d, dev = problem(2, T, B, H)
    dev["gate"].fill_(-30.0)                                    # products of gates underflow within a tile
    dev["h0"].fill_(float("nan"))
    assert np.all(np.isnan(run(dev, T, B, H, "f32", "mix", train=False)["h"]))


def test_states_handed_on_from_call_to_call():
    T, B, H = 400, 2, 96
    d, dev = problem(9, T, B, H, resets=0.01)
    whole = run(dev, T, B, H, "f32", "mix", train=False)
    h = torch.empty(T, B, H, device=DEV)
    state = dev["h0"].clone()
    at = 0
    for n in (1, 130, 200, 69):
        cfg = mg.GlrCfg(n, B, H)
        s = slice(at, at + n)
        mg.glr_forward(cfg, dev["gate"][s], dev["value"][s], state, dev["reset"][s], h[s], state, None,
                       space(mg.glr_workspace_bytes(cfg)))      # h_last into h0 itself
        at += n
    torch.cuda.synchronize()
    ref = expected(d, "mix")
    close({"h": h.double().cpu().numpy(), "h_last": state.double().cpu().numpy()}, ref, "f32")
    close({"h": whole["h"]}, ref, "f32")


@pytest.mark.parametrize("form", FORMS)
def test_gradients_against_differences(form):
    # the float64 oracle's loss, differentiated by central differences at some places
    T, B, H = 150, 2, 6
    d, dev = problem(21, T, B, H, form=form, resets=0.02)
    got = run(dev, T, B, H, "f32", form)
    loss = lambda **kw: (lambda e: np.sum(d["dh"] * e) + np.sum(d["dh_last"] * e[-1]))(  # noqa: E731
        orc.glr_forward(kw.get("gate", d["gate"]), kw.get("value", d["value"]), kw.get("h0", d["h0"]), d["reset"], form))
    rng, eps = np.random.default_rng(0), 1e-5
    for name, grad in (("gate", "dgate"), ("value", "dvalue"), ("h0", "dh0")):
        for _ in range(8):
            at = tuple(rng.integers(0, n) for n in d[name].shape)
            up, down = d[name].copy(), d[name].copy()
            up[at] += eps
            down[at] -= eps
            diff = (loss(**{name: up}) - loss(**{name: down})) / (2 * eps)
            # (differences: 1e-16 / eps times a loss of some hundreds, and eps^2)
            assert abs(got[grad][at] - diff) <= 1e-7 + GRAD_TOL * max(1.0, np.abs(got[grad]).max()), (name, at)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("H", [1, 96, 257])
def test_steps_are_the_sequence(dtype, form, H):
    T, B, S = 5, 4, 7
    d, dev = problem(31, T, B, H, dtype, form, resets=0.2)
    code, dt = TYPES[dtype]
    slots = torch.tensor([5, 0, -1, 3], dtype=torch.int32, device=DEV)      # row 2 is idle
    pool = torch.randn(S, H, device=DEV)
    before = pool.clone()
    for k, s in ((0, 5), (1, 0), (3, 3)):
        pool[s] = dev["h0"][k]
    h = torch.full((T, B, H), float("nan"), dtype=dt, device=DEV)
    for t in range(T):
        mg.glr_step(mg.GlrCfg(1, B, H, FORMS[form], code), dev["gate"][t], dev["value"][t], slots,
                    dev["reset"][t], pool, pool, h[t])
    torch.cuda.synchronize()
    ref = expected(d, form)["h"]
    got = h.double().cpu().numpy()
    on = [0, 1, 3]
    close({"h": got[:, on]}, {"h": ref[:, on]}, dtype)
    assert np.all(got[:, 2] == 0)
    state = pool.double().cpu().numpy()
    close({"h_last": state[[5, 0, 3]]}, {"h_last": ref[-1, on]}, dtype)
    assert torch.equal(pool[[1, 2, 4, 6]], before[[1, 2, 4, 6]])
    # without slots, into another pool; a slot beyond the pool is idle as well
    two = torch.full((B, H), 7.0, device=DEV)
    mg.glr_step(mg.GlrCfg(1, B, H, FORMS[form], code), dev["gate"][0], dev["value"][0], None, None, dev["h0"], two, h[0])
    far = torch.tensor([0, B, 1, 1 << 30], dtype=torch.int32, device=DEV)
    out = torch.full((B, H), 7.0, device=DEV)
    mg.glr_step(mg.GlrCfg(1, B, H, FORMS[form], code), dev["gate"][0], dev["value"][0], far, None, dev["h0"], out, h[1])
    torch.cuda.synchronize()
    d["reset"] = None
    close({"h_last": two.double().cpu().numpy()}, {"h_last": expected(d, form)["h"][0]}, dtype)
    assert torch.all(out[2:] == 7) and torch.all(h[1, [1, 3]] == 0) and torch.equal(out[0], two[0])


def test_another_stream_and_a_graph():
    T, B, H = 1000, 2, 130
    d, dev = problem(41, T, B, H, resets=0.01)
    ref = run(dev, T, B, H, "f32", "mix")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run(dev, T, B, H, "f32", "mix")
    assert all(np.array_equal(got[k], ref[k]) for k in ref)
    cfg = mg.GlrCfg(T, B, H)
    ws, saved = space(mg.glr_workspace_bytes(cfg)), space(mg.glr_saved_bytes(cfg))
    h, dgv = torch.empty(T, B, H, device=DEV), torch.empty(T, B, 2 * H, device=DEV)

    def step():
        mg.glr_forward(cfg, dev["gate"], dev["value"], dev["h0"], dev["reset"], h, None, saved, ws)
        mg.glr_backward(cfg, dev["gate"], dev["value"], dev["reset"], saved, dev["dh"], dev["dh_last"],
                        dgv[..., :H], dgv[..., H:], None, ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        h.fill_(float("nan"))
        dgv.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(h.double().cpu().numpy(), ref["h"])
        assert np.array_equal(dgv[..., :H].double().cpu().numpy(), ref["dgate"])
        (h.sum() + dgv.sum()).item()                             # eager work in between


@pytest.mark.parametrize("T,stride", [(40000, 1 << 15), (40, (1 << 25) + 2)])
def test_offsets_beyond_32_bits(T, stride):
    # 5 GB between the first step and the last: by many steps, and by few that lie 128 MB apart
    B, H = 1, 66
    d, dev = problem(51, T, B, H)
    mem = torch.empty((T - 1) * stride + 2 * H, device=DEV)
    wide = torch.as_strided(mem, (T, B, 2 * H), (stride, 2 * H, 1))
    wide[..., :H], wide[..., H:] = dev["gate"], dev["value"]
    dev["gate"], dev["value"] = wide[..., :H], wide[..., H:]
    close(run(dev, T, B, H, "f32", "mix"), expected(d, "mix"), "f32")
    cfg = mg.GlrCfg(T, B, H)
    ws = space(mg.glr_workspace_bytes(cfg))
    gate, value = dev["gate"].clone(), dev["value"].clone()
    mem.fill_(7.0)
    mg.glr_forward(cfg, gate, value, dev["h0"], None, wide[..., :H], None, None, ws)
    torch.cuda.synchronize()
    close({"h": wide[..., :H].double().cpu().numpy()}, expected(d, "mix"), "f32")
    assert torch.all(wide[..., H:] == 7)


@pytest.mark.parametrize("gate", [88.0, 89.0, 95.0, 99.0, 100.0, 101.0, 200.0, 1e4, 3e38])
def test_a_factor_beyond_the_floats_is_infinite(gate):
    """One step from a state of 1, exp(gate) + 1: within the floats to some units, beyond them infinite."""
    B, H = 2, 40
    given = torch.full((B, H), gate, device=DEV)
    step, pool = torch.full((B, H), float("nan"), device=DEV), torch.ones(B, H, device=DEV)
    mg.glr_step(mg.GlrCfg(1, B, H, mg.GLR_DECAY), given, torch.ones(B, H, device=DEV), None, None, pool, pool, step)
    with np.errstate(over="ignore"):
        want = np.float64(np.float32(np.exp(np.float64(np.float32(gate)))))
    for got in (step.double().cpu().numpy(), pool.double().cpu().numpy()):
        if np.isinf(want):
            assert np.isposinf(got).all(), got.flat[0]
        else:
            assert (np.abs(got - want) <= 2.0 ** -24 * 100 * want).all()
