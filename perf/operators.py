"""Performance cases of the operators of a gated linear recurrent student: how it is trained, served and scored.

Four operators, each one pass through public entry points of ``paper_2203_04738_amd``:

* the gated linear recurrence ``h_t = a_t h_{t-1} + b_t`` over long sequences (forward, forward + backward, and
  one token at a time on a pool of states);
* the log probabilities of given tokens, with the entropy and the top alternatives of every row;
* the distillation loss from a teacher's top logits, with its gradient (in one pass, or forward and backward apart);
* the product in 8-bit integers with a scale for each token and each channel, quantising its tokens on the way.

With ``own`` false the same outputs come from elementary torch operations in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _scan(name, kind, dtype, T, B, H, form="mix", batch_first=False, reset=False):
    c = {"kind": kind, "dtype": dtype, "T": T, "B": B, "H": H, "form": form, "batch_first": batch_first,
         "reset": reset}
    return dict(c, name=name) if name else c


def _step(name, dtype, B, H, slots, form="mix"):
    c = {"kind": "step", "dtype": dtype, "B": B, "H": H, "slots": slots, "form": form}
    return dict(c, name=name) if name else c


def _rows(name, kind, dtype, N, V, K, temperature=1.0):
    c = {"kind": kind, "dtype": dtype, "N": N, "V": V, "K": K, "temperature": temperature}
    return dict(c, name=name) if name else c


def _q8(name, dtype, M, K, N, bias=True):
    c = {"kind": "q8", "dtype": dtype, "M": M, "K": K, "N": N, "bias": bias}
    return dict(c, name=name) if name else c


def listed():
    return [
        # serving: one token of a hundred running sequences, their states in a pool
        _step("step_serve", "bf16", 100, 1024, 128),
        # a ragged prompt read in: odd length, three sequences, a width that is no multiple of a tile
        _scan("scan_prompt", "scan", "f32", 777, 3, 500, batch_first=True),
        # a training step of the video shape (128 steps, batch 100, 1000 features)
        _scan("scan_train_video", "scan_train", "f32", 128, 100, 1000),
        # training on the longest sequences, several documents packed into each
        _scan("scan_train_long", "scan_train", "bf16", 16384, 4, 1024, reset=True),
        # the 51 classes of the classification head for a batch of a hundred
        _rows("logp_classes", "logp", "f32", 100, 51, 5),
        # one decoding step of eight sequences: the chosen tokens, and twenty alternatives of each
        _rows("logp_decode", "logp", "bf16", 8, 32768, 20),
        # scoring 2048 tokens of text on a large vocabulary
        _rows("logp_score", "logp", "bf16", 2048, 131072, 8),
        # a training step on 8192 tokens: loss and gradient together, 64 teacher logits per token
        _rows("distill_train", "distill", "bf16", 8192, 32768, 64, 2.0),
        # odd sizes in 32 bits, forward and backward as two calls
        _rows("distill_ragged", "distill_apart", "f32", 1003, 50021, 17),
        # serving: the gate product of eight tokens
        _q8("q8_decode", "bf16", 8, 2048, 2048),
        # a ragged prompt through a layer whose widths are no multiples of a tile
        _q8("q8_prompt", "f32", 777, 500, 1000),
        # reading in 4096 steps of a batch of eight: the gate product of the image shape (2048 features, 2 x 1024)
        _q8("q8_read_in", "bf16", 32768, 2048, 2048, bias=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    largest = {c["name"]: work(c) for c in listed()}
    kind = rng.choice(["step", "scan", "scan_train", "scan_train", "logp", "logp", "distill", "distill_apart", "q8",
                       "q8"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    form = rng.choice(["mix", "mix", "decay"])
    while True:
        if kind == "step":
            B = _log(rng, 1, 1024)
            return _step(None, dtype, B, _log(rng, 32, 2048), B + rng.randrange(64), form)
        if kind in ("scan", "scan_train"):
            c = _scan(None, kind, dtype, _log(rng, 1, 16384), _log(rng, 1, 100), _log(rng, 32, 2048), form,
                      rng.random() < 0.5, rng.random() < 0.5)
            top = largest["scan_train_long"]["bytes"]
        elif kind == "q8":
            c = _q8(None, dtype, _log(rng, 1, 32768), _log(rng, 32, 8192), _log(rng, 32, 8192), rng.random() < 0.5)
            top = largest["q8_read_in"]["flops"]
            if work(c)["flops"] > top:
                continue
            return c
        else:
            V = _log(rng, 2, 131072)
            K = min(V, _log(rng, 1, 64))
            c = _rows(None, kind, dtype, _log(rng, 1, 8192), V, K, rng.choice([1.0, 1.0, 0.7, 2.0]))
            top = largest["logp_score"]["bytes"]
        if work(c)["bytes"] <= top:
            return c


def work(case):
    """Every input read once, every output written once; for the arithmetic the multiply-adds of the formulas, an
    exponential counted as one operation."""
    c, e = case, SIZE[case["dtype"]]
    if c["kind"] == "step":
        n = c["B"] * c["H"]
        return {"bytes": n * (2 * e + 4 + 4 + e) + 4 * c["B"], "flops": 6 * n}
    if c["kind"] == "scan":
        n, s = c["T"] * c["B"] * c["H"], c["B"] * c["H"]
        return {"bytes": 3 * e * n + 8 * s + (c["T"] * c["B"] if c["reset"] else 0), "flops": 6 * n}
    if c["kind"] == "scan_train":
        n, s = c["T"] * c["B"] * c["H"], c["B"] * c["H"]
        # forward: gate, value -> states; backward: gate, value, dh -> dgate, dvalue
        return {"bytes": 8 * e * n + 16 * s + 2 * (c["T"] * c["B"] if c["reset"] else 0), "flops": 20 * n}
    if c["kind"] == "logp":
        return {"bytes": c["N"] * (c["V"] * e + 8 + 8 + 12 * c["K"]), "flops": 5 * c["N"] * c["V"]}
    if c["kind"] == "distill":
        return {"bytes": c["N"] * (2 * c["V"] * e + 12 * c["K"] + 12), "flops": 7 * c["N"] * c["V"]}
    if c["kind"] == "distill_apart":
        return {"bytes": c["N"] * (3 * c["V"] * e + 24 * c["K"] + 24), "flops": 7 * c["N"] * c["V"]}
    M, N, K = c["M"], c["N"], c["K"]
    return {"bytes": M * K * e + N * K + 4 * N * (2 if c["bias"] else 1) + M * N * e, "flops": 2 * M * N * K}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _time_major(c, x):
    """[T,B,W] view of a tensor stored [B,T,W] or [T,B,W]."""
    return x.transpose(0, 1) if c["batch_first"] else x


def _gate_value(c, gen, rows):
    """Gate and candidate of a layer as one product leaves them, side by side.  Every channel has a memory of its
    own: gates around sigmoid(0..6), or decays of e^-2 .. e^-0.002 per step."""
    H = c["H"]
    z = torch.randn(*rows, 2 * H, generator=gen, device="cuda")
    u = torch.rand(H, generator=gen, device="cuda")
    if c["form"] == "mix":
        z[..., :H] += 6 * u
    else:
        z[..., :H] = -torch.exp(0.3 * z[..., :H] - 6 * u)
    return z.to(DTYPES[c["dtype"]])


def prepare(case, seed):
    c, gen, dt = dict(case), _generator(seed), DTYPES[case["dtype"]]
    dev = torch.device("cuda")
    st = {"case": c}
    if c["kind"] == "step":
        B, H = c["B"], c["H"]
        st["gv"] = _gate_value(c, gen, (B,))
        st["state"] = torch.randn(c["slots"], H, generator=gen, device=dev)
        st["slots"] = torch.randperm(c["slots"], generator=gen, device=dev)[:B].to(torch.int32)
    elif c["kind"] in ("scan", "scan_train"):
        T, B, H = c["T"], c["B"], c["H"]
        rows = (B, T) if c["batch_first"] else (T, B)
        st["gv"] = _gate_value(c, gen, rows)
        st["h0"] = torch.randn(B, H, generator=gen, device=dev)
        st["reset"] = None
        if c["reset"]:               # documents of about 700 tokens
            st["reset"] = (torch.rand(T, B, generator=gen, device=dev) < 1 / 700).to(torch.uint8)
        if c["kind"] == "scan_train":
            st["dh"] = torch.randn(*rows, H, generator=gen, device=dev).to(dt)
            st["dh_last"] = torch.randn(B, H, generator=gen, device=dev)
    elif c["kind"] == "q8":
        M, K, N = c["M"], c["K"], c["N"]
        # tokens of different sizes, as after a layer without a norm
        st["x"] = (torch.randn(M, K, generator=gen, device=dev)
                   * torch.exp(0.5 * torch.randn(M, 1, generator=gen, device=dev))).to(dt)
        w = torch.randn(N, K, generator=gen, device=dev) / math.sqrt(K)
        # the weights as a program keeps them: 8 bits, rows padded with zeros to 128 bytes
        scale = (w.abs().amax(1) / 127).clamp_min(2.0 ** -126)
        q = torch.zeros(N, (K + 127) // 128 * 128, dtype=torch.int8, device=dev)
        q[:, :K] = torch.round(w / scale[:, None]).to(torch.int8)
        st["w_q"], st["w_scale"] = q, scale
        st["bias"] = 0.1 * torch.randn(N, generator=gen, device=dev) if c["bias"] else None
    else:
        N, V, K = c["N"], c["V"], c["K"]
        # a flat background and, in every row, a few tokens that stand out
        x = torch.randn(N, V, generator=gen, device=dev)
        u = torch.rand(N, V, generator=gen, device=dev) * (V / 16)
        x += 6 * u * (u < 1)
        if V > 256:                  # a vocabulary padded to a round size, and tokens that a mask forbids
            x[:, V - V // 128:] = -math.inf
            x[::3, : V // 8] = -math.inf
        st["logits"] = x.to(dt)
        lo, hi = (V // 8, V - V // 128) if V > 256 else (0, V)
        if c["kind"] == "logp":
            st["tokens"] = torch.where(torch.rand(N, generator=gen, device=dev) < 0.5, x.argmax(1),
                                       torch.randint(lo, hi, (N,), generator=gen, device=dev))
            st["tokens"][torch.rand(N, generator=gen, device=dev) < 1 / 16] = -1       # positions without a token
        else:
            K = min(K, hi - lo)
            ids = lo + (torch.randint(0, hi - lo, (N, 1), generator=gen, device=dev)
                        + torch.randint(1, max(2, (hi - lo) // K + 1), (N, c["K"]), generator=gen,
                                        device=dev).cumsum(1)) % (hi - lo)
            count = torch.randint(max(1, c["K"] // 2), c["K"] + 1, (N, 1), generator=gen, device=dev)
            count[torch.rand(N, 1, generator=gen, device=dev) < 1 / 16] = 0            # rows without a teacher
            st["ids"] = torch.where(torch.arange(c["K"], device=dev) < count, ids, -1)
            st["teacher"] = torch.sort(3 * torch.randn(N, c["K"], generator=gen, device=dev), dim=1,
                                       descending=True).values
            st["weight"] = torch.rand(N, generator=gen, device=dev) / N
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _coefficients(c, g, v):
    """(a, b, da, db): h = a h' + b, da = what dh/dg has of h', db = dh/dv, in 32 bits."""
    if c["form"] == "mix":
        a = torch.sigmoid(g)
        db = torch.sigmoid(-g)
        b = db * v
        da = a * db
    else:
        a = torch.exp(g)
        db = torch.ones_like(g)
        b = v
        da = a
    return a, b, da, db


def _linear_scan(a, b):
    """All h_t = a_t h_{t-1} + b_t along the first axis, h_0 = 0: composed over spans of 1, 2, 4, ... steps."""
    a, b, span = a.clone(), b.clone(), 1
    while span < len(a):
        b[span:] += a[span:] * b[:-span]
        a[span:] = a[span:] * a[:-span]
        span *= 2
    return b


def _plain_scan(c, gv, h0, reset):
    H = c["H"]
    g, v = gv[..., :H].float(), gv[..., H:].float()
    a, b, da, db = _coefficients(c, g, v)
    if reset is not None:
        a = a * (reset[..., None] == 0)
    b = torch.cat([b[:1] + a[:1] * h0, b[1:]])
    h = _linear_scan(a, b)
    return h, a, da, db, v


def _plain_scan_backward(c, h, h0, a, da, db, v, reset, dh, dh_last):
    dh = torch.cat([dh[:-1], dh[-1:] + dh_last])
    # lambda_t = dh_t + a_{t+1} lambda_{t+1}: the same scan from the other end
    back = torch.cat([torch.zeros_like(a[:1]), a[1:].flip(0)])
    lam = _linear_scan(back, dh.flip(0)).flip(0)
    prev = torch.cat([h0[None], h[:-1]])
    if reset is not None:
        prev = prev * (reset[..., None] == 0)
    dg = lam * (prev - v) * da if c["form"] == "mix" else lam * prev * da
    return torch.cat([dg, lam * db], dim=-1), a[0] * lam[0]


def _keys(x):
    """A whole number per value, larger for larger values and, among equal ones, for lower indices."""
    bits = (x.float() + 0.0).contiguous().view(torch.int32)
    order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits).to(torch.int64)
    return order * 2 ** 32 + (2 ** 32 - 1 - torch.arange(x.shape[-1], device=x.device))


def _plain_logp(st):
    c, x = st["case"], st["logits"].float() / st["case"]["temperature"]
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    s = e.sum(1, keepdim=True)
    p = e / s
    lse = m + torch.log(s)
    entropy = -torch.where(p > 0, p * (x - lse), torch.zeros_like(p)).sum(1)
    tok = st["tokens"]
    logp = torch.where(tok >= 0, (x.gather(1, tok.clamp(min=0)[:, None]) - lse)[:, 0], torch.zeros_like(entropy))
    ids = 2 ** 32 - 1 - torch.topk(_keys(st["logits"]), c["K"], dim=1).values % 2 ** 32
    return logp, entropy, x.gather(1, ids) - lse, ids


def _teacher(st):
    """The teacher's weights over its own entries (none for padding) and, where a row has any, True."""
    t = torch.where(st["ids"] >= 0, st["teacher"] / st["case"]["temperature"], -math.inf)
    some = (st["ids"] >= 0).any(1, keepdim=True)
    e = torch.exp(t - torch.where(some, t.amax(1, keepdim=True), torch.zeros_like(t[:, :1])))
    return e / torch.where(some, e.sum(1, keepdim=True), torch.ones_like(t[:, :1])), some


def _plain_distill(st):
    c = st["case"]
    x = st["logits"].float() / c["temperature"]
    q, some = _teacher(st)
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    s = e.sum(1, keepdim=True)
    lse = m + torch.log(s)
    at = st["ids"].clamp(min=0)
    part = torch.where(q > 0, q * (torch.log(q) - x.gather(1, at) + lse), torch.zeros_like(q))
    loss = part.sum(1)
    grad = (e / s * some).scatter_add_(1, at, -q)
    grad = grad * (st["weight"][:, None] / c["temperature"])
    return loss, grad.to(st["logits"].dtype)


def _plain_q8(st):
    x = st["x"].float()
    scale = (x.abs().amax(1, keepdim=True) / 127).clamp_min(2.0 ** -126)
    q = torch.round(x / scale)
    y = (q @ st["w_q"][:, : st["case"]["K"]].float().T) * scale * st["w_scale"]
    if st["bias"] is not None:
        y = y + st["bias"]
    return y.to(st["x"].dtype)


def _plain(st):
    c = st["case"]
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "step":
        at = st["slots"].long()
        a, b, _, _ = _coefficients(c, st["gv"][:, : c["H"]].float(), st["gv"][:, c["H"]:].float())
        h = a * st["state"][at] + b
        state = st["state"].clone()
        state[at] = h
        return {"h": h.to(dt), "state": state}
    if c["kind"] in ("scan", "scan_train"):
        gv = _time_major(c, st["gv"])
        h, a, da, db, v = _plain_scan(c, gv, st["h0"], st["reset"])
        out = {"h": _time_major(c, h).to(dt).contiguous(), "h_last": h[-1]}
        if c["kind"] == "scan_train":
            dgv, dh0 = _plain_scan_backward(c, h, st["h0"], a, da, db, v, st["reset"],
                                            _time_major(c, st["dh"]).float(), st["dh_last"])
            out["dgv"], out["dh0"] = _time_major(c, dgv).to(dt).contiguous(), dh0
        return out
    if c["kind"] == "logp":
        logp, entropy, top, ids = _plain_logp(st)
        return {"logp": logp, "entropy": entropy, "top_logp": top, "top_ids": ids}
    if c["kind"] in ("distill", "distill_apart"):
        loss, grad = _plain_distill(st)
        return {"loss": loss, "dlogits": grad}
    return {"y": _plain_q8(st)}


# ---------------------------------------------------------------------------
# the framework's entry points
# ---------------------------------------------------------------------------
def _kept(st, key, make):
    """What a program keeps from call to call: its workspaces and output buffers."""
    if key not in st:
        st[key] = make()
    return st[key]


def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def _own(st):
    import paper_2203_04738_amd as mg
    c = st["case"]
    dt = DTYPES[c["dtype"]]
    code = {"f32": mg.MGRIT_F32, "bf16": mg.MGRIT_BF16, "f16": mg.MGRIT_F16}[c["dtype"]]
    new = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if c["kind"] in ("step", "scan", "scan_train"):
        H, form = c["H"], {"mix": mg.GLR_MIX, "decay": mg.GLR_DECAY}[c["form"]]
    if c["kind"] == "step":
        cfg = mg.GlrCfg(1, c["B"], H, form, code)
        h, state = _kept(st, "out", lambda: (new(c["B"], H, dtype=dt), st["state"].clone()))
        mg.glr_step(cfg, st["gv"][:, :H], st["gv"][:, H:], st["slots"], None, st["state"], state, h)
        return {"h": h, "state": state}
    if c["kind"] in ("scan", "scan_train"):
        T, B = c["T"], c["B"]
        cfg = mg.GlrCfg(T, B, H, form, code)
        train = c["kind"] == "scan_train"
        ws = _kept(st, "ws", lambda: _bytes(mg.glr_workspace_bytes(cfg)))
        saved = _kept(st, "saved", lambda: _bytes(mg.glr_saved_bytes(cfg))) if train else None
        h, h_last = _kept(st, "out", lambda: (new(*st["gv"].shape[:2], H, dtype=dt), new(B, H)))
        gv = _time_major(c, st["gv"])
        mg.glr_forward(cfg, gv[..., :H], gv[..., H:], st["h0"], st["reset"], _time_major(c, h), h_last, saved, ws)
        out = {"h": h, "h_last": h_last}
        if train:
            dgv, dh0 = _kept(st, "grads", lambda: (torch.empty_like(st["gv"]), new(B, H)))
            d = _time_major(c, dgv)
            mg.glr_backward(cfg, gv[..., :H], gv[..., H:], st["reset"], saved, _time_major(c, st["dh"]),
                            st["dh_last"], d[..., :H], d[..., H:], dh0, ws)
            out["dgv"], out["dh0"] = dgv, dh0
        return out
    if c["kind"] == "q8":
        cfg = mg.Q8Cfg(c["M"], c["N"], c["K"], code)
        ws = _kept(st, "ws", lambda: _bytes(mg.q8_workspace_bytes(cfg)))
        y = _kept(st, "out", lambda: new(c["M"], c["N"], dtype=dt))
        mg.q8_linear(cfg, st["x"], st["w_q"], st["w_scale"], st["bias"], y, ws)
        return {"y": y}
    N, V, K = c["N"], c["V"], c["K"]
    cfg = mg.LogitsCfg(N, V, K, code, c["temperature"])
    ws = _kept(st, "ws", lambda: _bytes(mg.logits_workspace_bytes(cfg)))
    if c["kind"] == "logp":
        logp, entropy, top, ids = _kept(st, "out", lambda: (new(N), new(N), new(N, K), new(N, K, dtype=torch.int64)))
        mg.token_logprobs(cfg, st["logits"], st["tokens"], logp, entropy, top, ids, ws)
        return {"logp": logp, "entropy": entropy, "top_logp": top, "top_ids": ids}
    loss, grad = _kept(st, "out", lambda: (new(N), new(N, V, dtype=dt)))
    if c["kind"] == "distill":
        mg.distill_topk(cfg, st["logits"], st["ids"], st["teacher"], st["weight"], loss, None, grad, ws)
    else:
        stats = _kept(st, "stats", lambda: new(N, 2))
        mg.distill_topk(cfg, st["logits"], st["ids"], st["teacher"], None, loss, stats, None, ws)
        mg.distill_topk_backward(cfg, st["logits"], st["ids"], st["teacher"], stats, st["weight"], grad)
    return {"loss": loss, "dlogits": grad}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# the same outputs in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _exact_gates(c, gv):
    g, v = gv[..., : c["H"]].double(), gv[..., c["H"]:].double()
    if c["form"] == "mix":
        z = 1 / (1 + torch.exp(-g))
        return z, 1 / (1 + torch.exp(g)), v
    return torch.exp(g), None, v


def exact(case, seed):
    c, st = case, prepare(case, seed)
    if c["kind"] == "step":
        z, y, v = _exact_gates(c, st["gv"])
        at, state = st["slots"].long(), st["state"].double()
        state[at] = z * state[at] + (y * v if y is not None else v)
        return {"h": state[at], "state": state}
    if c["kind"] in ("scan", "scan_train"):              # step by step, forward and back
        z, y, v = _exact_gates(c, _time_major(c, st["gv"]))
        T, H = c["T"], c["H"]
        keep = torch.ones(T, c["B"], 1, dtype=torch.float64, device=z.device)
        if st["reset"] is not None:
            keep = (st["reset"] == 0).double()[..., None]
        h = torch.empty(T + 1, c["B"], H, dtype=torch.float64, device=z.device)
        h[0] = st["h0"].double()
        for t in range(T):
            h[t + 1] = z[t] * keep[t] * h[t] + (y[t] * v[t] if y is not None else v[t])
        out = {"h": _time_major(c, h[1:]).contiguous(), "h_last": h[T]}
        if c["kind"] == "scan_train":
            dh, lam = _time_major(c, st["dh"]).double(), st["dh_last"].double()
            grads = torch.empty(T, c["B"], 2 * H, dtype=torch.float64, device=z.device)
            for t in range(T - 1, -1, -1):
                lam = lam + dh[t]
                past = keep[t] * h[t]
                grads[t, :, :H] = lam * z[t] * (y[t] * (past - v[t]) if y is not None else past)
                grads[t, :, H:] = lam * y[t] if y is not None else lam
                lam = keep[t] * z[t] * lam
            out["dgv"], out["dh0"] = _time_major(c, grads).contiguous(), lam
        return out
    if c["kind"] == "q8":
        # the definition rounds twice to 32 bits: a token's scale, and the quotient that is rounded to 8 bits
        x = st["x"].float().cpu().numpy()
        scale = np.maximum(np.abs(x).max(axis=1, keepdims=True) / np.float32(127), np.float32(2.0 ** -126))
        q = torch.from_numpy(np.rint(x / scale)).to("cuda", torch.float64)
        y = torch.matmul(q, st["w_q"][:, : c["K"]].double().t().contiguous())
        y = y * torch.from_numpy(scale).to("cuda", torch.float64) * st["w_scale"].double()
        return {"y": y if st["bias"] is None else y + st["bias"].double()}
    parts, step = [], max(1, (1 << 26) // c["V"])        # in blocks of rows of at most 2^26 values
    for i in range(0, c["N"], step):
        x = st["logits"][i:i + step].double() / c["temperature"]
        lse = torch.logsumexp(x, 1)
        p = torch.softmax(x, 1)
        if c["kind"] == "logp":
            tok = st["tokens"][i:i + step]
            logp = torch.where(tok < 0, 0.0, x.gather(1, tok.clamp(min=0)[:, None])[:, 0] - lse)
            top, ids = torch.sort(x, dim=1, descending=True, stable=True)
            parts.append((logp, torch.special.entr(p).sum(1), top[:, : c["K"]] - lse[:, None],
                          ids[:, : c["K"]].clone()))
            continue
        ids, w = st["ids"][i:i + step], st["weight"][i:i + step].double()
        t = torch.where(ids < 0, -math.inf, st["teacher"][i:i + step].double() / c["temperature"])
        q = torch.softmax(t, 1).nan_to_num(0.0)          # rows without a teacher: no weights
        at = ids.clamp(min=0)
        nll = torch.where(q > 0, lse[:, None] - x.gather(1, at), 0.0)
        grad = p * q.sum(1, keepdim=True)
        grad.scatter_add_(1, at, -q)
        parts.append(((torch.special.xlogy(q, q) + q * nll).sum(1), grad * (w / c["temperature"])[:, None]))
    names = ("logp", "entropy", "top_logp", "top_ids") if c["kind"] == "logp" else ("loss", "dlogits")
    return {name: torch.cat([p[k] for p in parts]) for k, name in enumerate(names)}
