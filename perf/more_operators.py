"""Performance cases of the operators of a recurrent student over tokens: tokens in, memory, learning from a reward.

Four operators, each one pass through public entry points of ``paper_2203_04738_amd``:

* the embedding of tokens, scaled, with its gradient;
* the short causal convolution of every channel (forward, forward + backward);
* the selective state space scan, several states per channel (forward, forward + backward), and one token at a time
  through convolution and scan on pools of states;
* the clipped policy loss with a KL term on rows of logits, with its gradient (in one pass, or forward and backward
  apart).

With ``own`` false the same outputs come from elementary torch operations in 32 bits (64 for what a row's loss is made
of), rounded once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
CLIP_LOW, CLIP_HIGH = 0.2, 0.28


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _embed(name, kind, dtype, N, V, D):
    c = {"kind": kind, "dtype": dtype, "N": N, "V": V, "D": D}
    return dict(c, name=name) if name else c


def _conv(name, kind, dtype, T, B, H, W, silu=True, batch_first=False, reset=False):
    c = {"kind": kind, "dtype": dtype, "T": T, "B": B, "H": H, "W": W, "silu": silu, "batch_first": batch_first,
         "reset": reset}
    return dict(c, name=name) if name else c


def _scan(name, kind, dtype, T, B, H, S, gated=True, batch_first=False, reset=False):
    c = {"kind": kind, "dtype": dtype, "T": T, "B": B, "H": H, "S": S, "gated": gated, "batch_first": batch_first,
         "reset": reset}
    return dict(c, name=name) if name else c


def _step(name, dtype, B, H, S, W, slots):
    c = {"kind": "step", "dtype": dtype, "B": B, "H": H, "S": S, "W": W, "slots": slots}
    return dict(c, name=name) if name else c


def _policy(name, kind, dtype, N, V, kl, temperature=1.0):
    c = {"kind": kind, "dtype": dtype, "N": N, "V": V, "kl": kl, "temperature": temperature}
    return dict(c, name=name) if name else c


def listed():
    return [
        # serving: the embeddings of the next tokens of eight sequences
        _embed("embed_decode", "embed", "bf16", 8, 32768, 2048),
        # a training step on 16384 tokens: their embeddings, and the gradient of the whole table
        _embed("embed_train", "embed_train", "bf16", 16384, 32768, 1024),
        # the same in 32 bits at odd sizes
        _embed("embed_ragged", "embed_train", "f32", 1003, 50021, 500),
        # a ragged prompt through a convolution of three taps, without an activation
        _conv("conv_prompt", "conv", "f32", 777, 3, 500, 3, silu=False, batch_first=True),
        # training on the longest sequences, several documents packed into each
        _conv("conv_train_long", "conv_train", "bf16", 16384, 4, 1024, 4, reset=True),
        # serving: one token of a hundred running sequences through convolution and scan, their states in pools
        _step("step_serve", "bf16", 100, 1024, 16, 4, 128),
        # a ragged prompt read in: odd length, three sequences, a width that is no multiple of a tile
        _scan("scan_prompt", "scan", "f32", 777, 3, 500, 16, batch_first=True),
        # a training step of the video shape (128 steps, batch 100, 1000 features)
        _scan("scan_train_video", "scan_train", "f32", 128, 100, 1000, 16),
        # training on long sequences, several documents packed into each
        _scan("scan_train_long", "scan_train", "bf16", 8192, 4, 1024, 16, reset=True),
        # the 51 classes of the classification head as actions, for a batch of a hundred
        _policy("policy_classes", "policy", "f32", 100, 51, 0.0),
        # a training step on 8192 sampled tokens: loss and gradient together
        _policy("policy_train", "policy", "bf16", 8192, 32768, 0.05),
        # odd sizes in 32 bits, forward and backward as two calls
        _policy("policy_ragged", "policy_apart", "f32", 1003, 50021, 0.05, 0.7),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    largest = {c["name"]: work(c)["bytes"] for c in listed()}
    kind = rng.choice(["embed", "embed_train", "embed_train", "conv", "conv_train", "step", "scan", "scan_train",
                       "scan_train", "policy", "policy", "policy_apart"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    while True:
        if kind in ("embed", "embed_train"):
            c = _embed(None, kind, dtype, _log(rng, 1, 65536), _log(rng, 2, 131072), _log(rng, 8, 4096))
            top = largest["embed_train"]
        elif kind in ("conv", "conv_train"):
            c = _conv(None, kind, dtype, _log(rng, 1, 16384), _log(rng, 1, 100), _log(rng, 32, 2048),
                      rng.choice([2, 3, 4, 4, 5, 7]), rng.random() < 0.7, rng.random() < 0.5, rng.random() < 0.5)
            top = largest["conv_train_long"]
        elif kind == "step":
            B = _log(rng, 1, 1024)
            return _step(None, dtype, B, _log(rng, 32, 2048), _log(rng, 2, 64), rng.choice([2, 3, 4, 4, 5]),
                         B + rng.randrange(64))
        elif kind in ("scan", "scan_train"):
            c = _scan(None, kind, dtype, _log(rng, 1, 8192), _log(rng, 1, 100), _log(rng, 32, 2048),
                      rng.choice([16, 16, 16, _log(rng, 2, 64)]), rng.random() < 0.7, rng.random() < 0.5,
                      rng.random() < 0.5)
            top = largest["scan_train_long"]
            if c["T"] * c["B"] * c["H"] * c["S"] > 8192 * 4 * 1024 * 16:
                continue
        else:
            c = _policy(None, kind, dtype, _log(rng, 1, 8192), _log(rng, 2, 131072), rng.choice([0.0, 0.05, 0.2]),
                        rng.choice([1.0, 1.0, 0.7, 2.0]))
            top = largest["policy_train"]
        if work(c)["bytes"] <= top:
            return c


def work(case):
    """Every input read once, every output written once; for the arithmetic the multiply-adds of the formulas, an
    exponential counted as one operation."""
    c, e = case, SIZE[case["dtype"]]
    if c["kind"] in ("embed", "embed_train"):
        N, V, D = c["N"], c["V"], c["D"]
        rows = min(N, V)                                 # (a row that several tokens name is read once)
        n = {"bytes": 8 * N + e * D * (rows + N), "flops": N * D}
        if c["kind"] == "embed_train":
            n["bytes"] += e * D * (N + V)
            n["flops"] += 2 * N * D
        return n
    if c["kind"] in ("conv", "conv_train"):
        n, s, W = c["T"] * c["B"] * c["H"], c["B"] * c["H"], c["W"]
        marks = c["T"] * c["B"] if c["reset"] else 0
        if c["kind"] == "conv":
            return {"bytes": 2 * e * n + 4 * s * 2 * (W - 1) + marks, "flops": (2 * W + 3) * n}
        return {"bytes": 5 * e * n + 4 * s * 4 * (W - 1) + 2 * marks, "flops": (8 * W + 12) * n}
    if c["kind"] == "step":
        B, H, S, W = c["B"], c["H"], c["S"], c["W"]
        return {"bytes": B * H * (4 * e + 8 * (W - 1 + S)) + B * 2 * S * e + 4 * H * (S + W + 3),
                "flops": B * H * (6 * S + 2 * W + 16)}
    if c["kind"] in ("scan", "scan_train"):
        n, s, S = c["T"] * c["B"] * c["H"], c["B"] * c["H"], c["S"]
        marks = c["T"] * c["B"] if c["reset"] else 0
        arrays, small = (4 if c["gated"] else 3), c["T"] * c["B"] * 2 * S * e
        if c["kind"] == "scan":
            return {"bytes": arrays * e * n + small + 8 * s * S + marks, "flops": (6 * S + 12) * n}
        # backward: x, dt, z and dy -> dx, ddt, dz
        back = 7 if c["gated"] else 5
        return {"bytes": (arrays + back) * e * n + 3 * small + 16 * s * S + 2 * marks, "flops": (22 * S + 40) * n}
    N, V = c["N"], c["V"]
    passes = 3 if c["kind"] == "policy_apart" else 2
    return {"bytes": N * (passes * V * e + 48), "flops": 6 * N * V}


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


def _blocks(c):
    """Rows of logits in blocks of at most 2^26 values."""
    step = max(1, (1 << 26) // c["V"])
    return [slice(i, min(i + step, c["N"])) for i in range(0, c["N"], step)]


def prepare(case, seed):
    c, gen, dt = dict(case), _generator(seed), DTYPES[case["dtype"]]
    dev = torch.device("cuda")
    randn = lambda *s: torch.randn(*s, generator=gen, device=dev)  # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=gen, device=dev)  # noqa: E731
    st = {"case": c}
    if c["kind"] in ("embed", "embed_train"):
        N, V, D = c["N"], c["V"], c["D"]
        st["table"] = (randn(V, D) / math.sqrt(D)).to(dt)
        # a few tokens are most of a text
        st["tokens"] = (V * rand(N) ** 4).long().clamp(max=V - 1)
        st["tokens"][rand(N) < 1 / 16] = -1              # padding
        st["scale"] = math.sqrt(D)
        if c["kind"] == "embed_train":
            st["dout"] = randn(N, D).to(dt)
        return st
    if c["kind"] == "step":
        B, H, S, W = c["B"], c["H"], c["S"], c["W"]
        st["xz"], st["x"] = randn(B, 2 * H).to(dt), randn(B, H).to(dt)
        st["slots"] = torch.randperm(c["slots"], generator=gen, device=dev)[:B].to(torch.int32)
        st["past"] = randn(c["slots"], W - 1, H)
        st["state"] = randn(c["slots"], H, S)
        rows = (B,)
    elif "W" in c:
        T, B, H, W = c["T"], c["B"], c["H"], c["W"]
        rows = (B, T) if c["batch_first"] else (T, B)
        st["xz"] = randn(*rows, 2 * H).to(dt)            # what one product gives for the convolution and a gate
        st["past"] = randn(B, W - 1, H)
        if c["kind"] == "conv_train":
            st["dy"], st["dlast"] = randn(*rows, H).to(dt), randn(B, W - 1, H)
    elif "S" in c:
        T, B, H, S = c["T"], c["B"], c["H"], c["S"]
        rows = (B, T) if c["batch_first"] else (T, B)
        st["xz"] = randn(*rows, 2 * H).to(dt)
        st["h0"] = randn(B, H, S)
        if c["kind"] == "scan_train":
            st["dy"], st["dh_last"] = randn(*rows, H).to(dt), randn(B, H, S)
    if "W" in c:
        st["weight"], st["bias"] = randn(c["H"], c["W"]) / math.sqrt(c["W"]), 0.1 * randn(c["H"])
    if "S" in c:
        # step sizes of 0.001 to 0.1 by channel, moved by the input; decays of 1 to S
        st["dbc"] = torch.cat([0.5 * randn(*rows, H), randn(*rows, 2 * S)], dim=-1).to(dt)
        d = torch.exp(math.log(0.001) + math.log(100.0) * rand(H))
        st["dt_bias"] = d + torch.log(-torch.expm1(-d))
        st["a"] = -torch.arange(1, S + 1, device=dev).float() * torch.exp(0.1 * randn(H, S))
        st["skip"] = 1 + 0.1 * randn(H)
    if "H" in c:
        st["reset"] = None
        if c.get("reset"):               # documents of about 700 tokens
            st["reset"] = (rand(T, B) < 1 / 700).to(torch.uint8)
        return st
    N, V = c["N"], c["V"]
    # a flat background and, in every row, a few tokens that stand out
    x = randn(N, V)
    u = rand(N, V) * (V / 16)
    x += 6 * u * (u < 1)
    if V > 256:                          # a vocabulary padded to a round size, and tokens that a mask forbids
        x[:, V - V // 128:] = -math.inf
        x[::3, : V // 8] = -math.inf
    st["logits"] = x.to(dt)
    lo, hi = (V // 8, V - V // 128) if V > 256 else (0, V)
    tok = torch.where(rand(N) < 0.7, x.argmax(1), torch.randint(lo, hi, (N,), generator=gen, device=dev))
    st["tokens"] = torch.where(rand(N) < 1 / 16, -1, tok)        # positions that were not sampled
    del x, u
    lp = torch.empty(N, dtype=torch.float64, device=dev)
    for i in _blocks(c):
        z = st["logits"][i].float() / c["temperature"]
        lp[i] = (z.gather(1, tok[i][:, None])[:, 0] - torch.logsumexp(z, 1)).double()
    # the policy has moved since it sampled; no ratio within a thousandth of where it is clipped (there 32 bits decide
    # one way or the other)
    moved = 0.25 * randn(N).double()
    for border in (math.log1p(-CLIP_LOW), math.log1p(CLIP_HIGH)):
        near = (moved - border).abs() < 1e-3
        moved = torch.where(near, moved + 3e-3, moved)
    st["old"] = (lp - moved).float()
    st["ref"] = (lp + 0.2 * randn(N)).float() if c["kl"] else None
    st["advantage"] = randn(N)
    st["weight"] = rand(N) / N
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _plain_embed(st):
    c, dt, tok = st["case"], DTYPES[st["case"]["dtype"]], st["tokens"]
    some, at = (tok >= 0)[:, None], tok.clamp(min=0)
    out = {"out": torch.where(some, st["scale"] * st["table"][at].float(), 0.0).to(dt)}
    if c["kind"] == "embed_train":
        grad = torch.zeros(c["V"], c["D"], device=tok.device)
        grad.index_add_(0, at, torch.where(some, st["dout"].float(), 0.0))
        out["dtable"] = (st["scale"] * grad).to(dt)
    return out


def _since_reset(reset, T, B, device):
    """Steps from the last reset (or from far before the start) to each step, [T,B]."""
    t = torch.arange(T, device=device)[:, None].expand(T, B)
    if reset is None:
        return t + (1 << 20)
    last = torch.cummax(torch.where(reset != 0, t, -(1 << 20)), 0).values
    return t - last


def _plain_conv(st):
    c = st["case"]
    T, B, H, W = c["T"], c["B"], c["H"], c["W"]
    dt, x = DTYPES[c["dtype"]], _time_major(c, st["xz"])[..., :H].float()
    dev = x.device
    ext = torch.cat([st["past"].transpose(0, 1), x])                     # [W-1+T,B,H]
    age = _since_reset(st["reset"], T, B, dev)
    p = st["bias"].expand(T, B, H).clone()
    seen = [(age >= W - 1 - k)[..., None] for k in range(W)]             # whether a step sees its input k
    for k in range(W):
        p += torch.where(seen[k], st["weight"][:, k] * ext[k:k + T], 0.0)
    sig = torch.sigmoid(p)
    y = p * sig if c["silu"] else p
    # what the next call goes on from: nothing before the last reset
    kept = torch.arange(W - 1, 0, -1, device=dev)[:, None] <= age[-1] + 1
    out = {"y": _time_major(c, y).to(dt).contiguous(),
           "last": torch.where(kept[..., None], ext[T:], 0.0).transpose(0, 1).contiguous()}
    if c["kind"] == "conv":
        return out
    dp = _time_major(c, st["dy"]).float()
    if c["silu"]:
        dp = dp * sig * (1 + p * (1 - sig))
    dext = torch.zeros_like(ext)
    dext[T:] = torch.where(kept[..., None], st["dlast"].transpose(0, 1), 0.0)
    dw = torch.empty_like(st["weight"])
    for k in range(W):
        dext[k:k + T] += torch.where(seen[k], st["weight"][:, k] * dp, 0.0)
        dw[:, k] = torch.where(seen[k], dp * ext[k:k + T], 0.0).sum((0, 1))
    out.update(dx=_time_major(c, dext[W - 1:]).to(dt).contiguous(), dweight=dw, dbias=dp.sum((0, 1)),
               dpast=dext[: W - 1].transpose(0, 1).contiguous())
    return out


def _linear_scan(a, b):
    """All h_t = a_t h_{t-1} + b_t along the first axis, h_0 = 0: composed over spans of 1, 2, 4, ... steps."""
    a, b, span = a.clone(), b.clone(), 1
    while span < len(a):
        b[span:] += a[span:] * b[:-span]
        a[span:] = a[span:] * a[:-span]
        span *= 2
    return b


def _softplus(x):
    return x.clamp(min=0) + torch.log1p(torch.exp(-x.abs()))


def _plain_scan(st):
    c = st["case"]
    H, S, dt = c["H"], c["S"], DTYPES[c["dtype"]]
    xz, dbc = _time_major(c, st["xz"]).float(), _time_major(c, st["dbc"]).float()
    x, z = xz[..., :H], xz[..., H:]
    raw, b, cm = dbc[..., :H] + st["dt_bias"], dbc[..., H:H + S], dbc[..., H + S:]
    d = _softplus(raw)
    a = torch.exp(d[..., None] * st["a"])                               # [T,B,H,S]
    if st["reset"] is not None:
        a = a * (st["reset"][..., None, None] == 0)
    u = (d * x)[..., None] * b[:, :, None]
    u[0] += a[0] * st["h0"]
    h = _linear_scan(a, u)
    del u
    s = (h * cm[:, :, None]).sum(-1) + st["skip"] * x
    sig = torch.sigmoid(z)
    g = z * sig if c["gated"] else torch.ones_like(x)
    out = {"y": _time_major(c, s * g).to(dt).contiguous(), "h_last": h[-1].clone()}
    if c["kind"] == "scan":
        return out
    dy = _time_major(c, st["dy"]).float()
    ds = dy * g
    lam = ds[..., None] * cm[:, :, None]
    lam[-1] += st["dh_last"]
    back = torch.cat([torch.zeros_like(a[:1]), a[1:].flip(0)])
    lam = _linear_scan(back, lam.flip(0)).flip(0)
    del back
    dc = (ds[..., None] * h).sum(2)
    past = torch.cat([st["h0"][None], h[:-1]]) * a * lam                 # lambda dh_t/d(log a_t)
    dd = (past * st["a"]).sum(-1)
    da = (past * d[..., None]).sum((0, 1))
    del past, h
    lb = (lam * b[:, :, None]).sum(-1)
    db = (lam * (d * x)[..., None]).sum(2)
    draw_ = (dd + lb * x) * torch.sigmoid(raw)
    dxz = [lb * d + ds * st["skip"]]
    if c["gated"]:
        dxz.append(dy * s * sig * (1 + z * (1 - sig)))
    out.update(dxz=_time_major(c, torch.cat(dxz, -1)).to(dt).contiguous(),
               ddbc=_time_major(c, torch.cat([draw_, db, dc], -1)).to(dt).contiguous(), da=da,
               dskip=(ds * x).sum((0, 1)), ddt_bias=draw_.sum((0, 1)), dh0=a[0] * lam[0])
    return out


def _plain_step(st):
    c = st["case"]
    H, S, dt, at = c["H"], c["S"], DTYPES[c["dtype"]], st["slots"].long()
    new = st["xz"][:, :H].float()
    window = torch.cat([st["past"][at], new[:, None]], 1)               # [B,W,H]
    p = st["bias"] + (window * st["weight"].t()).sum(1)
    # (the scan is of another layer: from a rounded result of this convolution its states would differ by roundings)
    x = st["x"].float()
    past, state = st["past"].clone(), st["state"].clone()
    past[at] = window[:, 1:]
    dbc, z = st["dbc"].float(), st["xz"][:, H:].float()
    d = _softplus(dbc[:, :H] + st["dt_bias"])
    h = torch.exp(d[..., None] * st["a"]) * state[at] + (d * x)[..., None] * dbc[:, None, H:H + S]
    state[at] = h
    y = ((h * dbc[:, None, H + S:]).sum(-1) + st["skip"] * x) * z * torch.sigmoid(z)
    return {"conv": (p * torch.sigmoid(p)).to(dt), "y": y.to(dt), "past": past, "state": state}


def _plain_policy(st):
    c, t = st["case"], st["case"]["temperature"]
    x = st["logits"].float() / t
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    s = e.sum(1, keepdim=True)
    at, some = st["tokens"].clamp(min=0), st["tokens"] >= 0
    # a row's loss, in 64 bits: exp(d) - d - 1 of small d
    lp = (x.gather(1, at[:, None]) - m)[:, 0].double() - torch.log(s[:, 0].double())
    ratio = torch.exp(lp - st["old"].double())
    gain, clipped = ratio * st["advantage"], ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * st["advantage"]
    loss, slope = -torch.minimum(gain, clipped), torch.where(gain <= clipped, -gain, 0.0)
    kl = torch.zeros_like(lp)
    if st["ref"] is not None:
        d = st["ref"].double() - lp
        kl = torch.expm1(d) - d
        loss, slope = loss + c["kl"] * kl, slope - c["kl"] * torch.expm1(d)
    w = torch.where(some, slope * st["weight"] / t, 0.0).float()[:, None]
    grad = (e / s * -w).scatter_add_(1, at[:, None], w)
    only = lambda v: torch.where(some, v, 0.0).float()  # noqa: E731
    return {"loss": only(loss), "logp": only(lp), "ratio": only(ratio), "kl": only(kl),
            "dlogits": grad.to(st["logits"].dtype)}


def _plain(st):
    kind = st["case"]["kind"]
    if kind in ("embed", "embed_train"):
        return _plain_embed(st)
    if kind in ("conv", "conv_train"):
        return _plain_conv(st)
    if kind in ("scan", "scan_train"):
        return _plain_scan(st)
    return _plain_step(st) if kind == "step" else _plain_policy(st)


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


def _new(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def _own_embed(mg, st, code):
    c, dt = st["case"], DTYPES[st["case"]["dtype"]]
    N, V, D = c["N"], c["V"], c["D"]
    cfg = mg.EmbedCfg(N, V, D, code, st["scale"])
    out = {"out": _kept(st, "out", lambda: _new(N, D, dtype=dt))}
    mg.embed_lookup(cfg, st["tokens"], st["table"], out["out"])
    if c["kind"] == "embed_train":
        out["dtable"] = _kept(st, "dtable", lambda: _new(V, D, dtype=dt))
        ws = _kept(st, "ws", lambda: _bytes(mg.embed_workspace_bytes(cfg)))
        mg.embed_backward(cfg, st["tokens"], st["dout"], out["dtable"], ws)
    return out


def _own_conv(mg, st, code):
    c, dt = st["case"], DTYPES[st["case"]["dtype"]]
    T, B, H, W = c["T"], c["B"], c["H"], c["W"]
    cfg = mg.ConvCfg(T, B, H, W, mg.CONV_SILU if c["silu"] else mg.CONV_LINEAR, code)
    x = _time_major(c, st["xz"])[..., :H]
    out = _kept(st, "out", lambda: {"y": _new(*st["xz"].shape[:2], H, dtype=dt), "last": _new(B, W - 1, H)})
    mg.causal_conv_forward(cfg, x, st["weight"], st["bias"], st["past"], st["reset"], _time_major(c, out["y"]),
                           out["last"])
    if c["kind"] == "conv":
        return out
    ws = _kept(st, "ws", lambda: _bytes(mg.causal_conv_workspace_bytes(cfg)))
    g = _kept(st, "grads", lambda: {"dx": torch.empty_like(st["dy"]), "dweight": _new(H, W), "dbias": _new(H),
                                    "dpast": _new(B, W - 1, H)})
    mg.causal_conv_backward(cfg, x, st["weight"], st["bias"], st["past"], st["reset"], _time_major(c, st["dy"]),
                            st["dlast"], _time_major(c, g["dx"]), g["dweight"], g["dbias"], g["dpast"], ws)
    return {**out, **g}


def _own_scan(mg, st, code):
    c, dt = st["case"], DTYPES[st["case"]["dtype"]]
    T, B, H, S = c["T"], c["B"], c["H"], c["S"]
    cfg = mg.SsmCfg(T, B, H, S, code)
    train = c["kind"] == "scan_train"

    def parts(xz, dbc):                  # x, dt, b, c, z
        xz, dbc = _time_major(c, xz), _time_major(c, dbc)
        return (xz[..., :H], dbc[..., :H], dbc[..., H:H + S], dbc[..., H + S:],
                xz[..., H:] if c["gated"] else None)

    inputs = parts(st["xz"], st["dbc"]) + (st["a"], st["skip"], st["dt_bias"])
    ws = _kept(st, "ws", lambda: _bytes(mg.ssm_workspace_bytes(cfg)))
    saved = _kept(st, "saved", lambda: _bytes(mg.ssm_saved_bytes(cfg))) if train else None
    out = _kept(st, "out", lambda: {"y": _new(*st["xz"].shape[:2], H, dtype=dt), "h_last": _new(B, H, S)})
    mg.ssm_forward(cfg, *inputs, st["h0"], st["reset"], _time_major(c, out["y"]), out["h_last"], saved, ws)
    if not train:
        return out
    g = _kept(st, "grads", lambda: {"dxz": _new(*st["xz"].shape[:2], 2 * H if c["gated"] else H, dtype=dt),
                                    "ddbc": torch.empty_like(st["dbc"]), "da": _new(H, S), "dskip": _new(H),
                                    "ddt_bias": _new(H), "dh0": _new(B, H, S)})
    mg.ssm_backward(cfg, *inputs, st["reset"], saved, _time_major(c, st["dy"]), st["dh_last"],
                    *parts(g["dxz"], g["ddbc"]), g["da"], g["dskip"], g["ddt_bias"], g["dh0"], ws)
    return {**out, **g}


def _own_step(mg, st, code):
    c, dt = st["case"], DTYPES[st["case"]["dtype"]]
    B, H, S, W = c["B"], c["H"], c["S"], c["W"]
    out = _kept(st, "out", lambda: {"conv": _new(B, H, dtype=dt), "y": _new(B, H, dtype=dt), "past": st["past"].clone(),
                                    "state": st["state"].clone()})
    dbc = st["dbc"]
    mg.causal_conv_step(mg.ConvCfg(1, B, H, W, mg.CONV_SILU, code), st["xz"][:, :H], st["weight"], st["bias"],
                        st["slots"], None, st["past"], out["past"], out["conv"])
    mg.ssm_step(mg.SsmCfg(1, B, H, S, code), st["x"], dbc[:, :H], dbc[:, H:H + S], dbc[:, H + S:], st["xz"][:, H:],
                st["a"], st["skip"], st["dt_bias"], st["slots"], None, st["state"], out["state"], out["y"])
    return out


def _own_policy(mg, st, code):
    c, dt = st["case"], DTYPES[st["case"]["dtype"]]
    N, V = c["N"], c["V"]
    cfg = mg.LogitsCfg(N, V, 0, code, c["temperature"])
    rule = mg.PolicyCfg(CLIP_LOW, CLIP_HIGH, c["kl"])
    ws = _kept(st, "ws", lambda: _bytes(mg.policy_workspace_bytes(cfg)))
    out = _kept(st, "out", lambda: {"loss": _new(N), "logp": _new(N), "ratio": _new(N), "kl": _new(N),
                                    "dlogits": _new(N, V, dtype=dt)})
    given = (st["logits"], st["tokens"], st["old"], st["ref"], st["advantage"])
    rows = (out["loss"], out["logp"], out["ratio"], out["kl"])
    if c["kind"] == "policy":
        mg.policy_loss(cfg, rule, *given, st["weight"], *rows, None, out["dlogits"], ws)
    else:
        stats = _kept(st, "stats", lambda: _new(N, 2))
        mg.policy_loss(cfg, rule, *given, None, *rows, stats, None, ws)
        mg.policy_loss_backward(cfg, rule, *given, stats, st["weight"], out["dlogits"])
    return out


def _own(st):
    import paper_2203_04738_amd as mg
    kind = st["case"]["kind"]
    code = {"f32": mg.MGRIT_F32, "bf16": mg.MGRIT_BF16, "f16": mg.MGRIT_F16}[st["case"]["dtype"]]
    if kind in ("embed", "embed_train"):
        return _own_embed(mg, st, code)
    if kind in ("conv", "conv_train"):
        return _own_conv(mg, st, code)
    if kind in ("scan", "scan_train"):
        return _own_scan(mg, st, code)
    return _own_step(mg, st, code) if kind == "step" else _own_policy(mg, st, code)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# the same outputs in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _exact_embed(st):
    c, tok = st["case"], st["tokens"]
    real = (tok >= 0).nonzero()[:, 0]
    out = torch.zeros(c["N"], c["D"], dtype=torch.float64, device=tok.device)
    out[real] = st["scale"] * st["table"].double()[tok[real]]
    if c["kind"] == "embed":
        return {"out": out}
    grad = torch.zeros(c["V"], c["D"], dtype=torch.float64, device=tok.device)
    grad.index_put_((tok[real],), st["scale"] * st["dout"][real].double(), accumulate=True)
    return {"out": out, "dtable": grad}


def _exact_conv(st):
    """Step by step, the window handed on; back through the same windows."""
    c = st["case"]
    T, B, H, W = c["T"], c["B"], c["H"], c["W"]
    x = _time_major(c, st["xz"])[..., :H].double()
    w, bias = st["weight"].double().t().contiguous(), st["bias"].double()          # [W,H]
    keep = torch.ones(T, B, 1, 1, dtype=torch.float64, device=x.device)
    if st["reset"] is not None:
        keep = (st["reset"] == 0).double()[..., None, None]
    window, windows, p = st["past"].double(), [], []
    for t in range(T):
        full = torch.cat([window * keep[t], x[t][:, None]], 1)                      # [B,W,H]
        windows.append(full)
        p.append(bias + (full * w).sum(1))
        window = full[:, 1:]
    p, act = torch.stack(p), c["silu"]
    gate = 1 / (1 + torch.exp(-p))
    out = {"y": _time_major(c, p * gate if act else p).contiguous(), "last": window.clone()}
    if c["kind"] == "conv":
        return out
    dp = _time_major(c, st["dy"]).double()
    dp = dp * (gate + p * gate * (1 - gate)) if act else dp
    carry, dx = st["dlast"].double(), torch.empty(T, B, H, dtype=torch.float64, device=x.device)
    dw = torch.zeros(W, H, dtype=torch.float64, device=x.device)
    for t in range(T - 1, -1, -1):
        full = dp[t][:, None] * w
        full[:, 1:] += carry
        dw += (dp[t][:, None] * windows[t]).sum(0)
        dx[t], carry = full[:, W - 1], full[:, : W - 1] * keep[t]
    return {**out, "dx": _time_major(c, dx).contiguous(), "dweight": dw.t().contiguous(), "dbias": dp.sum((0, 1)),
            "dpast": carry}


def _exact_scan(st):
    """Step by step, forward and back."""
    c = st["case"]
    T, B, H, S = c["T"], c["B"], c["H"], c["S"]
    xz, dbc = _time_major(c, st["xz"]).double(), _time_major(c, st["dbc"]).double()
    A, skip, dev = st["a"].double(), st["skip"].double(), xz.device
    raw = dbc[..., :H] + st["dt_bias"].double()
    step = torch.logaddexp(raw, torch.zeros_like(raw))
    keep = torch.ones(T, B, dtype=torch.float64, device=dev) if st["reset"] is None else (st["reset"] == 0).double()
    h = torch.empty(T + 1, B, H, S, dtype=torch.float64, device=dev)
    h[0] = st["h0"].double()
    s = torch.empty(T, B, H, dtype=torch.float64, device=dev)
    for t in range(T):
        past = torch.exp(step[t][..., None] * A) * (keep[t][:, None, None] * h[t])
        h[t + 1] = past + step[t][..., None] * xz[t, :, :H, None] * dbc[t, :, None, H:H + S]
        s[t] = (h[t + 1] * dbc[t, :, None, H + S:]).sum(-1) + skip * xz[t, :, :H]
    z = xz[..., H:]
    gate = z / (1 + torch.exp(-z)) if c["gated"] else torch.ones_like(z)
    out = {"y": _time_major(c, s * gate).contiguous(), "h_last": h[T].clone()}
    if c["kind"] == "scan":
        return out
    dy = _time_major(c, st["dy"]).double()
    ds, lam = dy * gate, st["dh_last"].double()
    dxz = torch.empty(T, B, 2 * H if c["gated"] else H, dtype=torch.float64, device=dev)
    ddbc = torch.empty(T, B, H + 2 * S, dtype=torch.float64, device=dev)
    da = torch.zeros(H, S, dtype=torch.float64, device=dev)
    for t in range(T - 1, -1, -1):
        lam = lam + ds[t][..., None] * dbc[t, :, None, H + S:]
        x, d = xz[t, :, :H], step[t]
        ddbc[t, :, H + S:] = (ds[t][..., None] * h[t + 1]).sum(1)
        ddbc[t, :, H:H + S] = ((d * x)[..., None] * lam).sum(1)
        lb = (lam * dbc[t, :, None, H:H + S]).sum(-1)
        lam = lam * torch.exp(d[..., None] * A) * keep[t][:, None, None]
        inner = lam * h[t]
        da += (inner * d[..., None]).sum(0)
        ddbc[t, :, :H] = (lb * x + (inner * A).sum(-1)) / (1 + torch.exp(-raw[t]))
        dxz[t, :, :H] = lb * d + ds[t] * skip
    if c["gated"]:
        sg = 1 / (1 + torch.exp(-z))
        dxz[..., H:] = dy * s * (sg + z * sg * (1 - sg))
    return {**out, "dxz": _time_major(c, dxz).contiguous(), "ddbc": _time_major(c, ddbc).contiguous(), "da": da,
            "dskip": (ds * xz[..., :H]).sum((0, 1)), "ddt_bias": ddbc[..., :H].sum((0, 1)), "dh0": lam}


def _exact_step(st):
    c, H, S = st["case"], st["case"]["H"], st["case"]["S"]
    past, state, xz, dbc = st["past"].double(), st["state"].double(), st["xz"].double(), st["dbc"].double()
    conv, ys = torch.empty_like(xz[:, :H]), torch.empty_like(xz[:, :H])
    for b, slot in enumerate(st["slots"].tolist()):
        window = torch.cat([past[slot], xz[b:b + 1, :H]])
        p = st["bias"].double() + (window.t() * st["weight"].double()).sum(1)
        past[slot] = window[1:]
        conv[b] = p / (1 + torch.exp(-p))
        x = st["x"][b].double()
        d = torch.logaddexp(dbc[b, :H] + st["dt_bias"].double(), torch.zeros_like(x))
        state[slot] = torch.exp(d[:, None] * st["a"].double()) * state[slot] + torch.outer(d * x, dbc[b, H:H + S])
        ys[b] = ((state[slot] * dbc[b, H + S:]).sum(1) + st["skip"].double() * x) * xz[b, H:] / (1 + torch.exp(-xz[b, H:]))
    return {"conv": conv, "y": ys, "past": past, "state": state}


def _exact_policy(st):
    c, t, parts = st["case"], st["case"]["temperature"], []
    for i in _blocks(c):
        x, tok = st["logits"][i].double() / t, st["tokens"][i]
        n, adv = torch.arange(len(tok), device=tok.device), st["advantage"][i].double()
        lse, p = torch.logsumexp(x, 1), torch.softmax(x, 1)
        lp = x[n, tok.clamp(min=0)] - lse
        r = torch.exp(lp - st["old"][i].double())
        # the smaller of the two gains counts: above the upper border of a good action, below the lower one of a bad
        # action, it does not move with the ratio
        up, low = (adv > 0) & (r > 1 + CLIP_HIGH), (adv < 0) & (r < 1 - CLIP_LOW)
        used = torch.where(up, 1 + CLIP_HIGH, torch.where(low, 1 - CLIP_LOW, r))
        loss, slope, kl = -adv * used, torch.where(up | low, 0.0, -adv * r), torch.zeros_like(lp)
        if st["ref"] is not None:
            d = st["ref"][i].double() - lp
            kl = torch.expm1(d) - d
            loss, slope = loss + c["kl"] * kl, slope + c["kl"] * (1 - torch.exp(d))
        loss, lp, r, kl, slope = (v.masked_fill(tok < 0, 0.0) for v in (loss, lp, r, kl, slope))
        coef = slope * st["weight"][i].double() / t
        grad = p * -coef[:, None]
        grad[n, tok.clamp(min=0)] += coef
        parts.append((loss, lp, r, kl, grad))
    return {k: torch.cat([p[j] for p in parts]) for j, k in enumerate(("loss", "logp", "ratio", "kl", "dlogits"))}


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("embed", "embed_train"):
        return _exact_embed(st)
    if kind in ("conv", "conv_train"):
        return _exact_conv(st)
    if kind in ("scan", "scan_train"):
        return _exact_scan(st)
    return _exact_step(st) if kind == "step" else _exact_policy(st)
