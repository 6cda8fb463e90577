"""Host-side checks of the operators over tokens: exported, bad arguments refused before anything touches the GPU, and what the
host code launches (on a stand-in for the HIP runtime)."""
import ctypes
import os
import re
import subprocess
import sys

import pytest
import torch

import paper_2203_04738_amd as mg
from paper_2203_04738_amd import ops, token_ops as tk
import test_ops_launch_limits as limits
import test_ops_launches as launches

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "mgrit_tokens.h")).read()
NULL, SIZE, ENUM, WORKSPACE, ALIGN = -1, -2, -4, -5, -6
P, BIG = 4096, 1 << 50                    # an aligned address that nothing reads
ref = ctypes.byref
runtime, threads_runtime = launches.runtime, limits.runtime


def test_every_declared_symbol_is_exported():
    names = re.findall(r"MGRIT_API\s+[\w\s\*]+?\b(\w+)\s*\(", HEADER)
    assert len(names) == 15
    for n in names:
        assert hasattr(tk._lib(), n) and hasattr(mg, n), n


@pytest.mark.parametrize("struct,cls", [("embed_cfg", mg.EmbedCfg), ("conv_cfg", mg.ConvCfg), ("ssm_cfg", mg.SsmCfg),
                                        ("ssm_inputs", tk.SsmInputs), ("ssm_grads", tk.SsmGrads), ("policy_cfg", mg.PolicyCfg)])
def test_structures_match_the_header(struct, cls):
    body = re.search(r"typedef struct \{((?:(?!typedef).)*?)\} " + struct + ";", HEADER, re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float, "glr_seq": ops.GlrSeq,
             "const float*": ctypes.c_void_p, "float*": ctypes.c_void_p}
    fields = [(n.strip(), kinds[kind]) for kind, ns in re.findall(
        r"(int32_t|int64_t|const float\*|float\*|float|glr_seq)\s+([\w,\s]+);", body) for n in ns.split(",")]
    assert fields == list(cls._fields_)


def test_constants_match_the_header():
    for name in ("CONV_LINEAR", "CONV_SILU"):
        assert int(re.search(name + r"\s*=\s*(\d+)", HEADER).group(1)) == getattr(mg, name)
    for name in ("CONV_MAX_W", "SSM_MAX_S"):
        assert int(re.search(name + r"\s+(\d+)", HEADER).group(1)) == getattr(mg, name)


def size(name, cfg):
    n = ctypes.c_size_t(0)
    return getattr(tk._lib(), name)(ref(cfg), ref(n)), n.value


def test_embedding_refusals():
    L = tk._lib()

    def strided(c, **kw):
        for k, v in kw.items():
            setattr(c, k, v)
        return c

    for cfg, code in ((mg.EmbedCfg(0, 2, 8), SIZE), (mg.EmbedCfg(4, 0, 8), SIZE), (mg.EmbedCfg(4, 2, 0), SIZE),
                      (mg.EmbedCfg((1 << 26) + 1, 2, 8), SIZE), (mg.EmbedCfg(4, (1 << 20) + 1, 8), SIZE),
                      (mg.EmbedCfg(4, 2, (1 << 20) + 1), SIZE), (strided(mg.EmbedCfg(4, 2, 8), ld_table=7), SIZE),
                      (strided(mg.EmbedCfg(4, 2, 8), ld_out=7), SIZE), (strided(mg.EmbedCfg(4, 2, 8), ld_out=1 << 41), SIZE),
                      (mg.EmbedCfg(4, 2, 8, 0, float("inf")), SIZE), (mg.EmbedCfg(4, 2, 8, 0, float("nan")), SIZE),
                      (mg.EmbedCfg(4, 2, 8, 2), ENUM)):
        assert size("embed_workspace_bytes", cfg)[0] == code
        assert L.embed_lookup(ref(cfg), P, P, P, None) == code
        assert L.embed_backward(ref(cfg), P, P, P, P, BIG, None) == code
    cfg = mg.EmbedCfg(100, 20, 8)
    rc, n = size("embed_workspace_bytes", cfg)
    assert rc == 0 and n >= 8 * 100 + 4 * 2 * 8 * 4
    assert L.embed_workspace_bytes(None, None) == NULL and L.embed_workspace_bytes(ref(cfg), None) == NULL
    for i in range(3):
        args = [P, P, P]
        args[i] = None
        assert L.embed_lookup(ref(cfg), *args, None) == NULL
        args[i] = P + (4 if i == 0 else 2)
        assert L.embed_lookup(ref(cfg), *args, None) == ALIGN
    for i in range(4):
        args = [P, P, P, P]
        args[i] = None
        assert L.embed_backward(ref(cfg), *args, BIG, None) == NULL
        args[i] = P + (4 if i in (0, 3) else 2)
        assert L.embed_backward(ref(cfg), *args, BIG, None) == ALIGN
    assert L.embed_backward(ref(cfg), P, P, P, P, n - 1, None) == WORKSPACE


def seq(data=P, t=16, b=8):
    return ref(ops.GlrSeq(data, t, b))


def test_convolution_refusals():
    L = tk._lib()

    def forward(cfg=mg.ConvCfg(5, 2, 8, 4), x=None, weight=P, bias=P, past=P, y=None, last=3 * P):
        return L.causal_conv_forward(ref(cfg), x or seq(), weight, bias, past, None, y or seq(), last, None)

    def backward(cfg=mg.ConvCfg(5, 2, 8, 4), x=None, weight=P, dy=None, dlast=P, dx=None, dw=P, db=P, dp=3 * P, ws=P, n=BIG):
        return L.causal_conv_backward(ref(cfg), x or seq(), weight, P, P, None, dy or seq(), dlast, dx or seq(), dw, db, dp, ws, n,
                                      None)

    for cfg, code in ((mg.ConvCfg(0, 2, 8, 4), SIZE), (mg.ConvCfg(5, 0, 8, 4), SIZE), (mg.ConvCfg(5, 2, 0, 4), SIZE),
                      (mg.ConvCfg(5, 2, 8, 0), SIZE), (mg.ConvCfg(5, 2, 8, 9), SIZE), (mg.ConvCfg(1 << 20, 1 << 11, 1, 2), SIZE),
                      (mg.ConvCfg(8, 1 << 16, 1 << 15, 2), SIZE), (mg.ConvCfg(5, 2, 8, 4, 2), ENUM),
                      (mg.ConvCfg(5, 2, 8, 4, 0, 3), ENUM)):
        assert size("causal_conv_workspace_bytes", cfg)[0] == code and forward(cfg) == code and backward(cfg) == code
    rc, n = size("causal_conv_workspace_bytes", mg.ConvCfg(5, 2, 8, 4))
    assert rc == 0 and n >= 4 * 8 * 5
    assert forward(x=seq(None)) == NULL and forward(y=seq(None)) == NULL and forward(weight=None) == NULL
    assert forward(x=seq(P + 2)) == ALIGN and forward(weight=P + 2) == ALIGN and forward(bias=P + 2) == ALIGN
    assert forward(past=P + 2) == ALIGN and forward(last=P + 2) == ALIGN
    assert forward(last=P) == SIZE and forward(mg.ConvCfg(5, 2, 8, 4), past=2 * P, last=2 * P) == SIZE    # the past itself
    assert backward(dp=P) == SIZE and backward(dlast=2 * P, dp=2 * P) == SIZE
    assert forward(x=seq(P, -16, 8)) == SIZE
    for t, b in ((0, 8), (15, 8), (8, 8), (16, 7), (7, 1 << 20)):            # outputs that would overlap themselves
        assert forward(y=seq(P, t, b)) == SIZE and backward(dx=seq(P, t, b)) == SIZE
    assert backward(dy=seq(None)) == NULL and backward(dx=seq(None)) == NULL and backward(ws=None) == NULL
    assert backward(weight=None) == NULL and backward(ws=P + 8) == ALIGN and backward(n=n - 1) == WORKSPACE
    for k in ("dlast", "dw", "db", "dp"):
        assert backward(**{k: P + 2}) == ALIGN

    def step(cfg=mg.ConvCfg(1, 4, 8, 4), slots=P, n=4, past=P, out=P, y=None, weight=P):
        return L.causal_conv_step(ref(cfg), seq(), weight, P, slots, n, None, past, out, y or seq(), None)

    assert step(cfg=mg.ConvCfg(2, 4, 8, 4)) == SIZE and step(n=0) == SIZE and step(slots=None, n=3) == SIZE
    assert step(past=None) == NULL and step(out=None) == NULL and step(weight=None) == NULL
    assert step(past=P + 2) == ALIGN and step(out=P + 2) == ALIGN and step(slots=P + 2) == ALIGN
    assert step(y=seq(P, 0, 7)) == SIZE


def inputs(z=True, **other):
    s = ops.GlrSeq(P, 16, 8)
    i = tk.SsmInputs(s, s, s, s, s if z else ops.GlrSeq(), P, P, P)
    for k, v in other.items():
        setattr(i, k, v)
    return i


def grads(z=True, **other):
    s = ops.GlrSeq(P, 16, 8)
    g = tk.SsmGrads(s, s, s, s, s if z else ops.GlrSeq(), P, P, P, P)
    for k, v in other.items():
        setattr(g, k, v)
    return g


def test_scan_refusals():
    L, ok = tk._lib(), mg.SsmCfg(100, 2, 8, 4)

    def forward(cfg=ok, i=inputs(), h0=P, y=None, saved=P, saved_n=BIG, ws=P, n=BIG, h_last=3 * P):
        return L.ssm_forward(ref(cfg), ref(i) if i else None, h0, None, y or seq(), h_last, saved, saved_n, ws, n, None)

    def backward(cfg=ok, i=inputs(), saved=P, saved_n=BIG, dy=None, dh=3 * P, g=grads(), ws=P, n=BIG):
        return L.ssm_backward(ref(cfg), ref(i) if i else None, None, saved, saved_n, dy or seq(), dh, ref(g) if g else None, ws, n,
                              None)

    for cfg, code in ((mg.SsmCfg(0, 2, 8, 4), SIZE), (mg.SsmCfg(5, 0, 8, 4), SIZE), (mg.SsmCfg(5, 2, 0, 4), SIZE),
                      (mg.SsmCfg(5, 2, 8, 0), SIZE), (mg.SsmCfg(5, 2, 8, 65), SIZE), (mg.SsmCfg(1 << 20, 1 << 11, 1, 1), SIZE),
                      (mg.SsmCfg(1, 1 << 16, 1 << 15, 1), SIZE), (mg.SsmCfg(1, 1 << 14, 1 << 14, 64), SIZE),
                      (mg.SsmCfg(5, 2, 8, 4, 2), ENUM)):
        assert size("ssm_workspace_bytes", cfg)[0] == code and size("ssm_saved_bytes", cfg)[0] == code
        assert forward(cfg) == code and backward(cfg) == code
    (_, n), (_, saved) = size("ssm_workspace_bytes", ok), size("ssm_saved_bytes", ok)
    assert n > 0 and saved == 4 * 13 * 2 * 8 * 4
    assert forward(i=None) == NULL and forward(i=inputs(a=None)) == NULL and forward(y=seq(None)) == NULL
    for k in ("x", "dt", "b", "c"):
        assert forward(i=inputs(**{k: ops.GlrSeq()})) == NULL and backward(i=inputs(**{k: ops.GlrSeq()})) == NULL
        assert forward(i=inputs(**{k: ops.GlrSeq(P + 2, 16, 8)})) == ALIGN
        assert forward(i=inputs(**{k: ops.GlrSeq(P, -1, 8)})) == SIZE
    assert forward(i=inputs(z=False), y=seq(P, 7, 1600)) == SIZE
    for k in ("a", "skip", "bias"):
        assert forward(i=inputs(**{k: P + 2})) == ALIGN
    assert forward(saved=P + 8) == ALIGN and forward(saved_n=saved - 1) == WORKSPACE and forward(h0=P + 1) == ALIGN
    assert forward(n=n - 1) == WORKSPACE and forward(ws=None) == NULL and forward(ws=P + 4) == ALIGN
    assert forward(h_last=P) == SIZE and backward(dh=P) == SIZE                          # h0, dh0 themselves
    assert backward(saved=None) == NULL and backward(g=None) == NULL and backward(g=grads(da=None)) == NULL
    assert backward(i=inputs(z=False)) == NULL and backward(g=grads(z=False)) == NULL
    assert backward(saved_n=saved - 1) == WORKSPACE and backward(n=n - 1) == WORKSPACE and backward(dy=seq(None)) == NULL
    for k in ("dx", "ddt", "db", "dc", "dz"):
        assert backward(g=grads(**{k: ops.GlrSeq(P, 16, 3)})) == SIZE
    for k in ("da", "dskip", "dbias", "dh0"):
        assert backward(g=grads(**{k: P + 2})) == ALIGN

    def step(cfg=mg.SsmCfg(1, 4, 8, 4), i=inputs(), slots=P, n=4, state=P, out=P, y=None):
        return L.ssm_step(ref(cfg), ref(i) if i else None, slots, n, None, state, out, y or seq(), None)

    assert step(cfg=mg.SsmCfg(2, 4, 8, 4)) == SIZE and step(n=0) == SIZE and step(slots=None, n=3) == SIZE
    assert step(i=None) == NULL and step(state=None) == NULL and step(out=None) == NULL
    assert step(state=P + 2) == ALIGN and step(slots=P + 2) == ALIGN and step(y=seq(P, 0, 7)) == SIZE


def test_a_result_that_begins_where_another_array_does_is_refused():
    """All other arguments are right: without the refusal the call would try to launch."""
    L, at = tk._lib(), [1 << 20]

    def new():
        at[0] += 1 << 20
        return at[0]

    cfg = mg.EmbedCfg(4, 5, 8)
    p = new()
    assert L.embed_lookup(ref(cfg), new(), p, p, None) == SIZE
    assert L.embed_backward(ref(cfg), new(), p, p, new(), BIG, None) == SIZE
    assert L.embed_backward(ref(cfg), new(), new(), p, p, BIG, None) == SIZE
    cfg = mg.ConvCfg(5, 2, 8, 4)
    assert L.causal_conv_forward(ref(cfg), seq(p), new(), None, None, None, seq(p), None, None) == SIZE
    for x, dy in ((p, new()), (new(), p)):
        assert L.causal_conv_backward(ref(cfg), seq(x), new(), None, None, None, seq(dy), None, seq(p), new(), None, None, new(),
                                      BIG, None) == SIZE
    assert L.causal_conv_backward(ref(cfg), seq(new()), new(), None, p, None, seq(new()), None, seq(new()), new(), None, p, new(),
                                  BIG, None) == SIZE
    assert L.causal_conv_step(ref(mg.ConvCfg(1, 2, 8, 4)), seq(p), new(), None, None, 2, None, new(), new(), seq(p), None) == SIZE
    cfg, names = mg.SsmCfg(100, 2, 8, 8), ("x", "dt", "b", "c", "z")

    def group(cls, **other):
        g = cls()
        for n in names:
            name = "d" + n if cls is tk.SsmGrads else n
            setattr(g, name, ops.GlrSeq(other.get(n) or new(), 16, 8))
        if cls is tk.SsmGrads:
            g.da = new()
        else:
            g.a = new()
        return g

    for n in names:
        assert L.ssm_step(ref(mg.SsmCfg(1, 2, 8, 8)), ref(group(tk.SsmInputs, **{n: p})), None, 2, None, new(), new(), seq(p),
                          None) == SIZE
        assert L.ssm_forward(ref(cfg), ref(group(tk.SsmInputs, **{n: p})), None, None, seq(p), None, None, 0, new(), BIG, None) == SIZE
        for inputs_, dy, out in ((dict(x=p), new(), {n: p}), ({}, p, {n: p}), ({}, new(), {n: p, "x" if n != "x" else "z": p})):
            assert L.ssm_backward(ref(cfg), ref(group(tk.SsmInputs, **inputs_)), None, new(), BIG, seq(dy), None,
                                  ref(group(tk.SsmGrads, **out)), new(), BIG, None) == SIZE
    cfg, rule = mg.LogitsCfg(4, 100, 0), mg.PolicyCfg()
    names = ("logits", "tok", "old", "ref", "adv", "w", "loss", "logp", "ratio", "kl", "stats", "grad")
    for k in names[6:11]:
        for other in names:
            a = {n: new() for n in names}
            a[k] = a[other]
            if k != other:
                assert L.policy_loss(ref(cfg), ref(rule), *(a[n] for n in names), None, 0, None) == SIZE, (k, other)


def test_a_gradient_that_begins_where_another_array_of_its_rows_does_is_refused():
    """Workgroups of other rows read those arrays while gradients are written; the logits alone may be the gradient."""
    L, cfg, rule = tk._lib(), mg.LogitsCfg(4, 100, 0), mg.PolicyCfg()
    names = ("logits", "tok", "old", "ref", "adv", "w", "loss", "logp", "ratio", "kl", "stats", "grad")
    for k in names[1:11]:
        a = {n: (i + 1) << 20 for i, n in enumerate(names)}
        a["grad"] = a[k]
        assert L.policy_loss(ref(cfg), ref(rule), *(a[n] for n in names), None, 0, None) == SIZE, k
        if k in ("loss", "logp", "ratio", "kl"):
            continue
        given = [a[n] for n in ("logits", "tok", "old", "ref", "adv", "stats", "w", "grad")]
        assert L.policy_loss_backward(ref(cfg), ref(rule), *given, None) == SIZE, k


def test_policy_refusals():
    L = tk._lib()

    def cfg(N=4, V=100, dtype=0, t=1.0, ld=None, ld_grad=None):
        c = mg.LogitsCfg(N, V, 0, dtype, t)
        c.ld, c.ld_grad = ld or V, ld_grad or V
        return c

    def both(c=None, rule=mg.PolicyCfg(0.2, 0.3, 0.1), code=0, **kw):
        a = dict(logits=P, tok=P, old=P, ref=P, adv=P, w=P, loss=P, logp=P, ratio=P, kl=P, stats=P, grad=P + 65536)
        a.update(kw)
        c = c or cfg()
        r = ref(rule) if rule else None
        got = [L.policy_loss(ref(c), r, a["logits"], a["tok"], a["old"], a["ref"], a["adv"], a["w"], a["loss"], a["logp"],
                             a["ratio"], a["kl"], a["stats"], a["grad"], P, BIG, None)]
        if not set(kw) & {"loss", "logp", "ratio", "kl"}:
            got.append(L.policy_loss_backward(ref(c), r, a["logits"], a["tok"], a["old"], a["ref"], a["adv"], a["stats"], a["w"],
                                              a["grad"], None))
        return set(got)

    for c, code in ((cfg(N=0), SIZE), (cfg(V=0), SIZE), (cfg(V=(1 << 20) + 1), SIZE), (cfg(ld=99), SIZE), (cfg(ld_grad=99), SIZE),
                    (cfg(dtype=2), ENUM), (cfg(t=0.0), SIZE), (cfg(t=float("nan")), SIZE)):
        assert both(c) == {code}
    for rule in (mg.PolicyCfg(-0.1, 0.2), mg.PolicyCfg(1.1, 0.2), mg.PolicyCfg(0.2, -0.1), mg.PolicyCfg(0.2, float("inf")),
                 mg.PolicyCfg(float("nan"), 0.2), mg.PolicyCfg(0.2, 0.2, -1.0), mg.PolicyCfg(0.2, 0.2, float("nan"))):
        assert both(rule=rule) == {SIZE}
    for k in ("logits", "tok", "old", "adv"):
        assert both(**{k: None}) == {NULL}
    assert both(rule=None) == {NULL} and both(loss=None) == {NULL}
    for k in ("tok", "old", "ref", "adv", "w", "loss", "logp", "ratio", "kl", "stats"):
        assert both(**{k: P + 2}) == {ALIGN}, k
    assert both(logits=P + 2) == {ALIGN} and both(grad=P + 65538) == {ALIGN}
    assert both(cfg(ld=200), grad=P) == {SIZE}                # in place with another stride
    long = cfg(V=50000)
    rc, n = size("policy_workspace_bytes", long)
    assert rc == 0 and n > 0 and size("policy_workspace_bytes", cfg()) == (0, 0)
    r = ref(mg.PolicyCfg())
    call = lambda ws, n: L.policy_loss(ref(long), r, P, P, P, None, P, None, P, None, None, None, None, None, ws, n, None)  # noqa: E731
    assert call(P, n - 1) == WORKSPACE and call(None, n) == NULL and call(P + 8, n) == ALIGN


def test_the_binding_refuses_other_tensors():
    z = torch.zeros
    ws = z(0, dtype=torch.uint8)
    tok = z(4, dtype=torch.int64)
    e = mg.EmbedCfg(4, 9, 8)
    with pytest.raises(ValueError, match="table: expected shape"):
        mg.embed_lookup(e, tok, z(9, 7), z(4, 8))
    with pytest.raises(TypeError, match="tokens: expected dtype"):
        mg.embed_lookup(e, tok.int(), z(9, 8), z(4, 8))
    with pytest.raises(ValueError, match="tokens: tensor must be contiguous"):
        mg.embed_lookup(e, z(8, dtype=torch.int64)[::2], z(9, 8), z(4, 8))
    with pytest.raises(TypeError, match="tokens: expected a CUDA tensor"):
        mg.embed_lookup(e, tok, z(9, 8), z(4, 8))
    with pytest.raises(TypeError, match="dout: expected a CUDA tensor"):
        mg.embed_backward(e, tok, [1], z(9, 8), ws)
    s = mg.SsmCfg(5, 2, 8, 4)
    x, b, a = z(5, 2, 8), z(5, 2, 4), z(8, 4)
    with pytest.raises(ValueError, match="c: expected shape"):
        mg.ssm_forward(s, x, x, b, x, None, a, None, None, None, None, x, None, None, ws)
    with pytest.raises(ValueError, match="x: the last dimension must be contiguous"):
        mg.ssm_forward(s, z(8, 2, 5).permute(2, 1, 0), x, b, b, None, a, None, None, None, None, x, None, None, ws)
    with pytest.raises(ValueError, match="dz: expected shape"):
        mg.ssm_backward(s, x, x, b, b, x, a, None, None, None, ws, x, None, x, x, b, b, b, a, None, None, None, ws)
    with pytest.raises(ValueError, match="state_out: expected shape"):
        mg.ssm_step(mg.SsmCfg(1, 2, 8, 4), x[0], x[0], b[0], b[0], None, a, None, None, None, None, z(3, 8, 4), z(4, 8, 4), x[0])
    c = mg.ConvCfg(5, 2, 8, 4)
    with pytest.raises(ValueError, match="past: expected shape"):
        mg.causal_conv_forward(c, x, z(8, 4), None, z(2, 4, 8), None, x, None)
    with pytest.raises(TypeError, match="x: expected dtype"):
        mg.causal_conv_forward(c, x.half(), z(8, 4), None, None, None, x, None)
    lc, lg = mg.LogitsCfg(4, 9, 0), z(4, 9)
    with pytest.raises(ValueError, match="advantage: expected shape"):
        mg.policy_loss(lc, mg.PolicyCfg(), lg, tok, z(4), None, z(5), None, z(4), None, None, None, None, None, ws)
    assert (lc.ld, e.ld_table, e.ld_out) == (9, 8, 8)


def test_tensors_of_another_device_are_refused(monkeypatch):
    # (a tensor says where it is; nothing is read)
    class On1(torch.Tensor):
        is_cuda = True

        def get_device(self):
            return 1

    t = torch.zeros(4, dtype=torch.int64).as_subclass(On1)
    with pytest.raises(ValueError, match="tokens: tensor on cuda:1, the current device is cuda:0"):
        tk._explain([(t, "tokens", torch.int64, (4,), 0)], 0)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(ops, "_stream", lambda: 0)
    with pytest.raises(ValueError, match="the current device is cuda:0"):
        tk._call("embed_lookup", mg.EmbedCfg(4, 9, 8), (t, "tokens", torch.int64, (4,), 0))


CALL = """
import ctypes, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
from ctypes import byref
import paper_2203_04738_amd as mg
from paper_2203_04738_amd import binding, ops, token_ops as tk
L, entry, n = tk._prototypes(ops._prototypes(binding.lib())), sys.argv[2], [int(a) for a in sys.argv[3:]]
A, big = [(i + 1) << 44 for i in range(16)], 1 << 60
if entry.startswith("embed"):
    c = mg.EmbedCfg(*n)
elif entry.startswith("causal"):
    c = mg.ConvCfg(*n)
elif entry.startswith("ssm"):
    c = mg.SsmCfg(*n)
else:
    c = mg.LogitsCfg(n[0], n[1], 0, *n[2:])
if entry[:3] in ("cau", "ssm"):
    T, B, H = n[:3]
    s = [ops.GlrSeq(a, B * H, H) for a in A]
if entry == "embed_lookup":
    rc = L.embed_lookup(byref(c), A[0], A[1], A[2], None)
elif entry == "embed_backward":
    rc = L.embed_backward(byref(c), A[0], A[1], A[2], A[3], big, None)
elif entry == "causal_conv_forward":
    rc = L.causal_conv_forward(byref(c), byref(s[0]), A[1], A[2], None, None, byref(s[3]), A[4], None)
elif entry == "causal_conv_backward":
    rc = L.causal_conv_backward(byref(c), byref(s[0]), A[1], A[2], None, None, byref(s[3]), None, byref(s[4]), A[5], A[6], None,
                                A[7], big, None)
elif entry == "causal_conv_step":
    rc = L.causal_conv_step(byref(c), byref(s[0]), A[1], A[2], None, B, None, A[3], A[4], byref(s[5]), None)
elif entry.startswith("ssm"):
    S = n[3]
    bc = [ops.GlrSeq(a, B * S, S) for a in A]
    i = tk.SsmInputs(s[0], s[1], bc[2], bc[3], s[4], A[5], A[6], A[7])
    g = tk.SsmGrads(s[8], s[9], bc[10], bc[11], s[12], A[13], None, None, None)
    if entry == "ssm_forward":
        rc = L.ssm_forward(byref(c), byref(i), None, None, byref(s[8]), A[9], A[10], big, A[11], big, None)
    elif entry == "ssm_backward":
        rc = L.ssm_backward(byref(c), byref(i), None, A[14], big, byref(s[15]), None, byref(g), 17 << 44, big, None)
    else:
        rc = L.ssm_step(byref(c), byref(i), None, B, None, A[9], A[10], byref(s[11]), None)
elif entry == "policy_loss":
    rc = L.policy_loss(byref(c), byref(mg.PolicyCfg()), *A[:6], A[6], None, None, None, None, A[7], A[8], big, None)
else:
    rc = L.policy_loss_backward(byref(c), byref(mg.PolicyCfg()), *A[:5], A[5], A[6], A[7], None)
print("returned", rc)
"""


def call(runtime, entry, *sizes, **env):
    """(what the call returned, [(workgroups, kernel)])"""
    r = subprocess.run([sys.executable, "-c", CALL, runtime, entry, *(str(v) for v in sizes)], cwd=ROOT,
                       env=dict(os.environ, **env), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    lines = [line.split(" ", 2) for line in r.stdout.splitlines()]
    (rc,) = (int(f[1]) for f in lines if f[0] == "returned")
    return rc, [(int(f[1]), f[2]) for f in lines if f[0] in ("launched", "failed")]


@pytest.mark.parametrize("entry,sizes,kernels", [
    ("embed_lookup", (8, 100, 64), ["embed_lookup_kernel<float, true>"]),
    ("embed_lookup", (8, 100, 63, 1), ["embed_lookup_kernel<mg::Bf16, false>"]),
    ("embed_backward", (8, 100, 64), ["embed_plan_kernel<float, true, 128>", "embed_sum_kernel<float, true, 8>"]),
    ("embed_backward", (8193, 100, 64), ["embed_plan_kernel<float, true, 512>", "embed_sum_kernel<float, true, 32>",
                                         "embed_join_kernel<float, true>"]),
    ("embed_backward", (33, 32769, 64, 1), ["embed_plan_kernel<mg::Bf16, true, 512>", "embed_sum_kernel<mg::Bf16, true, 8>",
                                            "embed_join_kernel<mg::Bf16, true>"]),
    ("embed_backward", (33, 131073, 3, 4), ["embed_plan_kernel<mg::F16, false, 2048>", "embed_sum_kernel<mg::F16, false, 8>",
                                            "embed_join_kernel<mg::F16, false>"]),
    ("causal_conv_forward", (100, 2, 130, 4), ["conv_forward_kernel<float, 2, 4>"]),
    ("causal_conv_forward", (100, 2, 33, 1, 0, 1), ["conv_forward_kernel<mg::Bf16, 1, 8>"]),
    ("causal_conv_backward", (100, 2, 130, 2, 1, 4), ["conv_backward_kernel<mg::F16, 2, 2>", "conv_params_kernel"]),
    ("causal_conv_backward", (100, 2, 31, 3), ["conv_backward_kernel<float, 1, 3>", "conv_params_kernel"]),
    ("causal_conv_step", (1, 4, 8, 4), ["conv_step_kernel<float>"]),
    ("ssm_forward", (16, 2, 70, 16), ["ssm_forward_kernel<float, 4, true>"]),
    ("ssm_forward", (128, 100, 1000, 16), ["ssm_forward_kernel<float, 4, true>"]),
    ("ssm_forward", (777, 3, 500, 16, 1), ["ssm_forward_kernel<mg::Bf16, 4, false>", "ssm_forward_kernel<mg::Bf16, 4, true>"]),
    ("ssm_forward", (4096, 1, 64, 3, 4), ["ssm_forward_kernel<mg::F16, 1, false>", "ssm_between_kernel",
                                          "ssm_forward_kernel<mg::F16, 1, true>"]),
    ("ssm_backward", (16, 2, 70, 64), ["ssm_backward_kernel<float, 16, 4>", "ssm_bc_kernel<float>", "ssm_params_kernel"]),
    ("ssm_backward", (777, 3, 500, 17), ["ssm_adjoint_ends_kernel<float, 8>", "ssm_backward_kernel<float, 8, 8>",
                                         "ssm_bc_kernel<float>", "ssm_params_kernel"]),
    ("ssm_backward", (4096, 1, 64, 8, 1), ["ssm_adjoint_ends_kernel<mg::Bf16, 2>", "ssm_between_kernel",
                                           "ssm_backward_kernel<mg::Bf16, 2, 8>", "ssm_bc_kernel<mg::Bf16>", "ssm_params_kernel"]),
    ("ssm_step", (1, 4, 8, 16), ["ssm_step_kernel<float, 4>"]),
    ("policy_loss", (100, 51), ["policy_kernel<float, 1>"]),
    ("policy_loss", (8, 8192), ["policy_kernel<float, 4>"]),
    ("policy_loss", (8, 32768, 1), ["policy_kernel<mg::Bf16, 16>"]),
    ("policy_loss", (64, 50000), ["distill_segment_kernel<float>", "policy_join_kernel<float>",
                                  "policy_grad_kernel<float, 16, false>"]),
    ("policy_loss_backward", (64, 500), ["policy_grad_kernel<float, 1, false>"]),
    ("policy_loss_backward", (64, 50000, 1), ["policy_grad_kernel<mg::Bf16, 16, false>"])])
def test_kernels_of_a_call_and_launches_that_fail(runtime, entry, sizes, kernels):
    rc, got = call(runtime, entry, *sizes)
    names = [name.replace("void mg::", "mg::") for _, name in got]
    assert rc == 0 and len(names) == len(kernels), names
    assert all("mg::" + k in n for k, n in zip(kernels, names)), names
    assert all(0 < groups < 2 ** 31 for groups, _ in got)
    for k in kernels:                                            # a failing launch ends the call and is reported
        rc, got = call(runtime, entry, *sizes, FAKE_HIP_FAIL=k.split("<")[0])
        assert rc == -7 and len(got) <= len(kernels)


M = 1 << 20


@pytest.mark.parametrize("entry,fits,more", [
    ("embed_lookup", (4 * M - 1, 9, 4096), (4 * M, 9, 4096)),
    ("embed_backward", (64 * M - 32, 9, 1024), (64 * M, 9, 1025)),
    ("causal_conv_forward", (2, 256 * M - 16, 1, 4), (2, 256 * M, 1, 4)),
    ("causal_conv_backward", (2, 256 * M - 16, 1, 4), (2, 256 * M, 1, 4)),
    ("ssm_forward", (2, 16 * M - 1, 2, 4), (2, 16 * M, 2, 4)),
    ("ssm_backward", (2, 16 * M - 1, 2, 4), (2, 16 * M, 2, 4)),
    ("ssm_backward", (64, 16 * M - 1, 2, 3), (64, 16 * M - 1, 2, 5)),
    ("causal_conv_step", (1, 64 * M, 8, 4), (1, 128 * M, 32, 4)),
    ("ssm_step", (1, 64 * M - 4, 16, 4), (1, 64 * M, 16, 4)),
    ("policy_loss", (4 * M - 1, 20000), (4 * M, 20000)),
    ("policy_loss", (2 * M - 1, 50000), (2 * M, 50000)),
    ("policy_loss_backward", (16 * M - 1, 5000), (16 * M, 5000))])
def test_launches_of_less_than_2_to_the_32_threads(threads_runtime, entry, fits, more):
    rc, got = call(threads_runtime, entry, *fits)
    assert rc == 0 and got and all(0 < n < 2 ** 32 for n, _ in got), (rc, got)
    assert call(threads_runtime, entry, *more) == (SIZE, [])
