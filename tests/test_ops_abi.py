"""Host-side checks of the operators' entry points: exported, and bad arguments refused before anything touches the GPU."""
import ctypes
import os
import re

import pytest
import torch

import paper_2203_04738_amd as mg
from paper_2203_04738_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "mgrit_ops.h")).read()
NULL, SIZE, ENUM, WORKSPACE, ALIGN = -1, -2, -4, -5, -6
P = 4096                                  # an aligned address that nothing reads


def test_every_declared_symbol_is_exported():
    names = re.findall(r"MGRIT_API\s+[\w\s\*]+?\b(\w+)\s*\(", HEADER)
    assert len(names) == 13
    for n in names:
        assert hasattr(ops._lib(), n), n


@pytest.mark.parametrize("struct,cls", [("glr_cfg", mg.GlrCfg), ("glr_seq", ops.GlrSeq), ("logits_cfg", mg.LogitsCfg),
                                        ("q8_cfg", mg.Q8Cfg)])
def test_structures_match_the_header(struct, cls):
    body = re.search(r"typedef struct \{((?:(?!typedef).)*?)\} " + struct + ";", HEADER, re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float, "void*": ctypes.c_void_p}
    fields = [(n.strip(), kinds[kind]) for kind, ns in re.findall(r"(int32_t|int64_t|float|void\*)\s+([\w,\s]+);", body)
              for n in ns.split(",")]
    assert fields == list(cls._fields_)


def test_constants_match_the_header():
    for name in ("GLR_MIX", "GLR_DECAY", "MGRIT_F16"):
        assert int(re.search(name + r"\s*=\s*(\d+)", HEADER).group(1)) == getattr(mg, name)
    for name in ("LOGPROBS_MAX_K", "DISTILL_MAX_K"):
        assert int(re.search(name + r"\s+(\d+)", HEADER).group(1)) == getattr(mg, name)


def size(name, cfg):
    n = ctypes.c_size_t(0)
    return getattr(ops._lib(), name)(ctypes.byref(cfg), ctypes.byref(n)), n.value


def seq(data=P, t=8, b=8):
    return ctypes.byref(ops.GlrSeq(data, t, b))


def forward(cfg, gate=None, value=None, h=None, h0=P, saved=P, saved_n=1 << 40, ws=P, ws_n=1 << 40):
    T, B, H = cfg.T, cfg.B, cfg.H
    dense = lambda: seq(P, B * H, H)  # noqa: E731
    return ops._lib().glr_forward(ctypes.byref(cfg), gate or dense(), value or dense(), h0, None, h or dense(), P, saved,
                                  saved_n, ws, ws_n, None)


def test_recurrence_refusals():
    L = ops._lib()
    big = mg.GlrCfg(1000, 2, 130)
    for cfg, code in ((mg.GlrCfg(0, 2, 8), SIZE), (mg.GlrCfg(8, 0, 8), SIZE), (mg.GlrCfg(8, 2, 0), SIZE),
                      (mg.GlrCfg(1 << 20, 1 << 11, 1), SIZE), (mg.GlrCfg(8, 1 << 16, 1 << 15), SIZE),
                      (mg.GlrCfg(8, 2, 8, 2), ENUM), (mg.GlrCfg(8, 2, 8, 0, 2), ENUM), (mg.GlrCfg(8, 2, 8, 0, 5), ENUM)):
        assert size("glr_workspace_bytes", cfg)[0] == code and size("glr_saved_bytes", cfg)[0] == code
        assert forward(cfg) == code
    assert L.glr_workspace_bytes(None, None) == NULL
    assert L.glr_workspace_bytes(ctypes.byref(big), None) == NULL
    # one tile: no workspace; several: words for each; a state per tile
    assert size("glr_workspace_bytes", mg.GlrCfg(16, 2, 130)) == (0, 0)
    assert size("glr_saved_bytes", mg.GlrCfg(16, 2, 130)) == (0, 4 * 2 * 130)
    rc, saved = size("glr_saved_bytes", big)
    assert rc == 0 and saved % (4 * 2 * 130) == 0 and saved > 4 * 2 * 130
    rc, n = size("glr_workspace_bytes", big)
    assert rc == 0 and n >= 2 * saved
    assert forward(big, gate=seq(0, 260, 130)) == NULL
    assert forward(big, gate=seq(P + 2, 260, 130)) == ALIGN
    assert forward(big, gate=seq(P, -260, 130)) == SIZE
    assert forward(big, gate=seq(P, 1 << 61, 130)) == SIZE
    assert forward(big, h0=P + 2) == ALIGN
    assert forward(big, ws_n=n - 1) == WORKSPACE
    assert forward(big, ws=None) == NULL
    assert forward(big, ws=P + 8) == ALIGN
    assert forward(big, saved_n=saved - 1) == WORKSPACE
    assert forward(big, saved=P + 8) == ALIGN
    # outputs that would overlap themselves
    for t, b in ((129, 1 << 20), (0, 130), (130, 130 * 999), (130, 0), (259, 130), (1 << 20, 129)):
        assert forward(big, h=seq(P, t, b)) == SIZE, (t, b)
    # backward: what it needs besides
    dense = lambda: seq(P, 260, 130)  # noqa: E731

    def backward(saved=P, saved_n=1 << 40, dh=None, dgate=None, ws_n=1 << 40):
        return L.glr_backward(ctypes.byref(big), dense(), dense(), None, saved, saved_n, dh or dense(), None,
                              dgate or dense(), dense(), None, P, ws_n, None)

    assert backward(saved=None) == NULL
    assert backward(saved=P + 4) == ALIGN
    assert backward(saved_n=saved - 1) == WORKSPACE
    assert backward(dh=seq(None)) == NULL
    assert backward(dgate=seq(P, 0, 0)) == SIZE
    assert backward(ws_n=n - 1) == WORKSPACE


def test_step_refusals():
    L = ops._lib()

    def step(cfg=mg.GlrCfg(1, 4, 8), slots=P, n=4, state=P, out=P, h=None):
        return L.glr_step(ctypes.byref(cfg), seq(), seq(), slots, n, None, state, out, h or seq(), None)

    assert step(cfg=mg.GlrCfg(2, 4, 8)) == SIZE
    assert step(n=0) == SIZE
    assert step(slots=None, n=3) == SIZE
    assert step(state=None) == NULL and step(out=None) == NULL
    assert step(state=P + 2) == ALIGN and step(slots=P + 2) == ALIGN
    assert step(h=seq(P, 0, 7)) == SIZE


def logits_cfg(N=4, V=100, K=5, dtype=0, t=1.0, ld=None, ld_grad=None):
    c = mg.LogitsCfg(N, V, K, dtype, t)
    c.ld, c.ld_grad = ld or V, ld_grad or V
    return c


def test_logits_refusals():
    L = ops._lib()

    def logprobs(cfg=None, x=P, tokens=P, logp=P, top=P, ids=P, ws=P, n=1 << 40):
        return L.token_logprobs(ctypes.byref(cfg or logits_cfg()), x, tokens, logp, P, top, ids, ws, n, None)

    def distill(cfg=None, x=P, ids=P, teacher=P, loss=P, grad=P * 2, ws=P, n=1 << 40):
        return L.distill_topk(ctypes.byref(cfg or logits_cfg()), x, ids, teacher, None, loss, None, grad, ws, n, None)

    inf, nan = float("inf"), float("nan")
    for cfg, code in ((logits_cfg(N=0), SIZE), (logits_cfg(V=0, ld=1), SIZE), (logits_cfg(V=(1 << 20) + 1), SIZE),
                      (logits_cfg(N=1 << 27), SIZE), (logits_cfg(K=-1), SIZE), (logits_cfg(ld=99), SIZE),
                      (logits_cfg(t=0.0), SIZE), (logits_cfg(t=-1.0), SIZE), (logits_cfg(t=inf), SIZE),
                      (logits_cfg(t=nan), SIZE), (logits_cfg(t=1e-44), SIZE), (logits_cfg(dtype=3), ENUM)):
        assert size("logits_workspace_bytes", cfg)[0] == code
        assert logprobs(cfg) == code and distill(cfg) == code
    assert logprobs(logits_cfg(K=65)) == SIZE and logprobs(logits_cfg(V=4, K=5)) == SIZE
    assert distill(logits_cfg(K=257)) == SIZE and distill(logits_cfg(K=0)) == SIZE
    assert logprobs(x=None) == NULL and logprobs(tokens=None) == NULL and logprobs(logp=None) == NULL
    assert logprobs(top=None) == NULL and logprobs(ids=None) == NULL and logprobs(logits_cfg(K=0)) == NULL
    assert distill(ids=None) == NULL and distill(teacher=None) == NULL and distill(loss=None) == NULL
    assert logprobs(x=P + 2) == ALIGN and logprobs(tokens=P + 4) == ALIGN and distill(ids=P + 4) == ALIGN
    assert distill(logits_cfg(ld_grad=99)) == SIZE
    assert distill(logits_cfg(ld=200), grad=P) == SIZE               # in place: one row stride
    # rows that one team holds need no workspace, longer ones do
    assert size("logits_workspace_bytes", logits_cfg(V=30000)) == (0, 0)
    long = logits_cfg(V=40000)
    rc, n = size("logits_workspace_bytes", long)
    assert rc == 0 and n > 0
    assert logprobs(long, n=n - 1) == WORKSPACE and distill(long, n=n - 1) == WORKSPACE
    assert logprobs(long, ws=None) == NULL and logprobs(long, ws=P + 8) == ALIGN

    def back(cfg=None, stats=P, grad=P * 2):
        return L.distill_topk_backward(ctypes.byref(cfg or logits_cfg()), P, P, P, stats, None, grad, None)

    assert back(stats=None) == NULL and back(grad=None) == NULL and back(logits_cfg(t=0.0)) == SIZE


def test_q8_refusals():
    L = ops._lib()

    def cfg(M=4, N=8, K=100, dtype=0, ldx=None, ldy=None):
        c = mg.Q8Cfg(M, N, K, dtype)
        c.ldx, c.ldy = ldx or K, ldy or N
        return c

    def linear(c=None, x=P, w=P, scale=P, y=P, ws=P, n=1 << 40):
        return L.q8_linear(ctypes.byref(c or cfg()), x, w, scale, None, y, ws, n, None)

    for c, code in ((cfg(M=0), SIZE), (cfg(N=0, ldy=1), SIZE), (cfg(K=0, ldx=1), SIZE), (cfg(K=131073), SIZE),
                    (cfg(ldx=99), SIZE), (cfg(ldy=7), SIZE), (cfg(dtype=2), ENUM), (cfg(M=1 << 30, N=1 << 30), SIZE)):
        assert size("q8_workspace_bytes", c)[0] == code and linear(c) == code
    rc, n = size("q8_workspace_bytes", cfg())
    assert rc == 0 and n >= 4 * (128 + 4)
    assert linear(n=n - 1) == WORKSPACE and linear(ws=None) == NULL and linear(ws=P + 4) == ALIGN
    assert linear(x=None) == NULL and linear(w=None) == NULL and linear(scale=None) == NULL and linear(y=None) == NULL
    assert linear(w=P + 8) == ALIGN and linear(x=P + 1) == ALIGN
    assert L.q8_quantize(ctypes.byref(cfg()), None, P, P, None) == NULL
    assert L.q8_quantize(ctypes.byref(cfg()), P, P + 8, P, None) == ALIGN
    assert mg.q8_row_bytes(1) == 128 and mg.q8_row_bytes(128) == 128 and mg.q8_row_bytes(129) == 256


def test_binding_refuses_tensors_that_do_not_fit():
    z = torch.zeros
    cfg, ws = mg.GlrCfg(4, 2, 8), z(0, dtype=torch.uint8)
    s = z(4, 2, 8)
    good = dict(gate=s, value=s, h0=z(2, 8), reset=z(4, 2, dtype=torch.uint8), h=s, h_last=z(2, 8), saved=None, workspace=ws)
    for over in (dict(gate=z(4, 2, 9)), dict(h0=z(8, 2)), dict(reset=z(2, 4, dtype=torch.uint8)), dict(h=z(2, 4, 8)),
                 dict(h_last=z(8))):
        with pytest.raises(ValueError):
            mg.glr_forward(cfg, **dict(good, **over))
    with pytest.raises(TypeError):                   # right sizes, but not device memory
        mg.glr_forward(cfg, **good)
    with pytest.raises(ValueError):
        mg.glr_step(mg.GlrCfg(1, 2, 8), z(1, 2, 8), z(2, 8), None, None, z(2, 8), z(2, 8), z(2, 8))
    with pytest.raises(ValueError):
        mg.glr_step(mg.GlrCfg(1, 2, 8), z(2, 8), z(2, 8), None, None, z(2, 8), z(3, 8), z(2, 8))
    lc, ids = mg.LogitsCfg(3, 10, 2), z(3, 2, dtype=torch.int64)
    with pytest.raises(ValueError):
        mg.token_logprobs(lc, z(3, 10), z(4, dtype=torch.int64), z(3), z(3), z(3, 2), ids, ws)
    with pytest.raises(ValueError):
        mg.distill_topk(lc, z(3, 10), ids, z(3, 2), z(3), z(3), z(3), z(3, 10), ws)
    with pytest.raises(ValueError):
        mg.distill_topk_backward(lc, z(3, 10), ids, z(3, 2), z(3, 2), z(3), z(3, 11))
    qc = mg.Q8Cfg(3, 5, 10)
    with pytest.raises(ValueError):                  # rows of weights are padded to 128 bytes
        mg.q8_linear(qc, z(3, 10), z(5, 10, dtype=torch.int8), z(5), None, z(3, 5), ws)
    with pytest.raises(ValueError):
        mg.q8_quantize(qc, z(3, 10), z(3, 10, dtype=torch.int8), z(3))
    with pytest.raises(mg.MgritGruError):
        mg.glr_workspace_bytes(mg.GlrCfg(0, 1, 1))
