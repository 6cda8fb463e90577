"""Host-side checks at the edges of what the operators' entry points take."""
import ctypes

import numpy as np
import pytest

import paper_2203_04738_amd as mg
from paper_2203_04738_amd import ops

SIZE = -2


@pytest.mark.parametrize("t,ok", [(4.5e-39, True), (4.2e-39, False), (3.0e-39, False), (2.0e-39, False), (3.4e38, True)])
def test_temperatures_whose_exponents_are_floats(t, ok):
    n = ctypes.c_size_t(0)
    cfg = mg.LogitsCfg(4, 100, 5, mg.MGRIT_F32, t)
    with np.errstate(over="ignore"):
        assert np.isfinite(np.float32(1.442695) / np.float32(t)) == ok
    assert ops._lib().logits_workspace_bytes(ctypes.byref(cfg), ctypes.byref(n)) == (0 if ok else SIZE)


def test_a_step_does_not_read_the_stride_of_time(tmp_path):
    """(on the host's runtime: nothing may be refused for it, nothing launched differently)"""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = str(tmp_path / "libfake_hip.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-o", out,
                           os.path.join(root, "tests", "fake_hip_runtime.cpp")])
    code = """
import ctypes, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
from ctypes import byref
from paper_2203_04738_amd import binding, ops
L = ops._prototypes(binding.lib())
for t in (0, 3, -7, 1 << 62, -1 << 63):
    s = [byref(ops.GlrSeq((i + 1) << 40, t, 8)) for i in range(3)]
    print("returned", L.glr_step(byref(ops.GlrCfg(1, 4, 8)), s[0], s[1], None, 4, None, 5 << 40, 6 << 40, s[2], None))
for i in range(3):
    s = [byref(ops.GlrSeq((i + 1) << 40, 0, 8)) for i in range(3)]
    s[i] = None
    print("returned", L.glr_step(byref(ops.GlrCfg(1, 4, 8)), s[0], s[1], None, 4, None, 5 << 40, 6 << 40, s[2], None))
"""
    r = subprocess.run([sys.executable, "-c", code, out], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    lines = r.stdout.splitlines()
    assert [int(n.split()[1]) for n in lines if n.startswith("returned")] == [0] * 5 + [-1] * 3
    assert [n for n in lines if n.startswith("launched")] == [
        "launched 1 void mg::glr_step_kernel<float, true, 0>(mg::GlrStepArgs)"] * 5


def test_a_call_leaves_the_configuration_alone():
    # (host memory: every call ends in an error, behind its look at the strides)
    import torch
    z = torch.zeros
    ws, ids = z(0, dtype=torch.uint8), z(3, 2, dtype=torch.int64)
    x, grad = z(3, 20)[:, :10], z(3, 30)[:, :10]
    lc, qc = mg.LogitsCfg(3, 10, 2), mg.Q8Cfg(3, 5, 10)
    w, y = z(5, 128, dtype=torch.int8), z(3, 9)[:, :5]
    for call in (lambda: mg.token_logprobs(lc, x, None, None, z(3), z(3, 2), ids, ws),
                 lambda: mg.distill_topk(lc, x, ids, z(3, 2), None, z(3), None, grad, ws),
                 lambda: mg.distill_topk_backward(lc, x, ids, z(3, 2), z(3, 2), None, grad),
                 lambda: mg.q8_quantize(qc, x, z(3, 128, dtype=torch.int8), z(3)),
                 lambda: mg.q8_linear(qc, x, w, z(5), None, y, ws)):
        with pytest.raises(TypeError):
            call()
        assert (lc.ld, lc.ld_grad, qc.ldx, qc.ldy) == (10, 10, 10, 5)


def test_threads_that_share_a_configuration_pass_their_own_strides(monkeypatch):
    # what reaches the library while another thread's call has just looked at its own tensors
    import torch
    x = {20: torch.zeros(3, 20)[:, :10], 50: torch.zeros(3, 50)[:, :10]}
    cfg, seen = mg.LogitsCfg(3, 10, 0), []

    def call(name, c, *args):
        if len(seen) == 0:                                   # (the other thread's call, in the middle of this one)
            seen.append(None)
            mg.token_logprobs(cfg, x[50], None, None, None, None, None, None)
        seen.append((args[0][0], c.ld))

    monkeypatch.setattr(ops, "_call", call)
    mg.token_logprobs(cfg, x[20], None, None, None, None, None, None)
    assert [(t is x[n], ld) for n, (t, ld) in zip((50, 20), seen[1:])] == [(True, 50), (True, 20)]
