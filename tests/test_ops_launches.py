"""What the operators' entry points launch, and what they make of a launch that fails, without a GPU (fake_hip_runtime.cpp)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CALL = """
import ctypes, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
from ctypes import byref
from paper_2203_04738_amd import binding, ops
L, entry, n = ops._prototypes(binding.lib()), sys.argv[2], [int(a) for a in sys.argv[3:]]
A, big = [(i + 1) << 40 for i in range(12)], 1 << 50
if entry.startswith("glr"):
    T, B, H = n[:3]
    c = ops.GlrCfg(*n)
    s = [byref(ops.GlrSeq(a, B * H, H)) for a in A]
if entry == "glr_forward":
    rc = L.glr_forward(byref(c), s[0], s[1], A[2], None, s[3], A[4], A[5], big, A[6], big, None)
elif entry == "glr_backward":
    rc = L.glr_backward(byref(c), s[0], s[1], None, A[2], big, s[3], None, s[4], s[5], A[6], A[7], big, None)
elif entry == "glr_step":
    rc = L.glr_step(byref(c), s[0], s[1], A[2], 9, None, A[3], A[4], s[5], None)
elif entry == "token_logprobs":
    rc = L.token_logprobs(byref(ops.LogitsCfg(*n)), A[0], A[1], A[2], A[3], A[4], A[5], A[6], big, None)
elif entry == "distill_topk":
    rc = L.distill_topk(byref(ops.LogitsCfg(*n)), A[0], A[1], A[2], A[3], A[4], None, A[5], A[6], big, None)
elif entry == "distill_topk_backward":
    rc = L.distill_topk_backward(byref(ops.LogitsCfg(*n)), A[0], A[1], A[2], A[3], A[4], A[5], None)
elif entry == "q8_linear":
    rc = L.q8_linear(byref(ops.Q8Cfg(*n)), A[0], A[1], A[2], A[3], A[4], A[5], big, None)
print("returned", rc)
"""


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("hip") / "libfake_hip.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-o", out,
                           os.path.join(ROOT, "tests", "fake_hip_runtime.cpp")])
    return out


def call(runtime, entry, *sizes, **env):
    """(what the call returned, [(workgroups, kernel)])"""
    r = subprocess.run([sys.executable, "-c", CALL, runtime, entry, *(str(v) for v in sizes)], cwd=ROOT,
                       env=dict(os.environ, **env), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    lines = [line.split(" ", 2) for line in r.stdout.splitlines()]
    (rc,) = (int(f[1]) for f in lines if f[0] == "returned")
    return rc, [(int(f[1]), f[2]) for f in lines if f[0] in ("launched", "failed")]


@pytest.mark.parametrize("entry,sizes,kernels", [
    ("glr_forward", (100, 2, 130), ["glr_forward_kernel<float, true, 0, 64>"]),
    ("glr_forward", (1000, 2, 130, 1, 1), ["glr_clear_kernel", "glr_forward_kernel<mg::Bf16, true, 1, 64>"]),
    ("glr_forward", (1000, 2, 33), ["glr_clear_kernel", "glr_forward_kernel<float, false, 0, 0>"]),
    ("glr_backward", (1000, 2, 130), ["glr_clear_kernel", "glr_backward_kernel<float, true, 0, 32>"]),
    ("glr_step", (1, 4, 8), ["glr_step_kernel<float, true, 0>"]),
    ("token_logprobs", (100, 51, 5), ["logprobs_kernel<float, 1, false>"]),
    ("token_logprobs", (8, 8192, 5), ["logprobs_kernel<float, 4, false>"]),
    ("token_logprobs", (8, 32768, 5, 1), ["logprobs_kernel<mg::Bf16, 16, false>"]),
    ("token_logprobs", (2048, 32768, 5, 1), ["logprobs_stream_kernel<mg::Bf16, false>"]),
    ("token_logprobs", (8, 100000, 5), ["logprobs_kernel<float, 16, true>", "logprobs_join_kernel<float>"]),
    ("token_logprobs", (2048, 100000, 5), ["logprobs_stream_kernel<float, true>", "logprobs_join_kernel<float>"]),
    ("distill_topk", (64, 32768, 8, 1), ["distill_kernel<mg::Bf16, 16>"]),
    ("distill_topk", (64, 50000, 8), ["distill_segment_kernel<float>", "distill_join_kernel<float>",
                                      "distill_grad_kernel<float, 16>"]),
    ("distill_topk_backward", (64, 500, 8), ["distill_grad_kernel<float, 1>"]),
    ("q8_linear", (8, 2048, 2048, 1), ["q8_fused_kernel<mg::Bf16>"]),
    ("q8_linear", (16, 2048, 8192, 1), ["q8_quantize_kernel", "q8_few_kernel<mg::Bf16, 1>"]),
    ("q8_linear", (64, 2048, 2048), ["q8_quantize_kernel", "q8_few_kernel<float, 4>"]),
    ("q8_linear", (65, 2048, 2048), ["q8_quantize_kernel", "q8_tile_kernel<float, 64, 64>"]),
    ("q8_linear", (8000, 2040, 200), ["q8_quantize_kernel", "q8_tile_kernel<float, 256, 256>"]),
    ("q8_linear", (2048, 2048, 2048, 1), ["q8_quantize_kernel<mg::Bf16, 1, 4>", "q8_tile_kernel<mg::Bf16, 128, 128>"]),
    ("q8_linear", (32768, 2048, 2048, 1), ["q8_quantize_kernel", "q8_tile_kernel<mg::Bf16, 256, 256>"]),
    ("q8_linear", (65, 16, 131072, 4), ["q8_quantize_long_kernel<mg::F16>", "q8_tile_kernel<mg::F16, 64, 64>"])])
def test_kernels_of_a_call_and_launches_that_fail(runtime, entry, sizes, kernels):
    rc, got = call(runtime, entry, *sizes)
    names = [name.replace("void mg::", "mg::") for _, name in got]
    assert rc == 0 and len(names) == len(kernels)
    assert all("mg::" + k in n for k, n in zip(kernels, names)), names
    assert all(0 < groups < 2 ** 31 for groups, _ in got)
    for k in kernels:                                            # a failing launch ends the call and is reported
        rc, got = call(runtime, entry, *sizes, FAKE_HIP_FAIL=k.split("<")[0])
        assert rc == -7 and len(got) <= len(kernels)
