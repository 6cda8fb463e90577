"""Calls whose launches would take 2^32 threads or more, without a GPU: refused as too large before anything is launched, and those
just below launched whole."""
import os
import subprocess
import sys

import pytest

import test_ops_launches as launches

ROOT = launches.ROOT
SIZE = -2


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    """The runtime of test_ops_launches, which prints threads instead of workgroups."""
    src = open(os.path.join(ROOT, "tests", "fake_hip_runtime.cpp")).read()
    for old, new in (("int hipLaunchKernel(const void* f, Dim g, Dim, void**", "int hipLaunchKernel(const void* f, Dim g, Dim b, void**"),
                     ('"%s %u %s\\n"', '"%s %llu %s\\n"'), ("g.x * g.y * g.z,", "1ull * g.x * g.y * g.z * b.x * b.y * b.z,")):
        assert src.count(old) == 1, old
        src = src.replace(old, new)
    tmp = tmp_path_factory.mktemp("hip")
    (tmp / "fake.cpp").write_text(src)
    out = str(tmp / "libfake_hip.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-o", out, str(tmp / "fake.cpp")])
    return out


M = 1 << 20


@pytest.mark.parametrize("entry,fits,more", [
    ("glr_forward", (2, 8 * M - 1, 2), (2, 8 * M, 2)),       # a tile a row: 2^23 workgroups of 512
    ("glr_backward", (2, 8 * M - 1, 2), (2, 8 * M, 2)),
    ("glr_forward", (512, 2 * M - 1, 40), (512, 2 * M, 40)),  # (the adjoint's tiles are half as long)
    ("glr_backward", (512, 2 * M - 1, 40), (512, 2 * M, 40)),
    ("distill_topk", (4 * M - 1, 20000, 4), (4 * M, 20000, 4)),
    ("distill_topk", (2 * M - 1, 50000, 4), (2 * M, 50000, 4)),
    ("distill_topk_backward", (2 * M - 1, 50000, 4), (2 * M, 50000, 4)),
    ("distill_topk_backward", (16 * M - 1, 5000, 4), (16 * M, 5000, 4)),
    ("token_logprobs", (16 * M - 1, 5000, 4), (16 * M, 5000, 4)),
    ("token_logprobs", (16 * M - 1, 20000, 4), (16 * M, 20000, 4)),
    ("token_logprobs", (8 * M - 1, 50000, 4), (8 * M, 50000, 4)),
    ("q8_linear", (16 * M - 1, 16, 2500), (16 * M, 16, 2500)),
    ("q8_linear", (4 * M - 1, 16, 9000), (4 * M, 16, 9000)),
    ("q8_linear", (4 * M - 1, 16, 60000), (4 * M, 16, 60000)),
    ("q8_linear", (2, 256 * M - 16, 16), (2, 256 * M, 16)),
    ("q8_linear", (2, 256 * M - 16, 16), (1, 2 ** 31 - 1, 16))])
def test_launches_of_less_than_2_to_the_32_threads(runtime, entry, fits, more):
    rc, got = launches.call(runtime, entry, *fits)
    assert rc == 0 and got and all(0 < n < 2 ** 32 for n, _ in got), (rc, got)
    assert launches.call(runtime, entry, *more) == (SIZE, [])


def test_a_step_has_limits_of_its_own(runtime):
    # no tiles: two channels of a row are a thread
    rc, got = launches.call(runtime, "glr_step", 1, 16 * M, 2)
    assert rc == 0 and [n for n, _ in got] == [16 * M]
