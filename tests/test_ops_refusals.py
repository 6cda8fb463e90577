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
