"""Idle rows of a served batch: a slot outside the pool touches no state, whether prompts are read or tokens taken."""
import pytest
import torch

from paper_2203_04738_amd.student import Served
from test_gpu_student import DEV, small

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("idle", [-1, -7, 6, 1 << 30])
def test_idle_rows_touch_no_state(idle):
    student, x, _, _ = small(seed=5)                         # three sequences
    served = Served(student, slots=6)
    for s in served.state:
        s.copy_(torch.randn_like(s))
    before = [s.clone() for s in served.state]
    slots = torch.tensor([4, idle, 0], dtype=torch.int32, device=DEV)
    logits = served.read(x, slots)
    after = [s.clone() for s in served.state]
    for a, b in zip(after, before):
        assert torch.equal(a[[1, 2, 3, 5]], b[[1, 2, 3, 5]]) and not torch.equal(a[[4, 0]], b[[4, 0]])
    served.next(x[0], slots)
    for s, a in zip(served.state, after):
        assert torch.equal(s[[1, 2, 3, 5]], a[[1, 2, 3, 5]]) and not torch.equal(s[[4, 0]], a[[4, 0]])
    # the others are what they are without an idle row beside them, states and logits
    alone = Served(student, slots=6)
    ref = alone.read(x, torch.tensor([4, 3, 0], dtype=torch.int32, device=DEV))
    assert torch.equal(logits[[0, 2]], ref[[0, 2]])
    for a, b in zip(after, alone.state):
        assert torch.equal(a[[4, 0]], b[[4, 0]])


def test_all_rows_idle():
    student, x, _, _ = small(seed=6)
    served = Served(student, slots=2)
    slots = torch.full((3,), -1, dtype=torch.int32, device=DEV)
    served.read(x, slots)
    served.next(x[0], slots)
    assert all(torch.all(s == 0) for s in served.state)
