"""How a student over tokens samples, without a GPU: the numbers at both ends of [0, 1)."""
import pytest
import torch

from paper_2203_04738_amd import token_student
from paper_2203_04738_amd.ops import LogitsCfg

LAST = 1.0 - 2.0 ** -24                                        # the largest float below 1


def act(logits, uniform, temperature=1.0):
    s = object.__new__(token_student.TokenStudent)
    N, s.V = logits.shape
    s.rows = LogitsCfg(N, s.V, 0, temperature=temperature)
    s.logits = lambda tokens, reset=None: logits
    s.log_probs = lambda out, actions: torch.log_softmax(out / temperature, 1).gather(1, actions[:, None])[:, 0]
    return s.act(None, uniform)


@pytest.mark.parametrize("V,first,last", [(5, 1, 3), (5, 0, 4), (5, 2, 2), (1, 0, 0), (2, 1, 1), (2, 0, 0), (1000, 17, 900)])
@pytest.mark.parametrize("number", [0.0, 2.0 ** -149, 0.25, 0.999, LAST])
def test_only_tokens_with_a_probability_are_sampled(V, first, last, number):
    g = torch.Generator().manual_seed(V)
    logits = torch.randn(200, V, generator=g)
    logits[:, :first] = logits[:, last + 1:] = -float("inf")
    actions, logp = act(logits, torch.full((200,), number))
    assert ((actions >= first) & (actions <= last)).all() and torch.isfinite(logp).all()
    if number == 0.0:
        assert (actions == first).all()


def test_a_number_picks_the_token_whose_share_it_falls_into():
    p = torch.tensor([0.0, 0.25, 0.0, 0.5, 0.25, 0.0])
    numbers = torch.tensor([0.0, 0.2, 0.26, 0.5, 0.7, 0.76, 0.9, LAST])   # (none at a border)
    actions, _ = act(torch.log(p).expand(8, 6).contiguous(), numbers)
    assert actions.tolist() == [1, 1, 3, 3, 3, 4, 4, 4]
