"""What the example of several answers to one question refuses, on the CPU: nothing is enqueued."""
import pytest
import torch

from paper_2505_12065_amd.agent_rollouts import Rollouts


def small():
    return Rollouts(2, layers=1, q_heads=2, heads=1, d=16, vocab=10, page=16, limit=64, own=16, passages=4, passage_tokens=3, dtype=torch.float32, device="cpu")


def test_the_context_does_not_grow_once_answers_have_begun():
    """... whose page tables and copied rows are those of the context as it was."""
    r = small()
    r.length = 20                                         # (as if 20 tokens had been taken in)
    r.begin()
    with pytest.raises(ValueError, match="begun"):
        r.take(torch.tensor([1, 2]))
    assert r.length == 20


def test_a_step_that_is_refused_leaves_the_answers_as_they_were():
    r = small()
    r.length = 20
    r.begin()
    room = r.table.shape[1] * r.page - r.length
    r.said = room
    for _ in range(2):
        with pytest.raises(ValueError, match="full"):
            r.step(torch.tensor([1, 2]))
    assert r.said == room
