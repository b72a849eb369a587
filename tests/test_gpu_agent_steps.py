"""The example that runs the operators together: its logits against a plain decoder in 64 bits that sees the same slots, and what it keeps."""
import pytest
import torch

from paper_2505_12065_amd import agent_steps

pytestmark = pytest.mark.gpu
PROMPT = list(range(3, 3 + 37))                           # two whole pages and some
QUESTIONS = [[50, 7], [600, 8], [7, 900], [333, 3]]


def plain_logits(a, tokens, q_heads, heads, d):
    """Logits of the last of `tokens`, all in 64 bits, every token seeing all before it."""
    x = a.embed.double()[torch.tensor(tokens, device=a.device)]
    n = len(tokens)
    turn = a.cos_sin[:n].double()
    c, s = turn[:, :d // 2], turn[:, d // 2:]

    def rotated(y):
        y = y / (y.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()
        u, v = y[..., :d // 2], y[..., d // 2:]
        return torch.cat([u * c[:, None] - v * s[:, None], v * c[:, None] + u * s[:, None]], -1)
    ahead = torch.ones(n, n, dtype=torch.bool, device=a.device).triu(1)
    for w_qkv, _, _, w_out in a.layers:
        y = torch.nn.functional.layer_norm(x, x.shape[-1:])
        qkv = (y @ w_qkv.double()).view(n, q_heads + 2 * heads, d)
        q, k, v = rotated(qkv[:, :q_heads]), rotated(qkv[:, q_heads:q_heads + heads]), qkv[:, q_heads + heads:]
        k, v = k.repeat_interleave(q_heads // heads, 1), v.repeat_interleave(q_heads // heads, 1)
        score = torch.einsum("ihd,jhd->hij", q, k) * d ** -0.5
        p = torch.softmax(score.masked_fill(ahead, -torch.inf), -1)
        x = x + torch.einsum("hij,jhd->ihd", p, v).flatten(1) @ w_out.double()
    return torch.nn.functional.layer_norm(x[-1:], x.shape[-1:]) @ a.head.double()


def test_logits_of_a_shared_prompt_and_beyond():
    """fp32 throughout: what differs is rounding, some hundred times 2^-24 of sums of a few hundred terms of order 1 in two layers; a wrong slot,
    rotation or head is of order 1."""
    a = agent_steps.Agents(PROMPT, QUESTIONS[:3], dtype=torch.float32, seed=3, limit=128)
    for extra in ([5, 9, 700], [44, 9, 1], [8, 8, 8]):
        a.logits, a.hidden = a.step(extra)
    for b in range(3):
        tokens = a.tokens[b, :a.told[b]].tolist()
        assert tokens[:len(PROMPT) + 2] == PROMPT + QUESTIONS[b] and len(tokens) == len(PROMPT) + 5
        torch.testing.assert_close(a.logits[b:b + 1].double(), plain_logits(a, tokens, 8, 2, 64), rtol=0, atol=1e-3)
    assert a.pages[0][:2] == a.pages[1][:2] == a.pages[2][:2] and len({p[2] for p in a.pages}) == 3


def test_run_keeps_to_its_limits():
    a = agent_steps.Agents(PROMPT, QUESTIONS, limit=96, budget=64, seed=1)
    said, given = a.run(120)
    assert all(len(s) == 120 for s in said) and all(agent_steps.PAD not in s for s in said)
    assert all(0 <= i < 2000 for g in given for i in g)
    for b in range(4):
        assert a.position[b] == a.told[b] == len(PROMPT) + 122 and a.slots_used[b] <= 96
        assert a.asked[b] <= 2 and len(given[b]) == 2 * a.asked[b]
    assert sum(a.asked) > 0
    held = [p for pages in a.pages for p in pages]
    assert sorted(held + a.free) == sorted(range(len(a.used))) and len(set(held)) == len(held)     # nothing shared is left, nothing lost
    # every layer's weights sum up to what was given out since: one for each query head and step (what was cut is gone)
    for m in a.mass:
        assert (m >= 0).all() and (m.sum(-1) <= 4 * (len(PROMPT) + 122) * (1 + 1e-3)).all()
    b = agent_steps.Agents(PROMPT, QUESTIONS, limit=96, budget=64, seed=1)
    assert b.run(120) == (said, given)
