"""The example of several answers to one question, against the same model without a cache."""
import math

import pytest
import torch

from paper_2505_12065_amd.agent_rollouts import Rollouts

pytestmark = pytest.mark.gpu


def plain(r, tokens):
    """Hidden states of a sequence in 64 bits, from r's weights."""
    x = r.embed[tokens].double().cpu()
    n, d, heads, G = len(tokens), r.d, r.heads, r.q_heads // r.heads
    angle = torch.arange(n, dtype=torch.float64)[:, None] * r.frequencies.cpu()
    c, s = angle.cos()[:, None] * r.amplitude, angle.sin()[:, None] * r.amplitude

    def turn(y):
        a, b = y[..., :d // 2], y[..., d // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)
    for w_qkv, w_out in r.layers:
        y = torch.nn.functional.layer_norm(x, x.shape[-1:])
        qkv = (y @ w_qkv.double().cpu()).view(n, r.q_heads + 2 * heads, d)
        q, k, v = turn(qkv[:, :r.q_heads]), turn(qkv[:, r.q_heads:r.q_heads + heads]), qkv[:, r.q_heads + heads:]
        score = torch.matmul(q.view(n, heads, G, d).permute(1, 2, 0, 3), k.permute(1, 2, 0)[:, None]) / math.sqrt(d)
        score.masked_fill_(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
        o = torch.matmul(torch.softmax(score, -1), v.transpose(0, 1)[:, None]).permute(2, 0, 1, 3).reshape(n, -1)
        x = x + o @ w_out.double().cpu()
    return torch.nn.functional.layer_norm(x, x.shape[-1:])


@pytest.mark.parametrize("prompt", [37, 48])
def test_answers_are_those_of_the_model(prompt):
    """fp32: a context that ends inside a page, and one that does not; answers that differ."""
    r = Rollouts(3, vocab=200, passages=300, passage_tokens=21, trained=64, dtype=torch.float32, seed=3)
    tokens = list(range(5, 5 + prompt))
    hidden = r.take(torch.tensor(tokens, device=r.device))
    # two layers of sums of up to 512 products and some hundred slots in binary32, 2^-24 each at sizes below 8: 1e-3 is some hundred times as much
    assert (hidden.cpu().double() - plain(r, torch.tensor(tokens, device=r.device))[-1:]).abs().max() < 1e-3
    found = r.search(2)
    context = tokens + r.passage_tokens[found].flatten().tolist()
    assert r.length == len(context) == prompt + 42
    r.begin()
    said = torch.randint(0, 200, (3, 20), generator=torch.Generator().manual_seed(1)).to(r.device)
    for i in range(20):
        logits = r.step(said[:, i])
    for b in range(3):
        h = plain(r, torch.tensor(context + said[b].tolist(), device=r.device))[-1]
        assert (logits[b].cpu().double() - h @ r.head.double().cpu()).abs().max() < 1e-2
    with pytest.raises(ValueError):
        r.take(torch.tensor([1], device=r.device))


def test_run_and_limits():
    r = Rollouts(4, vocab=200, passages=300, passage_tokens=20, limit=100, own=10)
    found, said = r.run(list(range(30)), 1, 5)
    assert len(found) == 2 and said.shape == (4, 5) and r.length == 70 and r.common == 64
    again = Rollouts(4, vocab=200, passages=300, passage_tokens=20, limit=100, own=10).run(list(range(30)), 1, 5)
    assert again[0] == found and torch.equal(again[1], said)
    r = Rollouts(2, limit=100)
    with pytest.raises(ValueError):
        r.take(torch.zeros(101, dtype=torch.long, device=r.device))
