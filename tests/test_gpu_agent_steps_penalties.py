"""The example's penalties: for tokens that an agent chose, not for those of its prompt, question and passages."""
from collections import Counter

import pytest

from paper_2505_12065_amd import agent_steps
from test_gpu_agent_steps import PROMPT, QUESTIONS        # (beside this file)

pytestmark = pytest.mark.gpu


def test_what_was_given_is_not_penalised_as_chosen(monkeypatch):
    rules, calls = agent_steps.ann.ann_logit_rules, []

    def spy(logits, tokens, lengths, prompt_lengths, *rest, **kw):
        calls.append((tokens.tolist(), lengths.tolist(), prompt_lengths.tolist()))
        return rules(logits, tokens, lengths, prompt_lengths, *rest, **kw)
    monkeypatch.setattr(agent_steps.ann, "ann_logit_rules", spy)
    a = agent_steps.Agents(PROMPT, QUESTIONS, limit=96, budget=64, seed=1)
    said, given = a.run(120)
    assert sum(map(len, given)) > 0
    taken = 0
    for tokens, lengths, prompts in calls:
        for b in range(4):
            n, p = lengths[b], prompts[b]
            own = len(PROMPT) + len(QUESTIONS[b])
            passages = a.passage_tokens[given[b]].flatten().tolist()[:p - own]
            assert own <= p <= n and len(passages) == p - own
            assert Counter(tokens[b][:p]) == Counter(PROMPT + QUESTIONS[b] + passages)
            assert Counter(tokens[b][:n]) == Counter(a.tokens[b, :n].tolist())
            taken = max(taken, p - own)
    assert taken >= a.passage_tokens.shape[1]             # whole passages came in
