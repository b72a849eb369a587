"""Several answers of a search agent to one question, on one GPU: a small decoder with random weights takes the prompt in at once, asks the exact search for passages, takes them in at once, and then
tries several continuations, which share all that came before.  An example of the library's operators for many tokens together, as a serving engine calls them:

    ann_rotate_append -> ann_chunk_attention      in every layer, for the tokens of a prompt or of passages
    ann_flat_search_typed                         between the two
    ann_rotate_append -> ann_shared_attention     in every layer, for one new token of every answer, whose leading slots are the same pages

    python -m paper_2505_12065_amd.agent_rollouts [--answers 8] [--steps 60]

The paper's agent (Section 3.1, Algorithm 1) has a trained model, an encoder and text in these places; products of matrices are torch's.
"""
from __future__ import annotations

import argparse
from typing import List

import torch

from . import binding as ann


class Rollouts:
    """A context that grows by whole passages, and `answers` continuations of it."""

    def __init__(self, answers: int, *, layers: int = 2, q_heads: int = 8, heads: int = 2, d: int = 64, vocab: int = 1000, page: int = 16, limit: int = 2048, own: int = 256,
                 trained: int = 512, passages: int = 2000, passage_tokens: int = 100, dtype=torch.bfloat16, seed: int = 0, device: str = "cuda:0"):
        g = torch.Generator(device).manual_seed(seed)
        self.answers, self.q_heads, self.heads, self.d, self.page, self.limit, self.dtype, self.device = answers, q_heads, heads, d, page, limit, dtype, device
        width = q_heads * d

        def matrix(*shape):
            return (torch.randn(*shape, generator=g, device=device) * shape[-2] ** -0.5).to(dtype)
        self.embed = matrix(1, vocab, width)[0] * vocab ** 0.5
        self.layers = [(matrix(width, (q_heads + 2 * heads) * d), matrix(width, width)) for _ in range(layers)]
        self.head = matrix(width, vocab)
        # contexts go beyond what such a model would have been trained with
        self.frequencies, self.amplitude = ann.ann_rotation_frequencies(d, scaling="ramp", factor=max(1.0, (limit + own) / trained), original=trained, device=device)
        self.corpus = torch.nn.functional.normalize(torch.randn(passages, width, generator=g, device=device), dim=1).to(torch.float16)
        self.passage_tokens = torch.randint(0, vocab, (passages, passage_tokens), generator=g, device=device)
        # pages of the context, then those of each answer's own tokens
        common, each = (limit + page - 1) // page, (own + page - 1) // page + 1
        pages = common + answers * each
        self.k = [torch.zeros(pages, heads, page, d, dtype=dtype, device=device) for _ in range(layers)]
        self.v = [torch.zeros_like(k) for k in self.k]
        self.context = self._ints([list(range(common))])
        self.own_pages = [list(range(common + b * each, common + (b + 1) * each)) for b in range(answers)]
        self.length, self.said, self.begun = 0, 0, False  # slots of the context; tokens of every answer; whether these share it as it is

    def _ints(self, x) -> torch.Tensor:
        return torch.tensor(x, dtype=torch.int32, device=self.device)

    def _forward(self, tokens: torch.Tensor, starts, lengths, table, attend) -> torch.Tensor:
        x = self.embed[tokens]
        for (w_qkv, w_out), k, v in zip(self.layers, self.k, self.v):
            y = torch.nn.functional.layer_norm(x.float(), x.shape[-1:]).to(self.dtype)
            qkv = (y @ w_qkv).view(len(tokens), self.q_heads + 2 * self.heads, self.d)
            q = ann.ann_rotate_append(qkv, starts, lengths, table, self.frequencies, k, v, amplitude=self.amplitude)
            x = x + attend(q, k, v).flatten(1) @ w_out
        return torch.nn.functional.layer_norm(x.float(), x.shape[-1:])

    def take(self, tokens: torch.Tensor) -> torch.Tensor:
        """Tokens that the context grows by; the hidden state of the last."""
        if self.begun:
            raise ValueError("the answers have begun")
        if self.length + len(tokens) > self.limit:
            raise ValueError(f"a context of more than {self.limit} tokens")
        self.length += len(tokens)
        starts, lengths = self._ints([0, len(tokens)]), self._ints([self.length])
        self.hidden = self._forward(tokens, starts, lengths, self.context, lambda q, k, v: ann.ann_chunk_attention(
            q, k, v, self.context, lengths, starts, max_length=self.length)[0])[-1:]
        return self.hidden

    def search(self, passages: int) -> List[int]:
        """Passages for the last hidden state, which are taken in."""
        query = torch.nn.functional.normalize(self.hidden, dim=1).to(torch.float16)
        ids, _ = ann.ann_flat_search_typed(self.corpus, query, passages)
        self.take(self.passage_tokens[ids[0].long()].flatten())
        return ids[0].tolist()

    def begin(self) -> None:
        """Answers begin: whole pages of the context are everyone's, and its last tokens, where they fill no page, are copied to each answer's first one."""
        self.begun = True
        whole, rest = self.length // self.page, self.length % self.page
        self.common = whole * self.page
        table = torch.tensor([list(range(whole)) + own for own in self.own_pages], dtype=torch.int32)
        if rest:
            for cache in self.k + self.v:
                for own in self.own_pages:
                    cache[own[0], :, :rest] = cache[whole, :, :rest]
        self.table = table.to(self.device)
        self.starts, self.groups, self.shared = self._ints(list(range(self.answers + 1))), self._ints([0, self.answers]), self._ints([self.common])

    def step(self, tokens: torch.Tensor) -> torch.Tensor:
        """One new token of every answer: logits [answers, vocabulary]."""
        n = self.length + self.said + 1
        if n > self.table.shape[1] * self.page:
            raise ValueError("the answers' pages are full")
        self.said += 1
        lengths = torch.full((self.answers,), n, dtype=torch.int32, device=self.device)
        hidden = self._forward(tokens, self.starts, lengths, self.table, lambda q, k, v: ann.ann_shared_attention(
            q, k, v, self.table, lengths, self.groups, self.shared, max_shared=self.common, max_own=n - self.common)[0])
        return hidden.to(self.dtype) @ self.head

    def run(self, prompt: List[int], searches: int, steps: int, *, passages: int = 2, seed: int = 0):
        """(passages that were found, tokens [answers, steps]) for a prompt; the answers are sampled."""
        g = torch.Generator(self.device).manual_seed(seed)
        self.take(torch.tensor(prompt, device=self.device))
        found = [i for _ in range(searches) for i in self.search(passages)]
        self.begin()
        logits = (self.hidden.to(self.dtype) @ self.head).expand(self.answers, -1)
        said = []
        for _ in range(steps):
            said.append(torch.multinomial(torch.softmax(logits.float(), 1), 1, generator=g)[:, 0])
            logits = self.step(said[-1])
        return found, torch.stack(said, 1)


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--answers", type=int, default=8)
    parser.add_argument("--steps", type=int, default=60)
    args = parser.parse_args()
    rollouts = Rollouts(args.answers, own=max(16, args.steps))
    found, said = rollouts.run(list(range(40)), 2, args.steps)
    print(f"context of {rollouts.length} tokens with passages {found}; slots in common {rollouts.common}")
    for b, tokens in enumerate(said.tolist()):
        print(f"answer {b}: {tokens[:12]} ... ({len(tokens)} tokens)")


if __name__ == "__main__":
    main()
