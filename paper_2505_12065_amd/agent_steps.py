"""Search agents between and at their retrievals, on one GPU: a small decoder with random weights goes token by token over
paged caches, asks the exact search for passages when its output says so, takes their tokens into its context, and has the
caches cut when they grow too long.  An example of the library's operators together, as a serving engine calls them:

    ann_qk_norm_rotate -> ann_paged_attention     in every layer, for one new token of every request
    ann_logit_rules                               on the logits: no token over and over, and only what the request's state allows
    ann_flat_search_typed                         when a request's next token is SEARCH
    ann_cache_evict                               when a context would not fit its limit

    python -m paper_2505_12065_amd.agent_steps [--requests 4] [--steps 200]

The paper's agent (Section 3.1, Algorithm 1) has a trained model, an encoder and text in these places; products of matrices are torch's.
"""
from __future__ import annotations

import argparse
from typing import List

import torch

from . import binding as ann

PAD, SEARCH, ANSWER, FIRST = 0, 1, 2, 3                   # FIRST: the first ordinary token


class Agents:
    """Agents with one prompt, whose whole pages they share, as prefix caching would have it, and a question each (of one length)."""

    def __init__(self, prompt: List[int], questions: List[List[int]], *, layers: int = 2, q_heads: int = 8, heads: int = 2, d: int = 64, vocab: int = 1000,
                 page: int = 16, limit: int = 256, budget: int = 128, passages: int = 2000, passage_tokens: int = 24, searches: int = 2,
                 dtype=torch.bfloat16, seed: int = 0, device: str = "cuda:0"):
        g, requests = torch.Generator(device).manual_seed(seed), len(questions)
        self.B, self.q_heads, self.heads, self.d, self.vocab, self.page = requests, q_heads, heads, d, vocab, page
        self.limit, self.budget, self.searches, self.device, self.dtype = limit, budget, searches, device, dtype
        width = q_heads * d

        def matrix(*shape):
            return (torch.randn(*shape, generator=g, device=device) * shape[-2] ** -0.5).to(dtype)
        self.embed = matrix(1, vocab, width)[0] * vocab ** 0.5
        self.layers = [(matrix(width, (q_heads + 2 * heads) * d), torch.ones(d, dtype=dtype, device=device), torch.ones(d, dtype=dtype, device=device),
                        matrix(width, width)) for _ in range(layers)]
        self.head = matrix(width, vocab)
        angle = torch.arange(8192, device=device)[:, None] * 10_000.0 ** (-torch.arange(0, d, 2, device=device) / d)
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
        # the knowledge base: embeddings and tokens of passages
        self.corpus = torch.nn.functional.normalize(torch.randn(passages, width, generator=g, device=device), dim=1).to(torch.float16)
        self.passage_tokens = torch.randint(FIRST, vocab, (passages, passage_tokens), generator=g, device=device)
        # caches of all layers have one page table; a request holds `limit` slots at most
        self.width = (limit + page - 1) // page
        pages = 2 * requests * self.width
        self.k = [torch.zeros(pages, heads, page, d, dtype=dtype, device=device) for _ in range(layers)]
        self.v = [torch.zeros_like(k) for k in self.k]
        self.mass = [torch.zeros(requests, heads, self.width * page, device=device) for _ in range(layers)]
        self.free, self.used = list(range(pages)), [0] * pages
        self.pages: List[List[int]] = [[] for _ in range(requests)]
        self.slots_used, self.position = [0] * requests, [0] * requests
        self.tokens = torch.zeros(requests, 8192, dtype=torch.int32, device=device)
        self.told, self.asked = [0] * requests, [0] * requests
        # the same tokens for the rules on logits, those that a request was given (prompt, question, passages) before those that it chose: penalties are for the latter,
        # and the words of a passage are what an answer should repeat
        self.history, self.given = torch.zeros_like(self.tokens), [0] * requests
        # what a state allows: row 0 anything, row 1 no further search; a token is a bit
        allowed = torch.ones(2, (vocab + 31) // 32 * 32, dtype=torch.int64)
        allowed[:, PAD], allowed[1, SEARCH] = 0, 0
        words = (allowed.view(2, -1, 32) << torch.arange(32)).sum(-1)
        self.masks = torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32).to(device)
        shared = len(prompt) // page * page
        for token in prompt[:shared]:                     # one request's work, whose pages the others take over
            self.step([token], [0])
        for b in range(1, requests):
            self.pages[b] = list(self.pages[0])
            for p in self.pages[b]:
                self.used[p] += 1
            self.slots_used[b], self.position[b], self.told[b], self.given[b] = self.slots_used[0], self.position[0], self.told[0], self.given[0]
            self.tokens[b, :shared], self.history[b, :shared] = self.tokens[0, :shared], self.history[0, :shared]
            for m in self.mass:
                m[b] = m[0]
        for tokens in [[token] * requests for token in prompt[shared:]] + [list(t) for t in zip(*questions)]:
            self.logits, self.hidden = self.step(tokens)

    def _take(self, count: int) -> List[int]:
        taken, self.free = self.free[:count], self.free[count:]
        for p in taken:
            self.used[p] = 1
        return taken

    def _give(self, pages: List[int]) -> None:
        for p in pages:
            self.used[p] -= 1
            if self.used[p] == 0:
                self.free.append(p)

    def _ints(self, x) -> torch.Tensor:
        return torch.tensor(x, dtype=torch.int32, device=self.device)

    def _table(self, rows: List[int]) -> torch.Tensor:
        return self._ints([self.pages[b] + [-1] * (self.width - len(self.pages[b])) for b in rows])

    def cut(self, rows: List[int]) -> torch.Tensor:
        """The caches of these requests, cut to `budget` slots by the weight they had; returns the slots that stayed, of the last layer."""
        old, lengths, index = self._table(rows), self._ints([self.slots_used[b] for b in rows]), torch.tensor(rows, device=self.device)
        new = [self._take((self.budget + self.page - 1) // self.page) for _ in rows]
        table = self._ints([p + [-1] * (self.width - len(p)) for p in new])
        for k, v, mass in zip(self.k, self.v, self.mass):
            kept, _, mass[index] = ann.ann_cache_evict(k, v, old, lengths, mass[index], table, self.budget, first=4, recent=self.budget // 4)
        for b, pages in zip(rows, new):
            self._give(self.pages[b])
            self.pages[b], self.slots_used[b] = pages, min(self.slots_used[b], self.budget)
        return kept

    def step(self, next_tokens: List[int], rows=None, chosen=()):
        """One new token of each of these requests (all, unless given), which those in `chosen` chose themselves: (logits [requests, vocab], last hidden state)."""
        rows = list(range(self.B)) if rows is None else rows
        full = [b for b in rows if self.slots_used[b] == self.limit]
        if full:
            self.cut(full)
        for b, token in zip(rows, next_tokens):
            if self.slots_used[b] % self.page == 0:       # a page of its own (one that is shared is full)
                self.pages[b] += self._take(1)
            self.slots_used[b] += 1
            self.tokens[b, self.told[b]] = self.history[b, self.told[b]] = token
            if b not in chosen:                           # (changes places with the first that was chosen: their order does not matter)
                self.history[b, self.told[b]] = self.history[b, self.given[b]]
                self.history[b, self.given[b]] = token
                self.given[b] += 1
            self.told[b] += 1
        slots = self._ints([self.pages[b][(self.slots_used[b] - 1) // self.page] * self.page + (self.slots_used[b] - 1) % self.page for b in rows])
        positions, lengths = self._ints([self.position[b] for b in rows]), self._ints([self.slots_used[b] for b in rows])
        table, index = self._table(rows), torch.tensor(rows, device=self.device)
        x = self.embed[torch.tensor(next_tokens, device=self.device)]
        for (w_qkv, q_weight, k_weight, w_out), k, v, mass in zip(self.layers, self.k, self.v, self.mass):
            y = torch.nn.functional.layer_norm(x.float(), x.shape[-1:]).to(self.dtype)
            qkv = (y @ w_qkv).view(len(rows), self.q_heads + 2 * self.heads, self.d)
            q = ann.ann_qk_norm_rotate(qkv, q_weight, k_weight, positions, self.cos_sin, slots, k, v)
            m = mass[index]
            out, _ = ann.ann_paged_attention(q, k, v, table, lengths, max_length=max(self.slots_used[b] for b in rows), mass=m)
            mass[index] = m
            x = x + out.flatten(1) @ w_out
        for b in rows:
            self.position[b] += 1
        hidden = torch.nn.functional.layer_norm(x.float(), x.shape[-1:])
        return (hidden.to(self.dtype) @ self.head), hidden

    def choose(self) -> List[int]:
        """The next token of every request by the rules of its state."""
        B = self.B
        told, given = self._ints(self.told), self._ints(self.given)
        rates = [torch.full((B,), r, device=self.device) for r in (1.1, 0.2, 0.05)]
        bias = self._ints([[SEARCH, ANSWER]] * B), torch.tensor([[2.0, 1.0 * a] for a in self.asked], device=self.device)
        logits = ann.ann_logit_rules(self.logits, self.history, told, given, *rates, bias_tokens=bias[0], bias_values=bias[1],
                                     masks=self.masks, mask_rows=self._ints([0 if a < self.searches else 1 for a in self.asked]))
        return logits.float().argmax(1).tolist()

    def run(self, steps: int):
        """`steps` tokens of every request; returns the tokens, and the passages that each was given."""
        given: List[List[int]] = [[] for _ in range(self.B)]
        pending: List[List[int]] = [[] for _ in range(self.B)]     # of a passage, still to be taken in
        said: List[List[int]] = [[] for _ in range(self.B)]
        for _ in range(steps):
            tokens = self.choose()
            asking = [b for b in range(self.B) if not pending[b] and tokens[b] == SEARCH]
            chosen = [b for b in range(self.B) if not pending[b]]
            tokens = [pending[b].pop(0) if pending[b] else tokens[b] for b in range(self.B)]
            if asking:
                query = torch.nn.functional.normalize(self.hidden[asking], dim=1).to(torch.float16)
                ids, _ = ann.ann_flat_search_typed(self.corpus, query, 2)
                for b, found in zip(asking, ids.tolist()):
                    self.asked[b] += 1
                    given[b] += found
                    pending[b] = self.passage_tokens[found].flatten().tolist()
            for b in range(self.B):
                said[b].append(tokens[b])
            self.logits, self.hidden = self.step(tokens, chosen=chosen)
        return said, given


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--requests", type=int, default=4)
    parser.add_argument("--steps", type=int, default=200)
    args = parser.parse_args()
    agents = Agents(list(range(FIRST, FIRST + 40)), [[100 + 7 * b, 500 + b, 900 - b] for b in range(args.requests)])
    said, given = agents.run(args.steps)
    for b in range(args.requests):
        print(f"request {b}: {len(said[b])} tokens, passages {given[b]}, position {agents.position[b]}, slots held {agents.slots_used[b]}")


if __name__ == "__main__":
    main()
