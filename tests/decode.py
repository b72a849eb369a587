"""Inputs and 64-bit definitions for the tests of the operators over a paged cache, on the CPU."""
import math

import numpy as np
import torch

U = 2.0 ** -24                                            # half a unit in the last place of 1, binary32
HALF_ULP = {t: torch.finfo(t).eps / 2 for t in (torch.float16, torch.bfloat16, torch.float32)}   # relative, of a rounding to the type
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0, torch.float32: 0.0}                  # ... absolute, where it is subnormal


def rows(*shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def paged(lengths, page, heads, d, dtype, seed, layout="heads", unused=float("nan"), spare=3):
    """A cache whose requests have pages in any order: (k, v) [pages, heads, slots, d], table [B, width]; every place that belongs
    to no slot holds `unused`, table entries behind the last page are no pages."""
    g = torch.Generator().manual_seed(seed)
    B, width = len(lengths), max(1, max((n + page - 1) // page for n in lengths))
    count = [(n + page - 1) // page for n in lengths]
    pages = sum(count) + spare
    order = torch.randperm(pages, generator=g).tolist()
    table = torch.full((B, width), -1, dtype=torch.int32)
    shape = (pages, heads, page, d) if layout == "heads" else (pages, page, heads, d)
    caches = []
    for c in range(2):
        x = torch.full(shape, unused, dtype=dtype)
        caches.append(x if layout == "heads" else x.transpose(1, 2))
    at = 0
    for b, n in enumerate(lengths):
        for i in range(count[b]):
            p = order[at]
            at += 1
            table[b, i] = p
            m = min(page, n - i * page)
            for x in caches:
                x[p, :, :m] = torch.randn(heads, m, d, generator=g).to(dtype)
    return caches[0], caches[1], table


def attention(q, k, v, table, lengths, scale, window=0):
    """(out, lse, weights [B, heads, slots], x of every slot or -inf, sum of p |v|) in 64 bits."""
    B, Hq, d = q.shape
    pages, heads, page, _ = k.shape
    G, n_slots = Hq // heads, table.shape[1] * page
    out = np.zeros((B, Hq, d))
    size = np.zeros((B, Hq, d))
    lse = np.full((B, Hq), -np.inf)
    weight = np.zeros((B, heads, n_slots))
    most = np.zeros((B, Hq))                              # largest sum |q k| of a slot, times scale
    k64, v64, q64 = k.double().numpy(), v.double().numpy(), q.double().numpy()
    with np.errstate(all="ignore"):
        for b in range(B):
            n = max(0, min(int(lengths[b]), n_slots))
            j = np.arange(max(0, n - window) if window else 0, n)
            p = table[b].numpy()[j // page]
            good = (p >= 0) & (p < pages)
            j, p = j[good], p[good]
            if not len(j):
                continue
            for h in range(Hq):
                keys, values = k64[p, h // G, j % page], v64[p, h // G, j % page]
                x = keys @ q64[b, h] * scale
                most[b, h] = (np.abs(keys) @ np.abs(q64[b, h])).max() * abs(scale)
                m = x.max() if not np.isnan(x).any() else np.nan
                if m == -np.inf:
                    continue
                e = np.exp(x - m)
                w = e / e.sum()
                lse[b, h] = m + np.log(e.sum())
                out[b, h] = w @ values
                size[b, h] = w @ np.abs(values)
                weight[b, h // G, j] += w
    return out, lse, weight, most, size


def attention_bounds(out, lse, weight, most, size, lengths, d, dtype, G):
    """What the kernel's arithmetic may be off by: an error `x` of every exponent (a dot product of d terms in binary32, the scaling, the
    difference to the maximum and its product with log2 e), weights rounded to 16 bits or more for the product with the values, sums of n terms in 16 partial
    sums or more, and one rounding of the output."""
    n = np.asarray(lengths, dtype=np.float64).clip(min=0)
    x = (d + 8) * U * most + 8 * U * (np.abs(np.where(np.isfinite(lse), lse, 0)) + most)
    sums = (n / 16 + 24)[:, None] * U
    rel = 2 * x + 2 * sums
    o = (rel + 2.0 ** -16)[..., None] * size + HALF_ULP[dtype] * (np.abs(out) * (1 + 2.0 ** -7)) + TINY[dtype] + 1e-37
    s = x + sums + 2 * U * np.abs(np.where(np.isfinite(lse), lse, 0)) + U
    per_head = rel.reshape(rel.shape[0], -1, G).max(-1) + (G + 4) * U
    return o, s, per_head[..., None] * weight + 1e-37


def rotate(qkv, q_heads, heads, wq, wk, eps, positions, cos_sin, interleaved):
    """(q, k, v) of every token, in 64 bits, and per element the sum of sizes its rotation adds."""
    x = qkv.double()
    qk = x[:, :q_heads + heads]
    w = torch.cat([wq.double().expand(q_heads, -1), wk.double().expand(heads, -1)])
    y = qk / (qk.pow(2).mean(-1, keepdim=True) + eps).sqrt() * w
    size = y.abs().clone()
    rot = cos_sin.shape[1]
    for t in range(x.shape[0]):
        p = int(positions[t])
        if not 0 <= p < cos_sin.shape[0]:
            y[t] = 0
            size[t] = 0
            continue
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, rot // 2 + i)
            c, s = float(cos_sin[p, i]), float(cos_sin[p, rot // 2 + i])
            ya, yb = y[t, :, a].clone(), y[t, :, b].clone()
            y[t, :, a], y[t, :, b] = ya * c - yb * s, yb * c + ya * s
            size[t, :, a], size[t, :, b] = (ya * c).abs() + (yb * s).abs(), (yb * c).abs() + (ya * s).abs()
    return y[:, :q_heads], y[:, q_heads:], x[:, q_heads + heads:], size


def evict(mass, lengths, most, budget, first, recent):
    """kept [B, heads, budget], new lengths, in whole numbers and exact comparisons."""
    B, heads, _ = mass.shape
    kept = np.full((B, heads, budget), -1, dtype=np.int32)
    new = np.zeros(B, dtype=np.int32)
    for b in range(B):
        n = max(0, min(int(lengths[b]), most))
        new[b] = min(n, budget)
        for h in range(heads):
            if n <= budget:
                kept[b, h, :n] = np.arange(n)
                continue
            rank = [(0 if math.isnan(float(m)) else 1, 0.0 if math.isnan(float(m)) else float(m)) for m in mass[b, h, :n]]
            middle = sorted(range(first, n - recent), key=lambda j: (-rank[j][0], -rank[j][1], j))
            some = middle[:budget - first - recent]
            kept[b, h] = sorted(list(range(first)) + some + list(range(n - recent, n)))
    return kept, new


def rules(logits, tokens, lengths, prompts, repetition, presence, frequency, bias=None, masks=None, mask_rows=None):
    """(answer, largest size of what is added up) in 64 bits."""
    out = logits.double().numpy().copy()
    B, V = out.shape
    with np.errstate(all="ignore"):
        size = np.abs(out)
        for b in range(B):
            n, p = max(0, min(int(lengths[b]), tokens.shape[1])), max(0, int(prompts[b]))
            told = tokens[b, :n].numpy()
            r, pr, f = (float(t[b]) for t in (repetition, presence, frequency))
            count = {}
            for t, v in enumerate(told.tolist()):
                if 0 <= v < V:
                    count[v] = count.get(v, 0) + (t >= p)
            for v, c in count.items():
                x = out[b, v]
                x = x / r if x > 0 else x * r
                size[b, v] = max(size[b, v], abs(x))
                if c:
                    x = x - f * c - pr
                    size[b, v] += abs(f * c) + abs(pr)
                out[b, v] = x
            if bias is not None:
                last = {int(v): float(w) for v, w in zip(bias[0][b], bias[1][b]) if 0 <= int(v) < V}
                for v, w in last.items():
                    out[b, v] += w
                    size[b, v] += abs(w)
            if masks is not None and 0 <= int(mask_rows[b]) < masks.shape[0]:
                words = masks[int(mask_rows[b])].numpy().view(np.uint32)
                bits = (words[np.arange(V) // 32] >> (np.arange(V) % 32).astype(np.uint32)) & 1
                out[b, bits == 0] = -np.inf
    return out, size
