"""Inputs and 64-bit definitions for the tests of the operators that take many tokens at once, on the CPU."""
import numpy as np
import torch

from decode import HALF_ULP, TINY, U


def ints(x):
    return torch.tensor(x, dtype=torch.int32)


def starts_of(new):
    return ints([0] + np.cumsum(new).tolist())


def attention(q, k, v, table, spans, scale):
    """Rows t = 0, 1, ... of q [T, query heads, d], each with (request, lo, hi) or None: (out, lse, largest |scale q k|, sum of p |v|, largest weight times the sum of
    |v|) in 64 bits; rows of None are NaN."""
    T, Hq, d = q.shape
    pages, heads, page, _ = k.shape
    G = Hq // heads
    out, size, flat = (np.zeros((T, Hq, d)) for _ in range(3))
    lse, most = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    count = np.zeros(T)
    k64, v64, q64 = k.double().numpy(), v.double().numpy(), q.double().numpy()
    with np.errstate(all="ignore"):
        for t, span in enumerate(spans):
            if span is None:
                out[t], lse[t] = np.nan, np.nan
                continue
            b, lo, hi = span
            j = np.arange(lo, max(lo, hi))
            p = table[b].numpy()[j // page]
            good = (p >= 0) & (p < pages)
            j, p = j[good], p[good]
            count[t] = len(j)
            if not len(j):
                continue
            for h in range(heads):
                keys, values = k64[p, h, j % page], v64[p, h, j % page]
                x = q64[t, h * G:(h + 1) * G] @ keys.T * scale
                most[t, h * G:(h + 1) * G] = (np.abs(q64[t, h * G:(h + 1) * G]) @ np.abs(keys).T).max(1) * abs(scale)
                for g in range(G):
                    m = x[g].max() if not np.isnan(x[g]).any() else np.nan
                    if m == -np.inf:
                        continue
                    e = np.exp(x[g] - m)
                    w, r = e / e.sum(), h * G + g
                    lse[t, r] = m + np.log(e.sum())
                    # (a weight that is 0 because its score is -inf meets finite values only in these tests)
                    out[t, r], size[t, r] = w @ values, w @ np.abs(values)
                    flat[t, r] = w.max() * np.abs(values).sum(0)
    return out, lse, most, size, flat, count


def bounds(out, lse, most, size, flat, count, d, dtype):
    """What the kernels' arithmetic may be off by: an error x of every exponent (a dot product of d terms in binary32, its scaling, the difference to the maximum); sums of `count`
    terms in binary32, in any order; weights rounded once to 16-bit types (fp16: no finer than 2^-32 of the largest); one rounding of the output."""
    finite = np.where(np.isfinite(lse), np.abs(lse), 0)
    x = (d + 8) * U * most + 8 * U * (finite + most)
    sums = (count + 32)[:, None] * U
    weight = HALF_ULP[dtype] * (1 + 2.0 ** -7) if dtype != torch.float32 else 0.0
    o = (2 * x + 2 * sums + weight)[..., None] * size + (2.0 ** -32 * flat if dtype == torch.float16 else 0) + \
        HALF_ULP[dtype] * np.abs(out) * (1 + 2.0 ** -6) + TINY[dtype] + 1e-37
    return o, x + sums + 2 * U * finite + U


def chunk_spans(new, lengths, max_length, window, T, first=0):
    """Spans of packed tokens, None in front of `first` and behind the last request."""
    spans = [None] * first
    for b, (n, length) in enumerate(zip(new, lengths)):
        for i in range(n):
            slot = max(length, 0) - n + i
            if not 0 <= slot < max_length:
                spans.append((b, 0, 0))
            else:
                spans.append((b, max(0, slot + 1 - window) if window else 0, slot + 1))
    return spans + [None] * (T - len(spans))


def shared_spans(lengths, group_starts, shared, max_shared, max_own):
    spans = []
    for b, length in enumerate(lengths):
        length, common = max(length, 0), 0
        for g in range(len(shared)):
            if group_starts[g] <= b < group_starts[g + 1]:
                common = min(max(shared[g], 0), max_shared, length)
        spans.append((b, 0, common + min(length - common, max_own)))
    return spans


def rotated(qkv, q_heads, heads, positions, frequencies, amplitude, interleaved):
    """(q, k, v) of every token in 64 bits, and the sum of sizes that a rotation adds; a negative position gives zeros."""
    x = qkv.double()
    qk = x[:, :q_heads + heads].clone()
    size = qk.abs()
    half = len(frequencies)
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    angle = positions.double()[:, None] * frequencies
    c, s = (f(angle)[:, None] * amplitude for f in (torch.cos, torch.sin))
    u, w = qk[..., a].clone(), qk[..., b].clone()
    qk[..., a], qk[..., b] = u * c - w * s, w * c + u * s
    # (of the rounded cosines and sines, products and sum: five roundings of amplitude (|u| + |w|) at most, and the cosine's own error)
    size[..., a] = size[..., b] = abs(amplitude) * (u.abs() + w.abs())
    qk[positions < 0] = 0
    return qk[:, :q_heads], qk[:, q_heads:], x[:, q_heads + heads:], size
