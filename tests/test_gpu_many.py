"""The operators that take many tokens at once against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import decode as D                                        # (beside this file)
import many as M
import paper_2505_12065_amd as ann

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def dev(x):
    """On the device with the same strides (a plain copy would lay it out again)."""
    if x is None:
        return None
    y = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=DEV)
    y.copy_(x)
    return y


def close(got, want, bound, what):
    got = got.double().cpu().numpy()
    finite = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), finite) and np.array_equal(got[~finite], want[~finite], equal_nan=True), what
    off = np.abs(got - np.where(finite, want, 0))[finite] - np.broadcast_to(bound, want.shape)[finite]
    assert off.size == 0 or off.max() <= 0, (what, off.max(), np.abs(got - want)[finite].max())


MARK = 77.0                                               # what rows hold that nobody writes


def check(call, q, k, v, table, spans, scale, d, dtype):
    T, Hq = q.shape[:2]
    out, lse = torch.full((T, Hq, d), MARK, dtype=dtype, device=DEV), torch.full((T, Hq), MARK, device=DEV)
    call(out, lse)
    want = M.attention(q, k, v, table, spans, scale)
    mine = torch.tensor([s is not None for s in spans])
    assert bool((out.cpu()[~mine] == MARK).all()) and bool((lse.cpu()[~mine] == MARK).all())
    want = [x[mine.numpy()] for x in want]
    o, s = M.bounds(*want, d, dtype)
    close(out.cpu()[mine], want[0], o, "out")
    close(lse.cpu()[mine], want[1], s, "lse")
    return out, lse


# ---- attention of new tokens -------------------------------------------------------------------

def chunk(dtype, new, held, Hq, heads, d, page, window=0, layout="heads", seed=1, q_scale=1.0, scale=None, max_length=None, edit=None, first=0, behind=0, wide=False):
    lengths = [n + h for n, h in zip(new, held)]
    k, v, table = D.paged(lengths, page, heads, d, dtype, seed, layout)
    T = first + sum(new) + behind
    q = D.rows(T, Hq, d, dtype=dtype, seed=seed + 7, scale=q_scale)
    if wide:                                              # rows of queries lie among others
        q = torch.cat([q, q], 1)[:, :Hq]
    if edit:
        q, k, v, table, lengths = edit(q, k, v, table, lengths)
    scale = d ** -0.5 if scale is None else scale
    most = max_length or table.shape[1] * page
    args = dev(q), dev(k), dev(v), dev(table), dev(M.ints(lengths)), dev(M.starts_of(new) + first)

    def call(out, lse):
        ann.ann_chunk_attention(*args, scale=scale, window=window, max_length=max_length, out=out, lse=lse)
    spans = M.chunk_spans(new, lengths, most, window, T, first)
    out, lse = check(call, q, k, v, table, spans, scale, d, dtype)
    again, lse2 = ann.ann_chunk_attention(*args, scale=scale, window=window, max_length=max_length)
    mine = torch.tensor([s is not None for s in spans], device=DEV)
    assert torch.equal(again[mine].view(torch.uint8), out[mine].view(torch.uint8)) and torch.equal(lse2[mine].view(torch.uint8), lse[mine].view(torch.uint8))
    return out


HEADS = [(8, 2, 128, 16), (3, 3, 64, 32), (7, 1, 80, 8), (16, 1, 256, 64), (5, 5, 8, 16), (34, 2, 96, 16), (12, 4, 72, 4), (24, 1, 136, 128), (6, 2, 200, 2), (40, 1, 48, 1),
         (4, 2, 128, 1024)]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("Hq,heads,d,page", HEADS)
def test_chunk_lengths_and_heads(dtype, Hq, heads, d, page):
    """Requests of no token, one and more, with contexts that end around tiles of 16, 32 and 64 slots, among rows that are nobody's."""
    new, held = [0, 1, 2, 5, 0, 17, 33, 1, 64, 9], [0, 0, 1, 14, 65, 30, 31, 129, 64, 300]
    chunk(dtype, new, held, Hq, heads, d, page, seed=d + page, first=3, behind=5)
    chunk(dtype, new, held, Hq, heads, d, page, seed=d + page + 1, layout="slots", wide=True, window=37)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("new,held,Hq,heads,d,page", [([300], [0], 8, 2, 128, 16), ([257, 3, 128], [100, 1000, 0], 4, 1, 64, 32), ([100], [1500], 32, 8, 128, 16), ([65, 1], [900, 70], 6, 3, 40, 64),
                                                      ([1], [2000], 4, 4, 256, 16), ([40, 0, 41], [512, 3, 511], 14, 2, 96, 8), ([2], [5000], 2, 1, 128, 64)])
def test_chunk_sizes(dtype, new, held, Hq, heads, d, page):
    """From less than a tile of rows to several, and few tokens of contexts that are divided."""
    chunk(dtype, new, held, Hq, heads, d, page)
    chunk(dtype, new, held, Hq, heads, d, page, window=130, seed=3, max_length=max(n + h for n, h in zip(new, held)))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 31, 32, 33, 64, 100, 1000, 2 ** 31 - 1])
def test_chunk_windows(dtype, window):
    chunk(dtype, [70, 1, 40], [0, 200, 333], 6, 2, 64, 16, window=window)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_chunk_pages_that_are_none(dtype):
    """Empty pages anywhere, a whole request of them, and page numbers far outside."""
    def edit(q, k, v, table, lengths):
        table[0, 1], table[0, 3], table[2] = -1, 2 ** 31 - 1, -5
        table[1, 0] = k.shape[0]
        return q, k, v, table, lengths
    chunk(dtype, [50, 20, 9, 30], [100, 40, 60, 0], 4, 2, 64, 16, edit=edit)
    chunk(dtype, [50, 20, 9, 30], [100, 40, 60, 0], 12, 1, 128, 4, edit=edit, window=20)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_chunk_tokens_without_a_slot(dtype):
    """Lengths below the number of new tokens, negative ones, and slots from max_length on."""
    def edit(q, k, v, table, lengths):
        return q, k, v, table, [10, -7, 150, 80, -2 ** 31]
    chunk(dtype, [20, 8, 30, 80, 3], [80, 10, 120, 0, 20], 4, 2, 64, 16, edit=edit, max_length=140)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("Hq,heads,d", [(4, 2, 64), (8, 1, 128), (2, 1, 256), (3, 3, 96)])
def test_chunk_values_that_are_not_attended_to(dtype, Hq, heads, d):
    """NaN and infinities in keys and values of later tokens do not matter to earlier ones; from their own token on they do."""
    new, held = [100, 40], [30, 200]
    lengths = [n + h for n, h in zip(new, held)]
    for bad_key in (False, True):
        k, v, table = D.paged(lengths, 16, heads, d, dtype, 5)
        q = D.rows(sum(new), Hq, d, dtype=dtype, seed=6)
        clean = ann.ann_chunk_attention(dev(q), dev(k), dev(v), dev(table), dev(M.ints(lengths)), dev(M.starts_of(new)))
        for b, i, value in ((0, 70, math.nan), (0, 90, math.inf), (1, 20, -math.inf)):
            j = held[b] + i
            for h in range(heads):
                if bad_key:
                    k[table[b, j // 16], h, j % 16, (7 * h + 3) % d] = math.nan
                else:
                    v[table[b, j // 16], h, j % 16, (7 * h + 3) % d] = value
        out, lse = ann.ann_chunk_attention(dev(q), dev(k), dev(v), dev(table), dev(M.ints(lengths)), dev(M.starts_of(new)))
        for b, i in ((0, 70), (1, 20)):
            t = sum(new[:b])
            assert torch.equal(out[t:t + i], clean[0][t:t + i]) and torch.equal(lse[t:t + i], clean[1][t:t + i])
            wrong = ~torch.isfinite(out[t + i:t + new[b]])
            if bad_key:
                assert bool(wrong.all()) and bool(torch.isnan(lse[t + i:t + new[b]]).all())
            else:
                columns = torch.zeros(Hq, d, dtype=torch.bool)
                for h in range(Hq):
                    columns[h, (7 * (h // (Hq // heads)) + 3) % d] = True
                assert torch.equal(wrong.cpu(), columns.expand(new[b] - i, Hq, d)) and torch.equal(lse, clean[1])
                assert torch.equal(torch.where(wrong, 0, out[t + i:t + new[b]]), torch.where(wrong, 0, clean[0][t + i:t + new[b]]))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_chunk_windows_leave_values_behind(dtype):
    """... and those that a window has left behind."""
    new, held, d = [90], [60], 64
    k, v, table = D.paged([150], 16, 2, d, dtype, 5)
    q = D.rows(90, 4, d, dtype=dtype, seed=6)
    args = dev(q), dev(table), dev(M.ints([150])), dev(M.starts_of(new))
    clean, _ = ann.ann_chunk_attention(args[0], dev(k), dev(v), *args[1:], window=40)
    v[table[0, 4], :, 2, 5] = math.nan                    # slot 66, of token 6
    out, _ = ann.ann_chunk_attention(args[0], dev(k), dev(v), *args[1:], window=40)
    assert torch.equal(out[:6], clean[:6]) and torch.equal(out[46:], clean[46:]) and bool(torch.isnan(out[6:46, :, 5]).all())


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_chunk_large_scores_and_other_scales(dtype):
    chunk(dtype, [60, 3], [100, 400], 4, 2, 64, 16, q_scale=40.0)
    chunk(dtype, [60, 3], [100, 400], 4, 2, 64, 16, scale=-0.3)
    chunk(dtype, [60, 3], [100, 400], 4, 2, 64, 16, scale=0.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new,held", [([70], [1000]), ([2], [4000])])
def test_chunk_values_near_the_largest(dtype, new, held):
    most = torch.finfo(dtype).max

    def edit(q, k, v, table, lengths):
        v.fill_(most * 0.99)
        return q, k, v, table, lengths
    chunk(dtype, new, held, 4, 2, 64, 16, edit=edit)


def test_chunk_weights_of_many_small_slots():
    """fp16: most of the weight lies in many slots that have little each, before one that has much."""
    def edit(q, k, v, table, lengths):
        q[:], k[:] = 0, 0
        q[..., 0] = 1.0
        j = lengths[0] - 3
        k[table[0, j // 16], :, j % 16, 0] = 8.0          # e^8 times the others' weight
        return q, k, v, table, lengths
    chunk(F16, [3], [6000], 4, 2, 64, 16, edit=edit, scale=1.0)
    chunk(F16, [130], [2000], 4, 2, 64, 16, edit=lambda *x: edit(*x[:4], [x[4][0]]), scale=1.0)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_chunk_is_paged_attention_for_single_tokens(dtype):
    held = [0, 5, 63, 200, 1000, 31]
    new = [1] * 6
    lengths = [h + 1 for h in held]
    k, v, table = D.paged(lengths, 16, 2, 128, dtype, 3)
    q = D.rows(6, 8, 128, dtype=dtype, seed=4)
    args = dev(q), dev(k), dev(v), dev(table), dev(M.ints(lengths))
    one, lse1 = ann.ann_paged_attention(*args)
    out, lse = ann.ann_chunk_attention(*args, dev(M.starts_of(new)))
    assert (one.double() - out.double()).abs().max() <= 4 * torch.finfo(dtype).eps * v.double().nan_to_num().abs().max()
    assert (lse1 - lse).abs().max() <= 1e-5


def test_chunk_offsets_beyond_32_bits():
    """Caches of more than 2^32 bytes, pages at their end, in memory of either order."""
    for layout in ("heads", "slots"):
        pages, heads, page, d = 9000, 8, 256, 128         # 4.7 GB each
        shape = (pages, heads, page, d) if layout == "heads" else (pages, page, heads, d)
        k, v = (torch.zeros(shape, dtype=BF16, device=DEV) for _ in range(2))
        k, v = (x if layout == "heads" else x.transpose(1, 2) for x in (k, v))
        g = torch.Generator(DEV).manual_seed(1)
        table = torch.tensor([[8999, 3, 8000]], dtype=torch.int32, device=DEV)
        for p in table[0].tolist():
            k[p] = torch.randn(heads, page, d, generator=g, device=DEV).to(BF16)
            v[p] = torch.randn(heads, page, d, generator=g, device=DEV).to(BF16)
        q = torch.randn(40, 16, d, generator=g, device=DEV).to(BF16)
        out, _ = ann.ann_chunk_attention(q, k, v, table, torch.tensor([700], dtype=torch.int32, device=DEV), torch.tensor([0, 40], dtype=torch.int32, device=DEV))
        small = M.ints([[0, 1, 2]])
        ks, vs = (torch.stack([x[p] for p in table[0].tolist()]).cpu() for x in (k, v))
        want = M.attention(q.cpu(), ks, vs, small, M.chunk_spans([40], [700], 768, 0, 40), d ** -0.5)
        close(out.cpu(), want[0], M.bounds(*want, d, BF16)[0], "out")
        del k, v


# ---- attention of groups with slots in common ---------------------------------------------------

def shared_cache(common, own, sizes, page, heads, d, dtype, seed, layout="heads"):
    """Groups of `sizes` requests with common[g] slots in common, of which the whole pages are the same pages, and own[b] more each: (k, v, table, lengths, group starts,
    shared)."""
    starts = [0] + np.cumsum(sizes).tolist()
    group = [g for g, n in enumerate(sizes) for _ in range(n)]
    lengths = [common[group[b]] // page * page + own[b] for b in range(len(own))]
    k, v, table = D.paged(lengths, page, heads, d, dtype, seed, layout)
    for b, g in enumerate(group):
        whole = common[g] // page
        table[b, :whole] = table[starts[g], :whole]
    return k, v, table, lengths, starts, [c // page * page for c in common]


def shared(dtype, common, own, sizes, Hq, heads, d, page, layout="heads", seed=1, max_shared=None, max_own=None, edit=None, scale=None, q_scale=1.0):
    k, v, table, lengths, starts, together = shared_cache(common, own, sizes, page, heads, d, dtype, seed, layout)
    q = D.rows(len(own), Hq, d, dtype=dtype, seed=seed + 9, scale=q_scale)
    if edit:
        q, k, v, table, lengths, starts, together = edit(q, k, v, table, lengths, starts, together)
    scale = d ** -0.5 if scale is None else scale
    most = table.shape[1] * page
    args = dev(q), dev(k), dev(v), dev(table), dev(M.ints(lengths)), dev(M.ints(starts)), dev(M.ints(together))
    kw = dict(scale=scale, max_shared=max_shared, max_own=max_own)
    spans = M.shared_spans(lengths, starts, together, most if max_shared is None else max_shared, most if max_own is None else max_own)
    out, lse = check(lambda out, lse: ann.ann_shared_attention(*args, out=out, lse=lse, **kw), q, k, v, table, spans, scale, d, dtype)
    again, lse2 = ann.ann_shared_attention(*args, **kw)
    assert torch.equal(again.view(torch.uint8), out.view(torch.uint8)) and torch.equal(lse2.view(torch.uint8), lse.view(torch.uint8))
    return out


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("Hq,heads,d,page", HEADS)
def test_shared_groups_and_heads(dtype, Hq, heads, d, page):
    """Groups of one request and more, nothing in common, nothing of one's own."""
    common, sizes = [130, 64, 0, 1000], [5, 1, 3, 2]
    own = [0, 1, 2, 33, 70, 5, 0, 9, 64, 200, 17]
    shared(dtype, common, own, sizes, Hq, heads, d, page, seed=d + page)
    shared(dtype, common, own, sizes, Hq, heads, d, page, seed=d + page + 1, layout="slots", max_shared=1000, max_own=200)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("common,own,sizes,Hq,heads,d,page", [([2000], [100, 20, 50, 7, 1], [5], 32, 8, 128, 16), ([500, 300], [40] * 70, [64, 6], 8, 2, 64, 32),
                                                              ([5000], [10, 900], [2], 4, 2, 128, 64), ([96], [500] * 9, [9], 14, 2, 256, 16), ([16], [3], [1], 2, 2, 40, 16)])
def test_shared_sizes(dtype, common, own, sizes, Hq, heads, d, page):
    shared(dtype, common, own, sizes, Hq, heads, d, page)
    shared(dtype, common, own, sizes, Hq, heads, d, page, max_shared=max(common), max_own=max(own) or 1, seed=5)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_shared_bounds_that_cut(dtype):
    """max_shared below what is shared leaves the rest to the requests; max_own below what is theirs leaves it out."""
    shared(dtype, [320], [70, 20, 0, 100], [4], 4, 2, 64, 16, max_shared=200, max_own=150)
    shared(dtype, [320], [70, 20, 0, 100], [4], 4, 2, 64, 16, max_shared=0, max_own=330)
    shared(dtype, [320], [70, 20, 0, 100], [4], 4, 2, 64, 16, max_own=1)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_shared_odd_arguments(dtype):
    """Requests in no group, lengths inside what is shared, negative numbers, pages that are none, groups of nobody."""
    def edit(q, k, v, table, lengths, starts, together):
        lengths[1], lengths[2], lengths[5] = 100, -3, 0
        table[0, 2], table[4, 11] = -1, k.shape[0] + 5
        # (the shared slots are read by the first request's pages; the definition here goes by each request's own)
        table[1:5, 2] = -1
        return q, k, v, table, lengths, [1, 1, 5, 5, 6], [50, 160, 9, -4]
    common, own = [160], [70, 20, 30, 64, 100, 20, 7]
    shared(dtype, common, own, [7], 6, 2, 64, 16, edit=edit)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_shared_values_near_the_largest(dtype):
    def edit(q, k, v, *rest):
        v.fill_(torch.finfo(dtype).max * 0.99)
        return q, k, v, *rest
    shared(dtype, [1000], [70, 20, 300], [3], 4, 2, 64, 16, edit=edit)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_shared_large_scores_and_other_scales(dtype):
    for kw in (dict(q_scale=40.0), dict(scale=-0.3), dict(scale=0.0)):
        shared(dtype, [200], [70, 20, 300], [3], 4, 2, 64, 16, **kw)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_shared_values_that_are_not_attended_to(dtype):
    """A request whose length ends inside the shared slots does not see what lies behind it."""
    k, v, table, lengths, starts, together = shared_cache([128], [10, 20, 5], [3], 16, 2, 64, dtype, 3)
    lengths[1] = 60
    q = D.rows(3, 4, 64, dtype=dtype, seed=2)
    rest = dev(table), dev(M.ints(lengths)), dev(M.ints(starts)), dev(M.ints(together))
    clean, lse1 = ann.ann_shared_attention(dev(q), dev(k), dev(v), *rest)
    v[table[0, 4], :, 3, 9] = math.nan                    # slot 67
    out, lse2 = ann.ann_shared_attention(dev(q), dev(k), dev(v), *rest)
    assert torch.equal(out[1], clean[1]) and torch.equal(lse1, lse2)
    assert bool(torch.isnan(out[0, :, 9]).all()) and bool(torch.isnan(out[2, :, 9]).all()) and int(torch.isnan(out).sum()) == 8


# ---- rotation and append ------------------------------------------------------------------------

def append(dtype, new, held, Hq, heads, d, page, rot, interleaved=False, layout="heads", seed=1, positions=None, amplitude=1.0, first=0, behind=0, wide=False, edit=None,
           base=10_000.0):
    lengths = [n + h for n, h in zip(new, held)]
    k, v, table = D.paged(lengths, page, heads, d, dtype, seed, layout, unused=MARK)
    T = first + sum(new) + behind
    x = D.rows(T, Hq + 2 * heads, d, dtype=dtype, seed=seed + 7)
    if wide:
        x = torch.cat([x, x], 1)[:, :Hq + 2 * heads]
    if edit:
        table, lengths = edit(table, lengths, k.shape[0])
    spans = M.chunk_spans(new, lengths, 2 ** 31, 0, T, first)
    slot = [None if s is None else max(lengths[s[0]], 0) - new[s[0]] + (t - first - sum(new[:s[0]])) for t, s in enumerate(spans)]
    p = torch.tensor([-1 if s is None else s for s in slot]).clamp(min=-1) if positions is None else positions(T)
    frequencies = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))
    q = torch.full((T, Hq, d), MARK, dtype=dtype, device=DEV)
    kd, vd = dev(k), dev(v)
    ann.ann_rotate_append(dev(x), dev(M.starts_of(new) + first), dev(M.ints(lengths)), dev(table), frequencies.to(DEV) if rot else None, kd, vd,
                          positions=None if positions is None else dev(p.to(torch.int32)), amplitude=amplitude, interleaved=interleaved, q=q)
    wq, wk, wv, size = M.rotated(x, Hq, heads, p, frequencies, amplitude, interleaved)
    # cosine and sine: 2 ulp of the function and two roundings of its argument, the amplitude's product and rounding, two products and a sum
    bound = size * (12 * D.U) + D.HALF_ULP[dtype] * size * (1 + 2.0 ** -10) + D.TINY[dtype]
    want_k, want_v = k.double(), v.double()
    bound_k = torch.zeros_like(want_k)
    mine = torch.tensor([s is not None for s in spans])
    for t, s in enumerate(spans):
        if s is None or int(p[t]) < 0 or not 0 <= slot[t] < table.shape[1] * page:
            continue
        at = int(table[s[0], slot[t] // page])
        if 0 <= at < k.shape[0]:
            want_k[at, :, slot[t] % page], want_v[at, :, slot[t] % page], bound_k[at, :, slot[t] % page] = wk[t], wv[t], bound[t, Hq:]
    assert bool((q.cpu()[~mine] == MARK).all())
    pad = p < 0
    assert bool((q.cpu()[mine & pad] == 0).all())
    assert bool(((q.cpu().double() - wq).abs() <= bound[:, :Hq])[mine & ~pad].all())
    assert bool(((kd.cpu().double() - want_k).abs() <= bound_k).all()) and torch.equal(vd.cpu().double(), want_v)
    if rot < d:                                           # bits that are not rotated stay
        assert torch.equal(q.cpu()[mine & ~pad][..., rot:], x[mine & ~pad][:, :Hq, rot:])


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("Hq,heads,d,page,rot", [(8, 2, 128, 16, 128), (3, 3, 64, 32, 64), (7, 1, 80, 8, 32), (16, 1, 256, 64, 256), (5, 5, 8, 16, 0), (20, 2, 96, 16, 96), (4, 4, 72, 4, 64),
                                                 (12, 1, 136, 128, 16), (6, 2, 200, 2, 192), (9, 3, 48, 1, 48)])
def test_append_heads_and_pairs(dtype, interleaved, Hq, heads, d, page, rot):
    new, held = [0, 1, 2, 5, 0, 17, 33, 1], [0, 0, 1, 14, 65, 30, 31, 129]
    append(dtype, new, held, Hq, heads, d, page, rot, interleaved, first=2, behind=3)
    append(dtype, new, held, Hq, heads, d, page, rot, interleaved, layout="slots", wide=True, amplitude=-1.37, seed=4)


@pytest.mark.parametrize("new", [[1], [1] * 9, [700], [40] * 70, [3, 0] * 40, [1] * 130])
def test_append_batches(new):
    """Enough tokens for several rows to a lane, and enough requests for the search for a token's to take two steps."""
    append(BF16, new, [7 * b % 50 for b in range(len(new))], 6, 2, 64, 16, 64)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_append_positions_of_their_own(dtype):
    """Positions that are not slots: far ones, negative ones (padding)."""
    append(dtype, [20, 30], [5, 100], 4, 2, 64, 16, 64,
           positions=lambda T: torch.tensor([(-1 if t % 7 == 3 else -2 ** 31 if t % 7 == 5 else 37 * t * t if t % 2 else 131_071 - t) for t in range(T)]))
    append(dtype, [20], [5], 4, 2, 64, 16, 64, positions=lambda T: torch.arange(2 ** 31 - 1 - T, 2 ** 31 - 1), base=500_000.0)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_append_slots_that_are_none(dtype):
    """Lengths below the number of new tokens, negative ones, beyond the table, and pages that are none."""
    def edit(table, lengths, pages):
        table[3, 0], table[3, 1] = pages, -9
        return table, [10, -7, 10 ** 6, 40]
    append(dtype, [20, 8, 30, 40], [80, 10, 12, 0], 4, 2, 64, 16, 64, edit=edit)


def test_append_is_norm_rotate_of_unit_rows():
    """With weights of one, rows of mean square 1 and the same angles ann_qk_norm_rotate does the same."""
    T, Hq, heads, d = 40, 4, 2, 64
    x = torch.randn(T, Hq + 2 * heads, d, generator=torch.Generator().manual_seed(1))
    x = (x / x.pow(2).mean(-1, keepdim=True).sqrt()).to(DEV)
    frequencies, amplitude = ann.ann_rotation_frequencies(d, device=DEV)
    caches = [torch.zeros(4, heads, 16, d, device=DEV) for _ in range(4)]
    at = torch.arange(T, dtype=torch.int32, device=DEV)
    angle = at.double()[:, None] * frequencies
    one = torch.ones(d, device=DEV)
    q1 = ann.ann_qk_norm_rotate(x, one, one, at, torch.cat([angle.cos(), angle.sin()], 1).float(), at, caches[0], caches[1], eps=0.0)
    q2 = ann.ann_rotate_append(x, M.ints([0, T]).to(DEV), M.ints([T]).to(DEV), M.ints([[0, 1, 2, 3]]).to(DEV), frequencies, caches[2], caches[3], amplitude=amplitude)
    assert (q1 - q2).abs().max() < 4e-6 and (caches[0] - caches[2]).abs().max() < 4e-6 and torch.equal(caches[1], caches[3])


# ---- together ------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F16, BF16])
def test_a_run_of_them_together(dtype):
    """A prompt for all, its pages shared, then a passage and a token for each: what the three operators leave is what dense attention over rotated rows of the same bits gives."""
    heads, Hq, d, page, B, prompt, passage = 2, 6, 64, 16, 4, 48, [5, 21, 0, 40]
    frequencies, amplitude = ann.ann_rotation_frequencies(d, 10_000.0, scaling="ramp", factor=4.0, original=32, device=DEV)
    k, v = (torch.full((40, heads, page, d), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
    free = torch.randperm(40, generator=torch.Generator().manual_seed(2)).tolist()
    table = torch.full((B, 8), -1, dtype=torch.int32)
    table[:, :3] = torch.tensor(free[:3])
    for b in range(B):
        table[b, 3:] = torch.tensor(free[3 + 5 * b:8 + 5 * b])
    held, rows, queries = [0] * B, [[] for _ in range(B)], [[] for _ in range(B)]
    table_d = table.to(DEV)

    def take(new, seed, which=None):
        which = list(range(B)) if which is None else which
        x = D.rows(sum(new), Hq + 2 * heads, d, dtype=dtype, seed=seed)
        for b, n in zip(which, new):
            held[b] += n
        lengths, starts, t = M.ints([held[b] for b in which]).to(DEV), M.starts_of(new).to(DEV), table_d[which].contiguous()
        q = ann.ann_rotate_append(x.to(DEV), starts, lengths, t, frequencies, k, v, amplitude=amplitude)
        return x, q, t, lengths, starts

    x, q, t, lengths, starts = take([prompt], 1, [0])
    first, _ = ann.ann_chunk_attention(q, k, v, t, lengths, starts)
    held[:] = [prompt] * B
    x2, q2, t, lengths, starts = take(passage, 2)
    second, _ = ann.ann_chunk_attention(q2, k, v, t, lengths, starts, max_length=max(held))
    x3, q3, t, lengths, starts = take([1] * B, 3)
    third, _ = ann.ann_shared_attention(q3, k, v, t, lengths, M.ints([0, B]).to(DEV), M.ints([prompt]).to(DEV), max_shared=prompt, max_own=max(held) - prompt)

    def dense(b, queries, last):
        """Queries [n, Hq, d] of the tokens in the slots before `last`."""
        at = torch.arange(last)
        keys, values = (c.cpu()[table[b, at // page].long(), :, at % page].double() for c in (k, v))
        n, G = queries.shape[0], Hq // heads
        s = torch.einsum("nhgd,jhd->nhgj", queries.double().cpu().view(n, heads, G, d), keys) / math.sqrt(d)
        s.masked_fill_(at > (torch.arange(n) + last - n)[:, None, None, None], -math.inf)
        return torch.einsum("nhgj,jhd->nhgd", torch.softmax(s, -1), values).reshape(n, Hq, d)

    tolerance = 4 * torch.finfo(dtype).eps * 4            # (values are below 5, sizes of sums below 4: one rounding of weights, one of the output)
    assert (first.cpu().double() - dense(0, q, prompt)).abs().max() < tolerance
    at = 0
    for b in range(B):
        if passage[b]:
            assert (second[at:at + passage[b]].cpu().double() - dense(b, q2[at:at + passage[b]], prompt + passage[b])).abs().max() < tolerance
        at += passage[b]
        assert (third[b:b + 1].cpu().double() - dense(b, q3[b:b + 1], prompt + passage[b] + 1)).abs().max() < tolerance
    # the keys are the rotated rows
    angle = torch.arange(prompt, dtype=torch.float64)[:, None] * frequencies.cpu()
    c, s = angle.cos()[:, None] * amplitude, angle.sin()[:, None] * amplitude
    y = x[:, Hq:Hq + heads].double()
    want = torch.cat([y[..., :d // 2] * c - y[..., d // 2:] * s, y[..., d // 2:] * c + y[..., :d // 2] * s], -1)
    at = torch.arange(prompt)
    assert (k.cpu()[table[0, at // page].long(), :, at % page].double() - want).abs().max() < 8 * torch.finfo(dtype).eps
