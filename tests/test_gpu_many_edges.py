"""The operators that take many tokens at once at the ends of their ranges, and ways to call them that take another path."""
import math

import numpy as np
import pytest
import torch

import decode as D                                        # (beside this file)
import many as M
import paper_2505_12065_amd as ann
from test_gpu_many import append, chunk, close, dev, shared, shared_cache

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
MOST = 2 ** 31 - 1


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("B,most", [(64, 3), (65, 3), (70, 90), (300, 2)])
def test_chunk_many_requests(dtype, B, most):
    """As many requests as a wave has lanes, and more; few rows of each, and many."""
    new = [(7 * b) % (most + 1) for b in range(B)]
    held = [(13 * b) % 97 for b in range(B)]
    chunk(dtype, new, held, 6, 2, 64, 16, seed=B)
    chunk(dtype, new, held, 4, 4, 40, 8, seed=B + 1, window=23, first=1, behind=2)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("groups", [63, 64, 65, 100])
def test_shared_many_groups(dtype, groups):
    """As many groups as a wave has lanes, less and more, and more requests than that."""
    sizes = [1 + g % 3 for g in range(groups)]
    common = [16 * (g % 7) for g in range(groups)]
    own = [(11 * b) % 50 for b in range(sum(sizes))]
    shared(dtype, common, own, sizes, 4, 2, 64, 16, seed=groups)
    shared(dtype, common, own, sizes, 4, 1, 128, 8, seed=groups, max_shared=64, max_own=30)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("Hq,heads,d", [(17, 1, 64), (70, 2, 128), (33, 1, 256), (130, 1, 72)])
def test_many_heads_to_a_cache_head(dtype, Hq, heads, d):
    """More query heads than a tile of rows holds."""
    chunk(dtype, [1, 2, 0, 3], [40, 100, 0, 500], Hq, heads, d, 16)
    shared(dtype, [150, 32], [20, 30, 4, 300], [3, 1], Hq, heads, d, 16)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_many_rows_in_common(dtype):
    """Groups whose rows fill tiles of 128 and leave some over, with enough to do that it is not done by few rows at a time."""
    shared(dtype, [3500, 900], [3 + b % 40 for b in range(50)], [40, 10], 32, 4, 128, 16, seed=3)
    shared(dtype, [6000], [100] * 33, [33], 16, 2, 256, 32, seed=4, layout="slots")


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_one_token_of_a_long_context(dtype):
    """A context that is divided into as many parts as there are."""
    k, v, table = D.paged([60_000], 64, 1, 64, dtype, 3)
    q = D.rows(1, 2, 64, dtype=dtype, seed=4)
    args = dev(q), dev(k), dev(v), dev(table), dev(M.ints([60_000]))
    out, lse = ann.ann_chunk_attention(*args, dev(M.ints([0, 1])))
    want = M.attention(q, k, v, table, [(0, 0, 60_000)], 64 ** -0.5)
    o, s = M.bounds(*want, 64, dtype)
    close(out.cpu(), want[0], o, "out")
    close(lse.cpu(), want[1], s, "lse")


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_the_longest_contexts(dtype):
    """As many slots as a token may attend to, and, with a window, as a page table may hold (its pages are the same three).  All scores are 0 and all values of a column the same, so each weighted sum is
    the sum of weights times a power of two: integers up to 2^26 and eight of them or more at a time, which binary32 holds."""
    page, d, n = 1024, 8, 2 ** 26 - 5
    width = (MOST - 65536) // page
    k, v = torch.randn(3, 4, page, d, device=DEV).to(dtype), torch.zeros(3, 4, page, d, dtype=dtype, device=DEV)
    v[..., 0], v[..., 1] = 1, -0.5
    table = torch.zeros(2, width, dtype=torch.int32, device=DEV)
    table[:, 1::3], table[:, 2::3] = 1, 2
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731

    def exact(out, lse, slots):
        assert (out[..., 0].float() - 1).abs().max() <= 2 * D.HALF_ULP[dtype] and (out[..., 1].float() + 0.5).abs().max() <= 2 * D.HALF_ULP[dtype]
        assert (lse.double() - torch.tensor(slots, dtype=torch.float64, device=DEV).log().view(-1, 1)).abs().max() <= 2.0 ** -17

    q = torch.zeros(2, 4, d, dtype=dtype, device=DEV)
    exact(*ann.ann_chunk_attention(q, k, v, table, ints(n, 100), ints(0, 1, 2), max_length=2 ** 26), [n, 100])
    # many rows: not divided
    rows = torch.zeros(600, 1024, d, dtype=dtype, device=DEV)[:, :4 if dtype == F32 else 512]
    exact(*ann.ann_chunk_attention(rows, k, v, table, ints(n, 1000), ints(0, 100, 600), max_length=2 ** 26), [*range(n - 99, n + 1), *range(501, 1001)])
    n = width * page - 5
    exact(*ann.ann_chunk_attention(q, k, v, table, ints(n, 100), ints(0, 1, 2), window=5000), [5000, 100])
    # the same slots, a request's first part in common with another
    n = 2 ** 26 + 10_000
    for common in (0, 20_000, 5 * 10 ** 7, 2 ** 26):
        exact(*ann.ann_shared_attention(q, k, v, table, ints(n, n), ints(0, 2), ints(common), max_shared=2 ** 26, max_own=2 ** 26), [min(n, common + 2 ** 26)] * 2)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_sums_of_many_small_weights(dtype):
    """One slot of a large score and many of equal small ones, whose weights are no powers of two: rounded at every one of them, sums would drift."""
    n, G, T, d = 131_072, 24, 2048, 64
    page = 256
    k, v = torch.zeros(n // page, 1, page, d, device=DEV), torch.ones(n // page, 1, page, d, dtype=dtype, device=DEV)
    k[0, 0, 0, 0] = 1
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    q = torch.zeros(T, G, d, device=DEV)
    q[:, :, 0] = torch.arange(G, device=DEV) / 8 + 4      # scores of the one slot, exact in every type
    table = torch.arange(n // page, dtype=torch.int32, device=DEV).view(1, -1)
    out, lse = ann.ann_chunk_attention(q.to(dtype), k.to(dtype), v, table, ints(n), ints(0, T), scale=1.0, max_length=n)
    slots = torch.arange(n - T, n, dtype=torch.float64)[:, None]
    want = (torch.exp(torch.arange(G, dtype=torch.float64) / 8 + 4) + slots).log()
    # a lane's sum: up to 2^12 tiles, each off by 2^-24 of the sum; a tile's: 32 weights; exponents, exp2 and the logarithm 2^-18 together
    assert (lse.double().cpu() - want).abs().max() <= 2.0 ** -12 + 2.0 ** -19 + 2.0 ** -18
    # products with V: fp32 2^12 tiles of 32, 16 bits eight slots at a time, and the weights' rounding and the output's; and the sum that they are divided by
    assert (out.double() - 1).abs().max() <= (2.0 ** -12 + 2.0 ** -19 if dtype == F32 else 2.0 ** -10 + 2 * D.HALF_ULP[dtype]) + 2.0 ** -12 + 2.0 ** -18


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("common", [0, 131_072])
def test_sums_of_many_small_weights_of_single_tokens(dtype, common):
    """The same for so many requests that nothing is divided; all slots in common, or none."""
    n, G, B, d, page = 131_072, 4, 16_384 if common else 600, 64, 256
    k, v = torch.zeros(n // page, 1, page, d, device=DEV), torch.ones(n // page, 1, page, d, dtype=dtype, device=DEV)
    k[0, 0, 0, 0] = 1
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    q = torch.zeros(B, G, d, device=DEV)
    q[:, :, 0] = torch.arange(G, device=DEV) / 8 + 4.3125
    table = torch.arange(n // page, dtype=torch.int32, device=DEV).repeat(B, 1)
    out, lse = ann.ann_shared_attention(q.to(dtype), k.to(dtype), v, table, ints(*[n] * B), ints(0, B), ints(common), max_shared=common, max_own=page if common else n, scale=1.0)
    want = (torch.exp(torch.arange(G, dtype=torch.float64) / 8 + 4.3125) + n - 1).log()
    # as above; by few rows a wave has a quarter of the slots, 32 at a time, and weights of 16 bits are two operands
    assert (lse.double().cpu() - want).abs().max() <= 2.0 ** -12 + 2.0 ** -19 + 2.0 ** -18
    assert (out.double() - 1).abs().max() <= (2.0 ** -12 + 2.0 ** -19 if dtype == F32 else 2.0 ** -10 + 2 * D.HALF_ULP[dtype]) + 2.0 ** -12 + 2.0 ** -18


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,n,common", [(1, 6000, None), (100, 6000, None), (5, 3000, 2990), (70, 9000, 8000), (600, 700, None)])
def test_parts_of_large_scores(dtype, T, n, common):
    """Scores near 1000, exact in every type, a part's largest not another's: what parts say of themselves has to be as exact as their weights."""
    d, heads, page = 64, 2, 16
    g = torch.Generator().manual_seed(n)
    width = (n + page - 1) // page
    k, v = torch.zeros(width, heads, page, d), torch.randn(width, heads, page, d, generator=g).to(dtype)
    k[..., 0], k[..., 1] = 1, torch.randint(0, 5, (width, heads, page), generator=g) + 3 * (torch.arange(width) // 16 % 2)[:, None, None]
    q = torch.zeros(T, heads, d)
    q[..., 0], q[..., 1] = 992, 1
    table = torch.randperm(width, generator=g).to(torch.int32).view(1, -1)
    if common is None:
        spans = M.chunk_spans([T], [n], n, 0, T)
        out, lse = ann.ann_chunk_attention(dev(q.to(dtype)), dev(k.to(dtype)), dev(v), dev(table), dev(M.ints([n])), dev(M.ints([0, T])), scale=1.0, max_length=n)
    else:
        table = table.repeat(T, 1)
        spans = [(b, 0, n) for b in range(T)]
        out, lse = ann.ann_shared_attention(dev(q.to(dtype)), dev(k.to(dtype)), dev(v), dev(table), dev(M.ints([n] * T)), dev(M.ints([0, T])), dev(M.ints([common])), max_shared=common,
                                            max_own=n - common, scale=1.0)
    want, want_lse = (torch.from_numpy(x) for x in M.attention(q.to(dtype), k.to(dtype), v, table, spans, 1.0)[:2])
    # differences of scores up to 7, as exponents of 2 up to 10.1: off by 2^-25 of them as 1 / ln 2 is rounded, 2^-24 each as exponents and as differences of parts; exp2 2^-22; sums 2^-15
    slack = 10.1 * 3 * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -15
    most = float(v.abs().max())
    assert (out.double().cpu() - want).abs().max() <= (slack + (3 * D.HALF_ULP[dtype] if dtype != F32 else 0)) * most
    # ... which 1000 / ln 2 is off by 2^-24 of, and its rounding, as ln 2's, and the logarithm's
    assert (lse.double().cpu() - want_lse).abs().max() <= 1000 * 3 * 2.0 ** -24 + slack


def test_many_tokens():
    """More tokens than 16 bits number, whose rows are looked at here and there."""
    T, d, held = 70_000, 16, 37
    g = torch.Generator(DEV).manual_seed(1)
    pages = (T + held + 255) // 256
    k, v = (torch.zeros(pages + 1, 1, 256, d, dtype=BF16, device=DEV) for _ in range(2))
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(2)).to(torch.int32).view(1, pages).to(DEV)
    first = torch.randn(held, 3, d, generator=g, device=DEV).to(BF16)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    frequencies, _ = ann.ann_rotation_frequencies(16, device=DEV)
    ann.ann_rotate_append(first, ints(0, held), ints(held), table, frequencies, k, v)
    x = torch.randn(T, 3, d, generator=g, device=DEV).to(BF16)
    q = ann.ann_rotate_append(x, ints(0, T), ints(held + T), table, frequencies, k, v)
    out, _ = ann.ann_chunk_attention(q, k, v, table, ints(held + T), ints(0, T), window=50)
    flat = table[0].long()
    for t in (0, 1, 100, 32_767, 65_535, 65_536, T - 1):
        slot = held + t
        j = torch.arange(max(0, slot - 49), slot + 1, device=DEV)
        keys, values = k[flat[j // 256], 0, j % 256].double(), v[flat[j // 256], 0, j % 256].double()
        p = torch.softmax(keys @ q[t, 0].double() / 4, 0)
        assert (out[t, 0].double() - p @ values).abs().max() < 4 * torch.finfo(BF16).eps
        want = x[t, 2] if t >= 0 else None
        assert torch.equal(v[flat[slot // 256], 0, slot % 256], want)
    angle = float(held + T - 1) * frequencies
    c, s = angle.cos(), angle.sin()
    a, b = x[-1, 0, :8].double(), x[-1, 0, 8:].double()
    assert (q[-1, 0].double() - torch.cat([a * c - b * s, b * c + a * s])).abs().max() < 8 * torch.finfo(BF16).eps


def test_starts_outside_the_tokens():
    """Starts count as within [0, T]."""
    k, v, table = D.paged([60, 40], 16, 2, 64, F16, 3)
    q = D.rows(30, 4, 64, dtype=F16, seed=2)
    args = dev(q), dev(k), dev(v), dev(table), dev(M.ints([60, 40]))
    want, _ = ann.ann_chunk_attention(*args, dev(M.ints([0, 10, 30])))
    out, _ = ann.ann_chunk_attention(*args, dev(M.ints([-2 ** 31, 10, MOST])))
    assert torch.equal(out, want)


# ---- workspace, streams and graphs ----------------------------------------------------------------

def inputs(dtype=BF16, seed=1):
    new, held = [3, 0, 40, 7], [900, 10, 300, 2500]
    lengths = [n + h for n, h in zip(new, held)]
    k, v, table = D.paged(lengths, 16, 2, 64, dtype, seed)
    q = D.rows(sum(new), 8, 64, dtype=dtype, seed=seed + 1)
    return [dev(x) for x in (q, k, v, table, M.ints(lengths), M.starts_of(new))], (q, k, v, table, M.chunk_spans(new, lengths, table.shape[1] * 16, 0, sum(new)))


def shared_inputs(dtype=BF16, seed=1):
    k, v, table, lengths, starts, together = shared_cache([800, 2000], [60, 0, 7, 130, 300], [3, 2], 16, 2, 64, dtype, seed)
    q = D.rows(5, 8, 64, dtype=dtype, seed=seed + 1)
    return [dev(x) for x in (q, k, v, table, M.ints(lengths), M.ints(starts), M.ints(together))], (q, k, v, table, M.shared_spans(lengths, starts, together, MOST, MOST))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_any_workspace(dtype):
    """With all of its own, with a buffer that holds some parts, and with one that holds none."""
    for f, make, need in ((ann.ann_chunk_attention, inputs, ann.ann_chunk_attention_workspace_bytes(50, 4, 8, 2, 64, dtype, 2512)),
                          (ann.ann_shared_attention, shared_inputs, ann.ann_shared_attention_workspace_bytes(5, 2, 8, 2, 64, dtype, 2304, 2304))):
        args, plain = make(dtype)
        want = M.attention(*plain, 64 ** -0.5)
        o, s = M.bounds(*want, 64, dtype)
        assert need > 0
        for size in (None, need, need // 2, need // 5, 256):
            try:
                if size is not None:
                    buf = torch.full((size + 512,), 255, dtype=torch.uint8, device=DEV)[:size]
                    ann.ann_set_workspace(buf)
                out, lse = f(*args)
                torch.cuda.synchronize()
            finally:
                ann.ann_set_workspace(None)
            close(out.cpu(), want[0], o, (f.__name__, size))
            close(lse.cpu(), want[1], s, (f.__name__, size))


def test_other_streams_and_given_outputs():
    args, _ = inputs()
    want, lse = ann.ann_chunk_attention(*args)
    sargs, _ = shared_inputs()
    swant, slse = ann.ann_shared_attention(*sargs)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        a = ann.ann_chunk_attention(*args)
        b = ann.ann_shared_attention(*sargs)
    out, l = torch.empty_like(want), torch.empty_like(lse)
    stream.synchronize()
    c = ann.ann_chunk_attention(*args, out=out, lse=l, stream=stream)
    stream.synchronize()
    assert c[0] is out and all(torch.equal(x, y) for x, y in ((a[0], want), (a[1], lse), (b[0], swant), (b[1], slse), (out, want), (l, lse)))


def test_graphs():
    """The three operators from one graph, replayed with other lengths, starts and contents between eager work."""
    heads, Hq, d, page, B = 2, 8, 64, 16, 3
    table = torch.arange(3 * 40, dtype=torch.int32, device=DEV).view(3, 40)
    table[1:, :10] = table[0, :10]                        # 160 slots in common
    k, v = (torch.randn(120, heads, page, d, device=DEV).to(BF16) for _ in range(2))
    x, one = torch.randn(20, Hq + 2 * heads, d, device=DEV).to(BF16), torch.randn(B, Hq + 2 * heads, d, device=DEV).to(BF16)
    starts, lengths = M.ints([0, 5, 5, 20]).to(DEV), M.ints([300, 160, 400]).to(DEV)
    ones, after = M.ints([0, 1, 2, 3]).to(DEV), lengths + 1
    groups, common = M.ints([0, 3]).to(DEV), M.ints([160]).to(DEV)
    frequencies, _ = ann.ann_rotation_frequencies(64, device=DEV)

    def run():
        q = ann.ann_rotate_append(x, starts, lengths, table, frequencies, k, v)
        a = ann.ann_chunk_attention(q, k, v, table, lengths, starts, max_length=640)
        q1 = ann.ann_rotate_append(one, ones, after, table, frequencies, k, v)
        return (q, *a, q1, *ann.ann_shared_attention(q1, k, v, table, after, groups, common, max_shared=160, max_own=480))
    for _ in range(2):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    cases = [([0, 5, 5, 20], [300, 160, 400]), ([0, 0, 20, 20], [170, 180, 161]), ([0, 1, 2, 3], [600, 200, 639]), ([0, 7, 14, 20], [167, 500, 333])]
    for i, (s, n) in enumerate(cases * 2):
        starts.copy_(M.ints(s)), lengths.copy_(M.ints(n)), after.copy_(M.ints(n) + 1)
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(i)).to(BF16))
        saved = k.clone(), v.clone()
        for o in outs:
            o.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        k.copy_(saved[0]), v.copy_(saved[1])
        want = run()
        torch.cuda.synchronize()
        last = s[-1]
        for j, (y, z) in enumerate(zip(got, want)):
            n_rows = last if j < 3 else B
            assert torch.equal(y[:n_rows], z[:n_rows]), (i, j)
        assert all(bool((o[last:] == 3.0).all()) for o in got[:3])


def test_calls_that_share_the_workspace_in_turn():
    """Calls of different sizes one after the other on one stream."""
    a, pa = inputs(seed=3)
    b, pb = shared_inputs(seed=4)
    first = ann.ann_chunk_attention(*a), ann.ann_shared_attention(*b)
    for _ in range(20):
        x, y = ann.ann_chunk_attention(*a), ann.ann_shared_attention(*b)
    assert all(torch.equal(p, q) for p, q in zip(x + y, first[0] + first[1]))


def test_no_tokens():
    k = torch.zeros(4, 2, 16, 64, device=DEV)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    q = torch.zeros(0, 4, 64, device=DEV)
    out, lse = ann.ann_chunk_attention(q, k, k, i(1, 2), i(1), i(2))
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    out, lse = ann.ann_shared_attention(q, k, k, i(0, 2), i(0), i(2), i(1))
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    assert ann.ann_rotate_append(torch.zeros(0, 8, 64, device=DEV), i(2), i(1), i(1, 2), None, k, k).shape == (0, 4, 64)


def test_refusals_of_the_binding():
    (q, k, v, table, lengths, starts), _ = inputs()
    for bad in (dict(q=q.float()), dict(q=q[0]), dict(table=table.long()), dict(table=table[:2]), dict(lengths=lengths[:3]), dict(starts=starts[:4]), dict(k=k[:, :1]), dict(starts=starts.cpu()),
                dict(window=-1), dict(max_length=10 ** 9), dict(max_length=0), dict(scale=math.inf), dict(window=2 ** 40), dict(out=q)):
        kw = dict(dict(q=q, k=k, v=v, table=table, lengths=lengths, starts=starts), **bad)
        pos = [kw.pop(n) for n in ("q", "k", "v", "table", "lengths", "starts")]
        if "out" in kw:
            kw["out"] = kw["out"].float()
        with pytest.raises((ValueError, ann.AnnError)):
            ann.ann_chunk_attention(*pos, **kw)
    args, _ = shared_inputs()
    for i, bad in ((5, args[5][:2]), (6, args[6].long()), (4, args[4][:4]), (3, args[3].t())):
        with pytest.raises((ValueError, ann.AnnError)):
            ann.ann_shared_attention(*args[:i], bad, *args[i + 1:])
    for kw in (dict(max_shared=-1), dict(max_own=0), dict(max_own=10 ** 9), dict(max_shared=2 ** 40)):
        with pytest.raises((ValueError, ann.AnnError)):
            ann.ann_shared_attention(*args, **kw)
    x = torch.zeros(4, 8, 64, dtype=BF16, device=DEV)
    f, _ = ann.ann_rotation_frequencies(64, device=DEV)
    for kw in (dict(frequencies=f.float()), dict(frequencies=f.cpu()), dict(frequencies=torch.zeros(33, dtype=torch.float64, device=DEV)), dict(positions=starts), dict(amplitude=math.nan), dict(x=x[:, :4]),
               dict(starts=starts[:3])):
        a = dict(dict(x=x, starts=starts, frequencies=f, positions=None, amplitude=1.0), **kw)
        with pytest.raises((ValueError, ann.AnnError)):
            ann.ann_rotate_append(a["x"], a["starts"], lengths, table, a["frequencies"], k, v, positions=a["positions"], amplitude=a["amplitude"])


def test_the_marshalled_and_the_python_way_agree(monkeypatch):
    from paper_2505_12065_amd import binding
    args, _ = inputs()
    sargs, _ = shared_inputs()
    fast = ann.ann_chunk_attention(*args, window=40, scale=0.2), ann.ann_shared_attention(*sargs, max_own=200)
    monkeypatch.setattr(binding, "_marshal", None)
    slow = ann.ann_chunk_attention(*args, window=40, scale=0.2), ann.ann_shared_attention(*sargs, max_own=200)
    assert all(torch.equal(x, y) for x, y in zip(fast[0] + fast[1], slow[0] + slow[1]))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_append_more_requests_than_lanes(dtype):
    append(dtype, [(5 * b) % 4 for b in range(4200)], [b % 20 for b in range(4200)], 2, 1, 16, 8, 16)
