"""The operators over a paged cache and the rules on logits against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import decode as D                                        # (beside this file)
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
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    finite = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), finite) and np.array_equal(got[~finite], want[~finite], equal_nan=True), what
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want)[finite] - np.broadcast_to(bound, want.shape)[finite]
    assert off.size == 0 or off.max() <= 0, (what, off.max(), np.abs(got - want)[finite].max())


# ---- attention ---------------------------------------------------------------------------------

def attend(dtype, lengths, Hq, heads, d, page, window=0, mass=False, layout="heads", seed=1, q_scale=1.0, scale=None, max_length=None, edit=None, which=True):
    k, v, table = D.paged(lengths, page, heads, d, dtype, seed, layout)
    q = D.rows(len(lengths), Hq, d, dtype=dtype, seed=seed + 7, scale=q_scale)
    lens = torch.tensor(lengths, dtype=torch.int32)
    if edit:
        q, k, v, table, lens = edit(q, k, v, table, lens)
    scale = d ** -0.5 if scale is None else scale
    want = D.attention(q, k, v, table, [min(n, max_length or n) for n in lens.tolist()], scale, window)
    before = torch.rand(len(lengths), heads, table.shape[1] * page + 3, generator=torch.Generator().manual_seed(seed)) if mass else None
    m = dev(before)
    args = dev(q), dev(k), dev(v), dev(table), dev(lens)
    out, lse = ann.ann_paged_attention(*args, scale=scale, window=window, max_length=max_length, mass=m)
    bounds = D.attention_bounds(*want, lens.tolist(), d, dtype, Hq // heads)
    if which:
        close(out, want[0], bounds[0], "out")
    else:
        finite = np.isfinite(want[0])
        assert np.array_equal(torch.isfinite(out).cpu().numpy(), finite) and not finite.all()
        close(torch.where(torch.isfinite(out), out, 0), np.where(finite, want[0], 0), np.where(finite, bounds[0], 0), "out")
    close(lse, want[1], bounds[1], "lse")
    if mass:
        n_slots = table.shape[1] * page
        total = before.double().numpy()
        total[..., :n_slots] += want[2]
        allowed = np.zeros_like(total)
        allowed[..., :n_slots] = bounds[2] + D.U * total[..., :n_slots]
        close(m, total, allowed, "mass")
        untouched = total == before.double().numpy()
        assert np.array_equal(m.cpu().numpy()[untouched], before.numpy()[untouched])
    again, lse2 = ann.ann_paged_attention(*args, scale=scale, window=window, max_length=max_length)
    if not mass:
        assert torch.equal(again.view(torch.uint8), out.view(torch.uint8)) and torch.equal(lse2.view(torch.uint8), lse.view(torch.uint8))
    return out


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 300]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("Hq,heads,d,page", [(8, 2, 128, 16), (3, 3, 64, 32), (7, 1, 80, 8), (16, 1, 256, 64), (5, 5, 8, 16), (34, 2, 96, 16),
                                             (12, 4, 72, 4), (24, 1, 136, 128), (6, 2, 200, 2), (40, 1, 48, 1), (4, 2, 128, 1024)])
def test_attention_lengths_and_heads(dtype, Hq, heads, d, page):
    attend(dtype, EDGES, Hq, heads, d, page, seed=d + page)
    attend(dtype, EDGES, Hq, heads, d, page, mass=True, layout="slots", seed=d + page + 1)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("window", [1, 2, 16, 17, 100, 128, 300, 5000])
def test_attention_window(dtype, window):
    attend(dtype, EDGES + [1000], 8, 2, 64, 16, window=window, mass=True, seed=window)
    attend(dtype, EDGES + [1000], 8, 2, 128, 2, window=window, mass=True, seed=window + 1)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("lengths,Hq,heads,d,page", [([5000], 8, 1, 128, 16), ([9000, 100, 4097], 14, 2, 64, 32), ([20_001], 4, 4, 80, 64),
                                                     ([3001, 0, 7], 12, 2, 256, 16), ([2500] * 40, 4, 2, 128, 16), ([40_000], 20, 1, 16, 8)])
def test_attention_long(dtype, lengths, Hq, heads, d, page):
    attend(dtype, lengths, Hq, heads, d, page, seed=3)
    attend(dtype, lengths, Hq, heads, d, page, seed=3, mass=True, window=lengths[0] // 2, layout="slots")


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("Hq,heads,d,page,longest,window", [
    (32, 32, 64, 16, 1020, 0), (128, 32, 16, 8, 1024, 0), (64, 32, 128, 32, 1025, 0), (64, 32, 96, 16, 1020, 333),
    (128, 32, 8, 64, 4030, 0), (32, 32, 8, 16, 4096, 0), (64, 32, 16, 16, 4200, 0)])
def test_attention_contexts_of_one_part_in_a_large_batch(dtype, Hq, heads, d, page, longest, window):
    """A cache head for every compute unit: contexts in one part up to some length, and weights added from scores that stay on the chip."""
    lengths = [longest, 0, 1, longest - 1, 64, 65, longest // 2, 300]
    for mass in (False, True):
        attend(dtype, lengths, Hq, heads, d, page, window, mass)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("Hq,heads,d", [(20, 1, 64), (40, 2, 128), (18, 1, 256), (34, 2, 104), (65, 1, 128), (6, 2, 64), (16, 1, 128), (8, 2, 256), (6, 3, 72), (4, 1, 200)])
def test_attention_tiles_of_heads_and_wide_tables(dtype, wide, Hq, heads, d):
    """More query heads than a tile has, and tables that are wide enough for 256 MiB of keys and values, of which only a little is there: caches of that size
    are read past the last cache, and a context has the most parts that there can be."""
    def edit(q, k, v, table, lens):
        if wide:
            width = (300 << 20) // (2 * len(lens) * heads * d * k.element_size() * 16)
            table = torch.nn.functional.pad(table, (0, width - table.shape[1]), value=-1)
        return q, k, v, table, lens
    attend(dtype, [900, 0, 33, 4097], Hq, heads, d, 16, seed=d + Hq, edit=edit)
    attend(dtype, [900, 0, 33, 4097], Hq, heads, d, 16, seed=d + Hq + 1, edit=edit, mass=True, window=700, layout="slots")


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_attention_large_scores(dtype):
    """Exponents that overflow where no maximum is taken off, maxima that come late, and a negative scale."""
    attend(dtype, [700, 33, 129], 6, 2, 128, 16, q_scale=20.0, scale=1.0, seed=5, mass=True)
    attend(dtype, [700, 33, 129], 6, 2, 128, 16, q_scale=20.0, scale=-0.3, seed=6)

    def late(q, k, v, table, lens):                       # the last slot of every request points where the queries do
        for b, n in enumerate(lens.tolist()):
            k[table[b, (n - 1) // 16], :, (n - 1) % 16] = q[b, ::3] * 4
        return q, k, v, table, lens
    attend(dtype, [700, 33, 129, 2000], 6, 2, 128, 16, seed=8, mass=True, edit=late)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("below", [10.0, 16.0, 16.6, 17.5, 20.0, 24.0])
def test_attention_weight_in_many_small_slots(dtype, below):
    """One slot has the largest score and a value of zero; all of the output comes from thousands whose weight is e^-below of its."""
    n, d = 20_000, 64

    def edit(q, k, v, table, lens):
        q[:] = 0
        q[..., 0] = 4.0
        k[:] = 0
        v[:] = 1.0
        at = table[0, 3000 // 16], slice(None), 3000 % 16
        k[at] = 0
        k[(*at, 0)] = below / 4
        v[at] = 0
        return q, k, v, table, lens
    attend(dtype, [n], 4, 2, d, 16, scale=1.0, seed=12, mass=True, edit=edit)


@pytest.mark.parametrize("page", [4, 16])
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_attention_empty_and_shared_pages(dtype, page):
    """Pages that are none leave out their slots, at the start, inside, at the end, or all; lengths are cut to what there is."""
    def edit(q, k, v, table, lens):
        pages = k.shape[0]
        table[0, 0] = -1
        table[1, 1] = pages
        table[2, (700 - 1) // page] = 2 ** 31 - 1
        table[3, :] = -5
        table[5] = table[4]                               # the same cache, other queries
        lens[4], lens[6] = 2 ** 31 - 1, -3
        used = -(-700 // page)
        for c in (k, v):                                  # what a length beyond the table's own reaches now
            c[table[4, used - 1].long()] = 1.0
        return q, k, v, table, lens
    attend(dtype, [700, 700, 700, 700, 700, 650, 300], 4, 2, 64, page, seed=9, mass=True, edit=edit)
    attend(dtype, [700, 500, 20], 4, 2, 64, page, seed=10, max_length=450)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_attention_infinities_and_nan(dtype):
    """Where the formula gives what is not finite, so does the kernel (an infinite value may come out as NaN: a weight is multiplied in
    two parts); for that head and request alone."""
    def edit(q, k, v, table, lens):
        v[table[0, 1], 0, 3, 5] = math.inf
        v[table[1, 0], 1, 0, 0] = math.nan
        k[table[2, 2], 0, 1, :] = math.nan
        q[3, 1] = math.nan
        return q, k, v, table, lens
    attend(dtype, [200, 60, 90, 40, 50], 4, 2, 64, 16, seed=11, edit=edit, which=False)


def test_attention_again_and_again():
    """Calls of different shapes between each other leave nothing behind: every call of a shape gives the same bits."""
    shapes = [([1500], 32, 8, 128), ([100, 0, 700, 33], 8, 2, 64), ([9], 40, 1, 64), ([700, 200], 40, 2, 128), ([60] * 20, 6, 3, 256), ([3000] * 30, 8, 2, 64)]
    calls, want = [], []
    for lengths, Hq, heads, d in shapes:
        k, v, table = (dev(t) for t in D.paged(lengths, 16, heads, d, BF16, 5, unused=0.0))
        q, lens = dev(D.rows(len(lengths), Hq, d, dtype=BF16, seed=2)), torch.tensor(lengths, dtype=torch.int32, device=DEV)
        slots = table.shape[1] * 16

        def call(q=q, k=k, v=v, table=table, lens=lens, heads=heads, slots=slots, mass=False):
            m = torch.zeros(len(lens), heads, slots, device=DEV) if mass else None
            return (*ann.ann_paged_attention(q, k, v, table, lens, mass=m), *([m] if mass else []))
        calls += [call, lambda call=call: call(mass=True)]
    want = [c() for c in calls]
    for a, b in zip(want[::2], want[1::2]):
        torch.testing.assert_close(a[0].float(), b[0].float(), rtol=1e-2, atol=1e-3)
    for _ in range(20):
        got = [c() for c in calls]
        assert all(torch.equal(x, y) for a, b in zip(got, want) for x, y in zip(a, b))


def test_attention_inputs_with_strides():
    """Queries that are part of a larger tensor, keys and values side by side in one, a single request."""
    lengths = [77, 300, 5]
    k, v, table = D.paged(lengths, 16, 2, 64, BF16, 2, unused=0.0)
    both = torch.empty(k.shape[0], 2, 16, 2, 64, dtype=BF16, device=DEV)     # [pages, (k, v), slots, heads, d]
    both[:, 0], both[:, 1] = k.transpose(1, 2).to(DEV), v.transpose(1, 2).to(DEV)
    qkv = D.rows(3, 10, 64, dtype=BF16, seed=4).to(DEV)
    lens = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    kk, vv = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    for b in (slice(0, 3), slice(1, 2)):
        out, lse = ann.ann_paged_attention(qkv[b, 3:7], kk, vv, dev(table)[b], lens[b])
        plain, plain_lse = ann.ann_paged_attention(qkv[b, 3:7].contiguous(), dev(k), dev(v), dev(table)[b], lens[b])
        assert torch.equal(out, plain) and torch.equal(lse, plain_lse)


def test_attention_offsets_beyond_32_bits():
    pages, stride = 4, 1_100_000_000                      # elements from page to page: 8.8 GB in all
    store = torch.zeros(pages * stride, dtype=BF16, device=DEV)
    k = store.as_strided((pages, 2, 16, 64), (stride, 1024, 64, 1))
    v = store.as_strided((pages, 2, 16, 64), (stride, 1024, 64, 1), 4096)
    small_k, small_v = D.rows(pages, 2, 16, 64, dtype=BF16, seed=1).to(DEV), D.rows(pages, 2, 16, 64, dtype=BF16, seed=2).to(DEV)
    k.copy_(small_k), v.copy_(small_v)
    q = D.rows(1, 4, 64, dtype=BF16, seed=3).to(DEV)
    table = torch.tensor([[3, 1, 2]], dtype=torch.int32, device=DEV)
    lens = torch.tensor([41], dtype=torch.int32, device=DEV)
    for a, b in zip(ann.ann_paged_attention(q, k, v, table, lens), ann.ann_paged_attention(q, small_k, small_v, table, lens)):
        assert torch.equal(a, b)
    mass = torch.rand(1, 2, 48, device=DEV)
    new = torch.tensor([[0]], dtype=torch.int32, device=DEV)
    for a, b in zip(ann.ann_cache_evict(k, v, table, lens, mass, new, 9), ann.ann_cache_evict(small_k, small_v, table, lens, mass, new, 9)):
        assert torch.equal(a, b)
    assert torch.equal(k, small_k) and torch.equal(v, small_v)
    qkv, w = D.rows(2, 8, 64, dtype=BF16, seed=4).to(DEV), torch.ones(64, dtype=BF16, device=DEV)
    at = torch.tensor([63, 5], dtype=torch.int32, device=DEV)
    turn = torch.rand(64, 64, device=DEV)
    for kk, vv in ((k, v), (small_k, small_v)):
        ann.ann_qk_norm_rotate(qkv, w, w, at, turn, at, kk, vv)
    assert torch.equal(k, small_k) and torch.equal(v, small_v)


def test_attention_workspace_of_any_size():
    """As much as is wanted, as much as one request needs, and too little."""
    lengths = [3000, 10, 2000, 0, 2999]
    k, v, table = D.paged(lengths, 16, 2, 64, F16, 2)
    args = dev(D.rows(5, 8, 64, dtype=F16, seed=4)), dev(k), dev(v), dev(table), torch.tensor(lengths, dtype=torch.int32, device=DEV)
    slots = table.shape[1] * 16
    for with_mass in (False, True):
        def run():
            m = torch.zeros(5, 2, slots, device=DEV) if with_mass else None
            got = ann.ann_paged_attention(*args, mass=m)
            return (*got, m) if with_mass else got
        want = run()
        whole = ann.ann_paged_attention_workspace_bytes(5, 8, 2, 64, F16, slots, with_mass)
        one = ann.ann_paged_attention_workspace_bytes(1, 8, 2, 64, F16, slots, with_mass)
        assert 0 < one <= whole
        for size in (whole, max(one, whole // 2), one):
            buffer = torch.empty(size, dtype=torch.uint8, device=DEV)
            ann.ann_set_workspace(buffer)
            try:
                for a, b in zip(run(), want):
                    torch.testing.assert_close(a, b, rtol=1e-2, atol=1e-3)      # (other parts, other roundings)
            finally:
                torch.cuda.synchronize()
                ann.ann_set_workspace(None)


# ---- norms, rotation, write into the cache ------------------------------------------------------

@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,heads,d,rot,page,layout", [(1, 4, 1, 64, 64, 16, "heads"), (7, 8, 2, 128, 128, 16, "slots"), (33, 3, 3, 80, 32, 8, "heads"),
                                                          (5, 40, 5, 96, 96, 1, "heads"), (300, 2, 1, 256, 64, 64, "slots"), (9, 5, 1, 8, 0, 2, "heads"),
                                                          (4, 28, 4, 72, 48, 32, "slots"), (3, 9, 3, 248, 240, 16, "heads"), (65, 1, 1, 16, 16, 128, "heads")])
def test_rotate(dtype, interleaved, T, Hq, heads, d, rot, page, layout):
    seed = T + d
    g = torch.Generator().manual_seed(seed)
    pages = -(-T // page) + 2
    qkv = D.rows(T, Hq + 2 * heads, d, dtype=dtype, seed=seed, scale=3.0)
    if T > 2:
        qkv[1, 0] = 0.0                                   # a row of zeros: nothing to divide by but eps
        qkv[2] *= 1e-3
    wq, wk = D.rows(d, dtype=dtype, seed=1), D.rows(d, dtype=dtype, seed=2)
    turn = torch.randn(50, rot, generator=g)
    positions = torch.randint(0, 50, (T,), generator=g, dtype=torch.int32)
    slots = torch.randperm(pages * page, generator=g)[:T].to(torch.int32)
    if T > 4:
        positions[3], positions[4], slots[0], slots[1] = -1, 50, -7, pages * page
    shape = (pages, heads, page, d) if layout == "heads" else (pages, page, heads, d)
    k, v = torch.full(shape, 7.0, dtype=dtype), torch.full(shape, -5.0, dtype=dtype)
    k, v = (k, v) if layout == "heads" else (k.transpose(1, 2), v.transpose(1, 2))
    q64, k64, v64, size = D.rotate(qkv, Hq, heads, wq, wk, 1e-5, positions, turn, interleaved)
    dk, dv = dev(k), dev(v)
    q = ann.ann_qk_norm_rotate(dev(qkv), dev(wq), dev(wk), dev(positions), dev(turn), dev(slots), dk, dv, eps=1e-5, interleaved=interleaved)
    # the sum of d squares, its mean, root and quotient, the two products; then two products and their sum
    rel = (d + 16) * D.U
    bound = lambda x, s: (rel * s + D.HALF_ULP[dtype] * (1 + 2.0 ** -7) * x.abs() + D.TINY[dtype] + 1e-37).numpy()  # noqa: E731
    close(q, q64.numpy(), bound(q64, size[:, :Hq]), "q")
    ek, ev, bk = k.double(), v.double(), torch.zeros(k.shape, dtype=torch.float64)
    for t in range(T):
        s, p = int(slots[t]), int(positions[t])
        if 0 <= s < pages * page and 0 <= p < 50:
            ek[s // page, :, s % page], ev[s // page, :, s % page] = k64[t], v64[t]
            bk[s // page, :, s % page] = torch.from_numpy(bound(k64[t], size[t, Hq:]))
    close(dk, ek.numpy(), bk.numpy(), "keys")
    assert torch.equal(dv.cpu().double(), ev)


@pytest.mark.parametrize("dtype,interleaved", [(F16, False), (BF16, True), (F32, False)])
@pytest.mark.parametrize("Hq,heads,d,rot,layout", [(20, 1, 64, 64, "heads"), (40, 4, 56, 32, "slots"), (60, 3, 128, 16, "heads"), (12, 4, 256, 32, "heads"),
                                                   (70, 2, 136, 48, "slots"), (36, 6, 80, 80, "heads"), (130, 1, 16, 16, "heads")])
def test_rotate_many_tokens(dtype, interleaved, Hq, heads, d, rot, layout):
    """Groups of lanes that take two, three or four heads of a token, the last of which may have none left."""
    test_rotate(dtype, interleaved, 520, Hq, heads, d, rot, 16, layout)


def test_rotate_part_of_a_larger_tensor_and_non_finite_values():
    T, Hq, heads, d = 6, 4, 2, 64
    big = D.rows(T, 2, Hq + 2 * heads, 96, dtype=BF16, seed=1)
    big[0, 1, 0, 3], big[1, 1, 1, 40], big[2, 1, Hq + 2 * heads - 1, 0] = math.nan, math.inf, math.nan
    w, turn = torch.ones(d, dtype=BF16), torch.randn(10, 32, generator=torch.Generator().manual_seed(1))
    at = torch.arange(T, dtype=torch.int32)
    answers = []
    for qkv in (dev(big)[:, 1, :, 16:80], dev(big[:, 1, :, 16:80].contiguous())):
        k, v = torch.zeros(1, heads, 16, d, dtype=BF16, device=DEV), torch.zeros(1, heads, 16, d, dtype=BF16, device=DEV)
        answers.append((ann.ann_qk_norm_rotate(qkv, dev(w), dev(w), dev(at), dev(turn), dev(at), k, v), k, v))
    for a, b in zip(*answers):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    q = answers[0][0].float().cpu()
    assert torch.isfinite(q[2:]).all() and torch.isfinite(q[0]).all()       # (0, 0, 3) lies outside the part
    assert torch.isnan(q[1, 1]).any() and torch.isfinite(q[1, 0]).all()


# ---- eviction -----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F16, 64), (F32, 72), (F32, 256), (BF16, 8)])
@pytest.mark.parametrize("lengths,budget,first,recent,page,layout", [
    ([0, 1, 63, 64, 65, 200], 64, 0, 0, 16, "heads"), ([300, 5, 299], 100, 4, 32, 8, "slots"), ([1000], 1, 0, 0, 16, "heads"),
    ([1000, 70], 60, 60, 0, 4, "heads"), ([1000, 61], 60, 0, 60, 32, "slots"), ([5000, 4999, 77], 2000, 16, 500, 64, "heads"),
    ([2100, 2000], 33, 1, 1, 1, "heads"), ([20_000], 1500, 0, 7, 128, "heads"),
    ([40_000, 33_000], 3000, 5, 100, 64, "slots")])
def test_evict(dtype, d, lengths, budget, first, recent, page, layout):
    heads, seed = 3, budget + d
    g = torch.Generator().manual_seed(seed)
    B, new_width = len(lengths), -(-budget // page) + 1
    k, v, table = D.paged(lengths, page, heads, d, dtype, seed, layout, unused=9.0, spare=B * new_width + 2)
    free = [p for p in range(k.shape[0]) if p not in set(table.flatten().tolist())]
    new_table = torch.tensor(free[:B * new_width], dtype=torch.int32).view(B, new_width)
    slots = table.shape[1] * page
    mass = torch.randn(B, heads, slots, generator=g).pow(3)
    mass[:, 1] = (mass[:, 1] * 2).round() / 2             # equal ones by the hundred, 0 and -0 among them
    mass[:, 2, ::5] = 0.25
    mass[0, 0, 3::7], mass[0, 0, 4::11], mass[0, 2, 2::9] = math.nan, math.inf, -math.inf
    mass[-1, 2] = math.nan
    lens = torch.tensor(lengths, dtype=torch.int32)
    want, new = D.evict(mass.numpy(), lengths, slots, budget, first, recent)
    dk, dv = dev(k), dev(v)
    kept, got_new, got_mass = ann.ann_cache_evict(dk, dv, dev(table), dev(lens), dev(mass), dev(new_table), budget, first=first, recent=recent)
    assert np.array_equal(kept.cpu().numpy(), want) and np.array_equal(got_new.cpu().numpy(), new)
    ek, ev, em = k.clone(), v.clone(), torch.zeros(B, heads, new_width * page)
    for b in range(B):
        i = np.arange(new[b])
        for h in range(heads):
            j = want[b, h, :new[b]]
            em[b, h, :new[b]] = mass[b, h, j]
            for e, s in ((ek, k), (ev, v)):
                e[new_table[b, i // page].long(), h, i % page] = s[table[b, j // page].long(), h, j % page]
    assert torch.equal(dk.cpu(), ek) and torch.equal(dv.cpu(), ev)
    assert np.array_equal(got_mass.cpu().numpy(), em.numpy(), equal_nan=True)


def test_evict_empty_pages_and_lengths_out_of_range():
    """Rows of a page that is none are zeros, rows that would go to one are dropped; lengths are cut to the table."""
    heads, d, page = 2, 64, 16
    k, v, table = D.paged([64, 64, 64], page, heads, d, BF16, 3, unused=1.0, spare=7)
    free = [p for p in range(k.shape[0]) if p not in set(table.flatten().tolist())]
    new_table = torch.tensor([free[0:2], [free[2], -1], [free[4], k.shape[0]]], dtype=torch.int32)
    table[0, 1] = -1
    mass = torch.arange(64).float().expand(3, heads, 64).contiguous()
    mass[0, :, 16:32] += 100                              # the slots of the page that is none are wanted
    lens = torch.tensor([2 ** 31 - 1, 64, -1], dtype=torch.int32)
    dk, dv = dev(k), dev(v)
    kept, new, _ = ann.ann_cache_evict(dk, dv, dev(table), dev(lens), dev(mass), dev(new_table), 20)
    assert new.tolist() == [20, 20, 0]
    assert kept[0, 0].tolist() == list(range(16, 32)) + [60, 61, 62, 63] and kept[1, 1].tolist() == list(range(44, 64))
    assert (kept[2] == -1).all()
    ek, ev = k.clone(), v.clone()
    for e, s in ((ek, k), (ev, v)):
        e[free[0]] = 0
        e[free[1], :, :4] = s[table[0, 3], :, 12:]
        e[free[2]] = torch.cat([s[table[1, 2], :, 12:], s[table[1, 3], :, :12]], 1)
    assert torch.equal(dk.cpu(), ek) and torch.equal(dv.cpu(), ev)


# ---- rules on logits ------------------------------------------------------------------------------

def rule_inputs(dtype, B, V, T, K, M, seed):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(B, V, generator=g) * 4).to(dtype)
    x[:, ::17] = 0.0
    if V > 40:
        x[0, 5], x[0, 6], x[0, 7] = math.inf, -math.inf, math.nan
    tokens = (V * torch.rand(B, T, generator=g) ** 3).to(torch.int32)
    if T > 10:
        tokens[:, 3], tokens[:, 4], tokens[:, 5], tokens[:, 6] = -1, V, V - 1, 0
        tokens[:, 7:9] = 6
    lengths = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32)
    lengths[0], lengths[B - 1] = T + 9, -2 if B > 1 else T
    prompts = (lengths.float() * torch.rand(B, generator=g)).to(torch.int32)
    if B > 2:
        prompts[1], prompts[2] = 10 * T, -4
    params = [1 + torch.rand(B, generator=g), torch.randn(B, generator=g), torch.randn(B, generator=g) * 0.2]
    bias = masks = rows = None
    if K:
        bias = (torch.randint(-2, V + 2, (B, K), generator=g, dtype=torch.int32), torch.randn(B, K, generator=g) * 6)
        bias[0][:, -1] = bias[0][:, 0]                    # one token twice: the last counts
        bias[1][0, 0] = -math.inf
    if M:
        masks = torch.randint(-2 ** 31, 2 ** 31, (M, (V + 31) // 32), generator=g, dtype=torch.int64).to(torch.int32)
        masks[0] = 0                                      # nothing is allowed
        rows = torch.randint(-1, M + 1, (B,), generator=g, dtype=torch.int32)
        rows[0] = 0 if B > 1 else M - 1
    return x, tokens, lengths, prompts, params, bias, masks, rows


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("B,V,T,K,M", [(1, 1, 1, 1, 1), (3, 7, 20, 3, 2), (4, 32, 0, 0, 3), (5, 33, 50, 40, 0), (2, 4096, 300, 17, 2), (3, 4097, 1000, 0, 4),
                                       (2, 8191, 64, 300, 1), (7, 20_011, 5000, 33, 7), (1, 100_003, 30_000, 4096, 1), (33, 1000, 129, 1, 2)])
def test_rules(dtype, B, V, T, K, M):
    x, tokens, lengths, prompts, params, bias, masks, rows = rule_inputs(dtype, B, V, T, K, M, V + T)
    want, size = D.rules(x, tokens, lengths, prompts, *params, bias, masks, rows)
    kw = dict(bias_tokens=dev(bias[0]) if K else None, bias_values=dev(bias[1]) if K else None, masks=dev(masks), mask_rows=dev(rows))
    args = [dev(t) for t in (tokens, lengths, prompts, *params)]
    got = ann.ann_logit_rules(dev(x), *args, **kw)
    with np.errstate(all="ignore"):                       # at most six operations on what was added up, and one rounding
        bound = np.where(np.isfinite(want), 6 * D.U * size + D.HALF_ULP[dtype] * (1 + 2.0 ** -7) * np.abs(want), 0) + D.TINY[dtype] + 1e-37
    if dtype == F16:
        want = np.where(np.abs(want) > 65519, np.sign(want) * np.inf, want)
    close(got, want, bound, "out")
    # part of a larger tensor, rows that start anywhere, in place
    wide = torch.full((B, V + 5), 3.0, dtype=dtype, device=DEV)
    wide[:, 3:V + 3] = dev(x)
    part = wide[:, 3:V + 3]
    assert ann.ann_logit_rules(part, *args, out=part, **kw) is part
    nan = torch.isnan(got)
    assert torch.equal(torch.where(nan, 0, part), torch.where(nan, 0, got)) and torch.equal(torch.isnan(part), nan)
    assert (wide[:, :3] == 3).all() and (wide[:, V + 3:] == 3).all()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("B,V,T,K,M", [(300, 16_391, 40, 3, 5), (130, 16_500, 300, 0, 2), (70, 16_380, 9, 20, 0), (513, 2049, 5, 1, 3),
                                       (2, 9000, 262_143, 4096, 1), (2, 9000, 262_144, 4096, 1), (1, 40, 300_000, 9, 1)])
def test_rules_many_rows_and_long_histories(dtype, B, V, T, K, M):
    """Every number of logits that a lane takes, and counts that no longer share a word with a bias."""
    test_rules(dtype, B, V, T, K, M)


# ---- streams and graphs ----------------------------------------------------------------------------

def all_four(stream=None):
    """One pass of the four, on inputs of its own: (call, outputs)."""
    lengths, heads, d, page, B = [300, 40, 511, 64], 2, 64, 16, 4
    k, v, table = (dev(t) for t in D.paged(lengths, page, heads, d, BF16, 21, unused=0.0, spare=20))
    free = torch.tensor([p for p in range(k.shape[0]) if p not in set(table.flatten().tolist())], dtype=torch.int32, device=DEV)
    new_table = free[:16].view(4, 4).contiguous()
    lens = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    qkv, w = dev(D.rows(B, 8 + 2 * heads, d, dtype=BF16, seed=5)), torch.ones(d, dtype=BF16, device=DEV)
    turn = torch.randn(600, 64, generator=torch.Generator().manual_seed(4)).to(DEV)
    slots = table.gather(1, ((lens - 1) // page).long()[:, None])[:, 0] * page + (lens - 1) % page
    x = rule_inputs(F32, B, 5000, 100, 5, 2, 3)
    rule = [dev(t) for t in (x[1], x[2], x[3], *x[4])]
    logits, bias, masks, rows = dev(x[0]), [dev(t) for t in x[5]], dev(x[6]), dev(x[7])
    mass = torch.zeros(B, heads, table.shape[1] * page, device=DEV)

    def call():
        mass.zero_()
        q = ann.ann_qk_norm_rotate(qkv, w, w, lens - 1, turn, slots.to(torch.int32), k, v, stream=stream)
        out, lse = ann.ann_paged_attention(q, k, v, table, lens, mass=mass, stream=stream)
        kept, new, new_mass = ann.ann_cache_evict(k, v, table, lens, mass, new_table, 48, first=2, recent=8, stream=stream)
        short, _ = ann.ann_paged_attention(q, k, v, new_table, new, stream=stream)
        y = ann.ann_logit_rules(logits, *rule, bias_tokens=bias[0], bias_values=bias[1], masks=masks, mask_rows=rows, stream=stream)
        return q, out, lse, kept, new, new_mass, short, torch.nan_to_num(y, nan=7.0)
    return call


def test_other_stream_and_graph():
    """The same on a stream of its own, and from a graph that is replayed between other work."""
    call = all_four()
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = all_four()()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call()
    for _ in range(4):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        torch.randn(1000, 1000, device=DEV).sum().item()


# ---- refusals ----------------------------------------------------------------------------------------

def test_refusals():
    k = torch.zeros(4, 2, 16, 64, dtype=BF16, device=DEV)
    q, table = torch.zeros(3, 4, 64, dtype=BF16, device=DEV), torch.zeros(3, 2, dtype=torch.int32, device=DEV)
    n, f = torch.zeros(3, dtype=torch.int32, device=DEV), torch.ones(3, device=DEV)
    at = lambda *a, **kw: (lambda: ann.ann_paged_attention(*a, **kw))  # noqa: E731
    ev = lambda *a, **kw: (lambda: ann.ann_cache_evict(*a, **kw))  # noqa: E731
    mass = torch.zeros(3, 2, 32, device=DEV)
    w, turn = torch.ones(64, dtype=BF16, device=DEV), torch.zeros(9, 64, device=DEV)
    qkv = torch.zeros(3, 8, 64, dtype=BF16, device=DEV)
    ro = lambda *a, **kw: (lambda: ann.ann_qk_norm_rotate(*a, **kw))  # noqa: E731
    x, tokens = torch.zeros(3, 40, device=DEV), torch.zeros(3, 5, dtype=torch.int32, device=DEV)
    ru = lambda *a, **kw: (lambda: ann.ann_logit_rules(*a, **kw))  # noqa: E731
    for call in (at(q.half(), k, k, table, n), at(q.cpu(), k, k, table, n), at(q, k, k[:3], table, n), at(q, k, k.half(), table, n),
                 at(q, k, k, table.long(), n), at(q, k, k, table[:2], n), at(q, k, k, table, n[:2]), at(q, k.transpose(2, 3), k.transpose(2, 3), table, n),
                 at(q, k, k, table, n, mass=mass[:, :1]), at(q, k, k, table, n, mass=mass.half()), at(q[..., :32], k, k, table, n),
                 ev(k, k, table, n, mass[:, :1], table, 8), ev(k, k, table, n, mass, table[:2], 8), ev(k, k, table, n.float(), mass, table, 8),
                 ro(qkv[:, :4], w, w, n, turn, n, k, k), ro(qkv, w.float(), w, n, turn, n, k, k), ro(qkv, w, w, n, turn.half(), n, k, k),
                 ro(qkv, w, w, n[:2], turn, n, k, k), ro(qkv[..., :32], w, w, n, turn, n, k, k), ro(qkv, w, w, n, turn, n, k, k, q=q[:2]),
                 ru(x.double(), tokens, n, n, f, f, f), ru(x, tokens[:2], n, n, f, f, f), ru(x, tokens, n, n, f[:2], f, f), ru(x.t(), tokens, n, n, f, f, f),
                 ru(x, tokens, n, n, f, f, f, bias_tokens=tokens), ru(x, tokens, n, n, f, f, f, masks=tokens[:, :2].contiguous()),
                 ru(x, tokens, n, n, f, f, f, masks=tokens, mask_rows=n)):
        with pytest.raises(ValueError):
            call()
    big = torch.zeros(4, 2, 24, 64, dtype=BF16, device=DEV)
    wide = torch.zeros(4, 2, 16, 264, dtype=BF16, device=DEV)
    for call in (at(q[:, :3], k, k, table, n), at(q, big, big, table, n), at(torch.zeros(3, 4, 264, dtype=BF16, device=DEV), wide, wide, table, n),
                 at(q, k, k, table, n, max_length=33), at(q, k, k, table, n, max_length=0), at(q, k, k, table, n, window=-1),
                 at(q, k, k, table, n, scale=math.nan), at(q, k, k, table, n, mass=mass[..., :31].contiguous()),
                 at(q[..., :60], k[..., :60], k[..., :60], table, n),
                 ev(k, k, table, n, mass, table, 0), ev(k, k, table, n, mass, table, 33), ev(k, k, table, n, mass, table, 8, first=5, recent=4),
                 ev(k, k, table, n, mass, table, 8, first=-1),
                 ro(qkv, w, w, n, turn[:, :24].contiguous(), n, k, k), ro(qkv, w, w, n, turn, n, k, k, eps=-1.0)):
        with pytest.raises(ann.AnnError):
            call()
    odd = torch.zeros(4 * 2 * 16 * 64 + 4, dtype=BF16, device=DEV)[4:].view(4, 2, 16, 64)
    for call in (at(q, odd, k, table, n), at(q, k[..., 4:60], k[..., 4:60], table, n)):
        with pytest.raises((ann.AnnError, ValueError)):
            call()


def test_nothing_to_do():
    k = torch.zeros(4, 2, 16, 64, dtype=BF16, device=DEV)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    f = torch.zeros(0, device=DEV)
    out, lse = ann.ann_paged_attention(torch.zeros(0, 4, 64, dtype=BF16, device=DEV), k, k, i(0, 3), i(0))
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    kept, new, mass = ann.ann_cache_evict(k, k, i(0, 3), i(0), torch.zeros(0, 2, 48, device=DEV), i(0, 2), 8)
    assert kept.shape == (0, 2, 8) and new.shape == (0,) and mass.shape == (0, 2, 32)
    w = torch.zeros(64, dtype=BF16, device=DEV)
    assert ann.ann_qk_norm_rotate(torch.zeros(0, 8, 64, dtype=BF16, device=DEV), w, w, i(0), torch.zeros(4, 64, device=DEV), i(0), k, k).shape == (0, 4, 64)
    assert ann.ann_logit_rules(torch.zeros(0, 40, device=DEV), i(0, 5), i(0), i(0), f, f, f).shape == (0, 40)


# ---- the binding's two halves -------------------------------------------------------------------------

def test_both_halves_of_the_binding(monkeypatch):
    """Native marshalling answers the usual calls with what the Python half gives, and leaves it the others."""
    lengths = [300, 40, 511]
    k, v, table = (dev(t) for t in D.paged(lengths, 16, 2, 64, BF16, 21, unused=0.0, spare=20))
    free = torch.tensor([p for p in range(k.shape[0]) if p not in set(table.flatten().tolist())], dtype=torch.int32, device=DEV)
    new_table, n = free[:12].view(3, 4).contiguous(), torch.tensor(lengths, dtype=torch.int32, device=DEV)
    qkv, w = dev(D.rows(3, 12, 64, dtype=BF16, seed=5)), torch.ones(64, dtype=BF16, device=DEV)
    turn, slots = torch.randn(600, 32, generator=torch.Generator().manual_seed(4)).to(DEV), free[12:15] * 16
    mass = torch.rand(3, 2, table.shape[1] * 16, device=DEV)
    x = rule_inputs(F32, 3, 500, 100, 5, 2, 3)
    x = [torch.nan_to_num(dev(x[0]), nan=3.0)] + [dev(t) for t in (x[1], x[2], x[3], *x[4], *x[5], x[6], x[7])]
    q = qkv[:, :8]
    rotate = lambda *a, **kw: (lambda: (ann.ann_qk_norm_rotate(qkv, w, w, n, turn, *a, k, v, **kw), k, v))  # noqa: E731
    attend = lambda *a, **kw: (lambda: ann.ann_paged_attention(q, k, v, *a, **kw))  # noqa: E731
    evict = lambda *a, **kw: (lambda: (*ann.ann_cache_evict(k, v, table, n, mass, *a, **kw), k, v))  # noqa: E731
    rules = lambda *a, **kw: (lambda: ann.ann_logit_rules(*a, **kw))  # noqa: E731

    def added():
        m = mass.clone()
        return (*ann.ann_paged_attention(q, k, v, table, n, mass=m), m)
    answered_calls = [
        rotate(slots), rotate(slots, eps=1e-3, interleaved=True), rotate(slots, eps=0), attend(table, n), attend(table, n, scale=0.3, window=7, max_length=400),
        attend(table, n, scale=1), added, evict(new_table, 48), evict(new_table, 30, first=3, recent=9), rules(*x[:7]),
        rules(*x[:7], bias_tokens=x[7], bias_values=x[8]), rules(*x[:7], masks=x[9], mask_rows=x[10]),
        rules(*x[:7], bias_tokens=x[7], bias_values=x[8], masks=x[9], mask_rows=x[10])]
    python_calls = [
        rotate(slots, q=torch.empty(3, 8, 64, dtype=BF16, device=DEV)), attend(table, n, scale=np.float64(0.2)), evict(new_table, np.int64(7)),
        rules(*x[:7], out=torch.empty_like(x[0]))]
    refused = [
        rotate(slots.long()), rotate(slots, eps=-1.0), attend(table, n.long()), attend(table, n, window=-2), attend(table, n, max_length=0), attend(table[:2], n),
        evict(new_table, 0), evict(new_table, -3), evict(new_table, 65), evict(new_table, 8, first=9), rules(x[0].double(), *x[1:7]), rules(*x[:7], masks=x[9]),
        rules(*x[:7], bias_tokens=x[7]), rules(x[0], x[1].long(), *x[2:7])]
    answered = []
    assert ann.binding._marshal is not None
    for name in ("rotate", "attend", "evict", "rules"):
        def spy(*args, native=getattr(ann.binding._marshal, name)):
            out = native(*args)
            answered.append(type(out) is tuple)
            return out
        monkeypatch.setattr(ann.binding._marshal, name, spy)
    for group, kind in ((answered_calls, "native"), (python_calls, "python"), (refused, "refused")):
        for number, call in enumerate(group):
            got = []
            for native in (True, False):
                with monkeypatch.context() as m:
                    if not native:
                        m.setattr(ann.binding, "_marshal", None)
                    del answered[:]
                    try:
                        out = call()
                        got.append([t.cpu().clone() for t in (out if isinstance(out, tuple) else (out,))])
                    except Exception as e:                # noqa: BLE001
                        got.append((type(e), str(e)))
                    assert any(answered) == (native and kind == "native"), (kind, number)
            a, b = got
            assert isinstance(a, tuple) == isinstance(b, tuple) == (kind == "refused"), (kind, number, a, b)
            if kind == "refused":
                assert a == b, (number, a, b)
            else:
                assert all(s.dtype == t.dtype and torch.equal(s, t) for s, t in zip(a, b)), (kind, number)
