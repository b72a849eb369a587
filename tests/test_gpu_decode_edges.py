"""The operators over a paged cache at the ends of their ranges, against their definitions in 64 bits, and ways to call them that take another path."""
import math

import numpy as np
import pytest
import torch

import decode as D                                        # (beside this file)
import paper_2505_12065_amd as ann
from test_gpu_decode import all_four, attend, dev

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
LEAST, MOST = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("page", [4, 16])
@pytest.mark.parametrize("window", [1, 1001, MOST - 1, MOST])
def test_attention_negative_lengths_with_any_window(dtype, page, window):
    """A negative length is none, whatever is taken off it."""
    def edit(q, k, v, table, lens):
        lens[1:5] = torch.tensor([LEAST, LEAST + 1000, -3, -1], dtype=torch.int32)
        return q, k, v, table, lens
    out = attend(dtype, [700, 10, 10, 10, 10, 0, 33], 4, 2, 64, page, window=window, mass=True, seed=31, edit=edit)
    assert (out[1:6] == 0).all()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("with_mass", [False, True])
def test_attention_of_the_longest_context(dtype, with_mass):
    """As many slots as a page table may hold (its pages are the same three).  All scores are 0, so every sum of a part is a whole number below 2^24 and exact;
    the parts' are added up with a relative 2^-24 each, the logarithm (21.5) is right to a few of its last places, 2^-19."""
    page, d, short = 1024, 8, 5
    width = (MOST - 65536) // page
    n = width * page - short
    k, v = torch.randn(3, 1, page, d, device=DEV).to(dtype), torch.zeros(3, 1, page, d, dtype=dtype, device=DEV)
    v[..., 0], v[1, ..., 1], v[2, ..., 2] = 1, 1024, 1024
    table = torch.zeros(1, width, dtype=torch.int32, device=DEV)
    table[0, -1], table[0, 0] = 1, 2                      # the last page, of which `short` slots are behind the end, and the first
    lens = torch.tensor([n], dtype=torch.int32, device=DEV)
    mass = torch.zeros(1, 1, width * page, device=DEV) if with_mass else None
    q = torch.zeros(1, 1, d, dtype=dtype, device=DEV)
    if with_mass:                                         # (the library's own buffer stays as small as it is)
        space = torch.empty(ann.ann_paged_attention_workspace_bytes(1, 1, 1, d, dtype, width * page, True), dtype=torch.uint8, device=DEV)
        ann.ann_set_workspace(space)
    try:
        out, lse = ann.ann_paged_attention(q, k, v, table, lens, mass=mass)
        torch.cuda.synchronize()
    finally:
        if with_mass:
            ann.ann_set_workspace(None)
    want = torch.tensor([1.0, (page - short) * 1024 / n, page * 1024 / n, 0, 0, 0, 0, 0], dtype=torch.float64)
    off = (out[0, 0].double().cpu() - want).abs()
    assert (off <= want * (D.HALF_ULP[dtype] * 1.01 + 2.0 ** -18) + D.TINY[dtype]).all(), off
    assert abs(lse.item() - torch.tensor(float(n), dtype=torch.float64).log().item()) <= 2.0 ** -17
    if with_mass:
        low, high = torch.aminmax(mass[0, 0, :n])
        assert abs(low.item() * n - 1) <= 2.0 ** -16 and abs(high.item() * n - 1) <= 2.0 ** -16 and not mass[0, 0, n:].any()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("d", [136, 256])
@pytest.mark.parametrize("G,heads,longest", [(32, 1, 192), (32, 1, 193), (32, 1, 250), (32, 1, 256), (32, 1, 257), (28, 32, 384), (28, 32, 400), (28, 32, 576),
                                             (28, 32, 577), (25, 32, 600), (32, 32, 448)])
def test_attention_weights_of_many_heads_beside_large_sums(dtype, d, G, heads, longest):
    """Two tiles of query heads of d > 128 leave little of a compute unit's LDS for scores, which go to the workspace where they do not fit."""
    lengths = [longest, 0, 1, 7, 33, 64, 65, 150] if heads > 1 else [longest, 200, 0]
    attend(dtype, lengths, G * heads, heads, d, 16, mass=True, seed=longest)


@pytest.mark.parametrize("dtype,largest", [(F16, 6e4), (BF16, 3e38), (F32, 3e38)])
@pytest.mark.parametrize("lengths,Hq,heads,d,page,window", [([300, 1, 17, 64, 0], 8, 2, 64, 16, 0), ([5000, 4, 700], 6, 2, 128, 16, 0), ([20_001, 90], 4, 4, 80, 64, 0),
                                                            ([5000, 3000], 40, 2, 128, 16, 2000), ([2100], 4, 1, 256, 4, 0), ([900, 40, 0, 1, 2, 3, 4, 5], 64, 32, 16, 16, 0)])
@pytest.mark.parametrize("same", [False, True])
def test_attention_of_values_near_the_largest(dtype, largest, lengths, Hq, heads, d, page, window, same):
    """Finite values whose sum over the slots, before it is divided, is beyond 32 bits: half the slots' of one sign, or all of one value."""
    def edit(q, k, v, table, lens):
        g = torch.Generator().manual_seed(5)
        v[:] = largest if same else (torch.randint(0, 4, v.shape, generator=g).clamp(max=2) - 1) * largest
        return q, k, v, table, lens
    attend(dtype, lengths, Hq, heads, d, page, window=window, seed=41, edit=edit)
    attend(dtype, lengths, Hq, heads, d, page, window=window, seed=42, edit=edit, mass=True)


@pytest.mark.parametrize("page", [2, 16])
@pytest.mark.parametrize("length,B,heads", [(90, 2, 2), (3000, 2, 2), (300, 8, 32)])
def test_weights_of_a_head_with_nan_leave_slots_without_a_row_alone(page, length, B, heads):
    """One part, parts that are joined, and scores that stay on the chip."""
    k, v, table = D.paged([length] * B, page, heads, 64, BF16, 3)
    q = D.rows(B, 2 * heads, 64, dtype=BF16, seed=4)
    q[1, 1, 3] = float("nan")                             # a query head of the first cache head of the second request
    table[:, 1] = -1
    slots = table.shape[1] * page
    before = torch.rand(B, heads, slots, generator=torch.Generator().manual_seed(1))
    mass = dev(before)
    ann.ann_paged_attention(dev(q), dev(k), dev(v), dev(table), torch.full((B,), length, dtype=torch.int32, device=DEV), mass=mass)
    mass = mass.cpu()
    j = torch.arange(slots)
    there = (j < length) & ((j < page) | (j >= 2 * page))
    assert torch.equal(mass[:, :, ~there], before[:, :, ~there])
    assert torch.isnan(mass[1, 0, there]).all() and torch.isfinite(mass[0]).all() and torch.isfinite(mass[1, 1:]).all() and torch.isfinite(mass[2:]).all()
    assert (mass[0][:, there] >= before[0][:, there]).all()


def test_whole_numbers_beyond_32_bits_are_refused():
    """Not taken for what is left of them in 32 bits."""
    k = torch.zeros(4, 2, 16, 64, dtype=BF16, device=DEV)
    q, table = torch.zeros(3, 4, 64, dtype=BF16, device=DEV), torch.zeros(3, 2, dtype=torch.int32, device=DEV)
    n, mass = torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(3, 2, 32, device=DEV)
    for kw in (dict(window=2 ** 32 + 1), dict(window=2 ** 32), dict(window=2 ** 31), dict(max_length=2 ** 32 + 8), dict(max_length=-2 ** 32 + 8)):
        with pytest.raises(ValueError):
            ann.ann_paged_attention(q, k, k, table, n, **kw)
    for budget, kw in ((2 ** 32 + 8, {}), (-2 ** 32 + 8, {}), (8, dict(first=2 ** 32 + 1)), (8, dict(recent=2 ** 32)), (8, dict(first=-2 ** 32))):
        with pytest.raises(ValueError):
            ann.ann_cache_evict(k, k, table, n, mass, table, budget, **kw)


@pytest.mark.parametrize("most", [4095, 4096, 4097, 8191, 8192, 8193, 12_001, 16_383, 16_384, 16_385, 32_767, 32_768, 32_769])
@pytest.mark.parametrize("budget,first,recent", [(700, 3, 40), (4000, 0, 0)])
def test_evict_on_both_sides_of_what_a_thread_holds(most, budget, first, recent):
    """Rows of as many slots as fit the ranks that a thread holds, one more and one less, and shorter requests among them."""
    heads, d, page, lengths = 3, 64, 16, [most, most - 1, most * 3 // 5]
    g = torch.Generator().manual_seed(most + budget)
    B, new_width = 3, -(-budget // page)
    k, v, table = D.paged(lengths, page, heads, d, BF16, most, unused=9.0, spare=B * new_width)
    free = [p for p in range(k.shape[0]) if p not in set(table.flatten().tolist())]
    new_table = torch.tensor(free[:B * new_width], dtype=torch.int32).view(B, new_width)
    mass = torch.randn(B, heads, most, generator=g).pow(3)
    mass[:, 1] = (mass[:, 1] * 2).round() / 2             # equal ones by the hundred
    mass[:, 2, ::5] = 0.25
    mass[0, 0, 3::7], mass[0, 0, 4::11], mass[0, 2, 2::9] = math.nan, math.inf, -math.inf
    mass[1, 2] = math.nan
    mass[2, 2] = 1.0
    want, new = D.evict(mass.numpy(), lengths, most, budget, first, recent)
    dk, dv = dev(k), dev(v)
    kept, got_new, got_mass = ann.ann_cache_evict(dk, dv, dev(table), torch.tensor(lengths, dtype=torch.int32, device=DEV), dev(mass), dev(new_table), budget,
                                                  first=first, recent=recent)
    assert np.array_equal(kept.cpu().numpy(), want) and np.array_equal(got_new.cpu().numpy(), new)
    for b in range(B):
        i = torch.arange(int(new[b]))
        for h in range(heads):
            j = torch.from_numpy(want[b, h, :int(new[b])]).long()
            assert np.array_equal(got_mass[b, h, :len(i)].cpu().numpy(), mass[b, h, j].numpy(), equal_nan=True)
            for got, source in ((dk, k), (dv, v)):
                assert torch.equal(got[new_table[b].long()[i // page].to(DEV), h, (i % page).to(DEV)].cpu(), source[table[b].long()[j // page], h, j % page])


def test_streams_that_are_named():
    """stream= of all four, a Stream or its handle, instead of the current one."""
    want = [t.clone() for t in all_four()()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        call = all_four(stream)
        torch.cuda.synchronize()                          # (its inputs were made on the current one)
        with torch.cuda.stream(side):                     # (what torch itself does inside)
            got = call()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    # the operators alone on `side`, torch's own work on the current stream
    k, v, table = (dev(t) for t in D.paged([300, 40], 16, 2, 64, BF16, 21, unused=0.0))
    q, n = dev(D.rows(2, 8, 64, dtype=BF16, seed=5)), torch.tensor([300, 40], dtype=torch.int32, device=DEV)
    plain = ann.ann_paged_attention(q, k, v, table, n)
    torch.cuda.synchronize()
    named = ann.ann_paged_attention(q, k, v, table, n, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(plain, named))


@pytest.mark.parametrize("lengths", [[300, 0, 33], [5000, 1, 0]])
@pytest.mark.parametrize("with_mass", [False, True])
def test_outputs_that_are_given_or_not_wanted(lengths, with_mass):
    k, v, table = (dev(t) for t in D.paged(lengths, 16, 2, 64, F16, 8))
    q, n = dev(D.rows(3, 8, 64, dtype=F16, seed=9)), torch.tensor(lengths, dtype=torch.int32, device=DEV)
    masses = [torch.zeros(3, 2, table.shape[1] * 16, device=DEV) if with_mass else None for _ in range(3)]
    want = ann.ann_paged_attention(q, k, v, table, n, mass=masses[0])
    out, lse = torch.full_like(want[0], 7), torch.full_like(want[1], 7)
    got = ann.ann_paged_attention(q, k, v, table, n, out=out, lse=lse, mass=masses[1])
    assert got[0] is out and got[1] is lse and torch.equal(out, want[0]) and torch.equal(lse, want[1])
    out = torch.full_like(out, 7)
    b = ann.binding
    cache = b._cache(k, v)
    rc = b.lib().ann_paged_attention(q.data_ptr(), 512, 64, 3, 8, cache, table.data_ptr(), table.shape[1], n.data_ptr(), table.shape[1] * 16, 0.125, 0,
                                     out.data_ptr(), None, masses[2].data_ptr() if with_mass else None, table.shape[1] * 16, torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(out, want[0])
    assert not with_mass or all(torch.equal(m, masses[0]) for m in masses)
    for bad in (dict(out=out.float()), dict(out=out[:2]), dict(lse=lse.half()), dict(lse=lse[:, :4]), dict(out=out.cpu())):
        with pytest.raises(ValueError):
            ann.ann_paged_attention(q, k, v, table, n, **bad)


@pytest.mark.parametrize("with_mass", [False, True])
@pytest.mark.parametrize("own", [False, True])
def test_captured_with_less_workspace_than_is_wanted(with_mass, own):
    """The library's buffer may not grow while a stream is captured, a caller's never does: the graph takes fewer requests at a time, with the same bits."""
    lengths = [3000, 10, 2000, 0, 2999, 1500, 700]
    k, v, table = D.paged(lengths, 16, 2, 64, F16, 2)
    args = dev(D.rows(7, 8, 64, dtype=F16, seed=4)), dev(k), dev(v), dev(table), torch.tensor(lengths, dtype=torch.int32, device=DEV)
    slots = table.shape[1] * 16
    want = ann.ann_paged_attention(*args, mass=None)
    mass = torch.zeros(7, 2, slots, device=DEV) if with_mass else None
    if with_mass:
        want = (*ann.ann_paged_attention(*args, mass=mass), mass.clone())
    one, whole = (ann.ann_paged_attention_workspace_bytes(B, 8, 2, 64, F16, slots, with_mass) for B in (1, 7))
    assert 1.3 * one < whole
    torch.cuda.synchronize()
    ann.ann_release_workspace()
    if own:                                               # (a call of one request, so that there is a little; it grows by a quarter more than that)
        ann.ann_paged_attention(args[0][:1], args[1], args[2], args[3][:1], args[4][:1], mass=None if mass is None else torch.zeros_like(mass[:1]))
    else:
        buffer = torch.empty(one, dtype=torch.uint8, device=DEV)            # (the library keeps its address alone)
        ann.ann_set_workspace(buffer)
    torch.cuda.synchronize()
    try:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            if with_mass:
                mass.zero_()
            got = ann.ann_paged_attention(*args, mass=mass)
        got = (*got, mass) if with_mass else got
        for _ in range(4):
            for t in got:
                t.fill_(3)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            torch.randn(1000, 1000, device=DEV).sum().item()
    finally:
        torch.cuda.synchronize()
        ann.ann_set_workspace(None)


@pytest.mark.parametrize("dtype,bits", [(F32, 0), (F16, 2.0 ** -22), (BF16, 2.0 ** -17)])
def test_bits_of_a_weight(dtype, bits):
    """An output that is one weight: its exponent t log2 e is off by two roundings, |t| <= 3 times 2 U, the power of two, the sum, its reciprocal and the product
    by 1 to 2 U each; 16-bit types have the weight in two parts, which are off by `bits`, and round the output.  An fp32 weight in two such parts would be seen."""
    B, d, g = 256, 8, torch.Generator().manual_seed(7)
    t = (3 * torch.rand(B, generator=g)).to(dtype)
    q, k, v = torch.zeros(B, 1, d, dtype=dtype), torch.zeros(B, 1, 16, d, dtype=dtype), torch.zeros(B, 1, 16, d, dtype=dtype)
    q[:, 0, 0], k[:, 0, 1, 0], v[:, 0, 1] = 1, -t, 1
    table, n = torch.arange(B, dtype=torch.int32).view(B, 1), torch.full((B,), 2, dtype=torch.int32)
    out, lse = ann.ann_paged_attention(dev(q), dev(k), dev(v), dev(table), dev(n), scale=1.0)
    w = torch.exp(-t.double())
    want = (w / (1 + w))[:, None, None]
    off = ((out.double().cpu() - want) / want).abs().max().item()
    assert off <= 20 * D.U + bits + (D.HALF_ULP[dtype] * 1.01 if dtype != F32 else 0), off
    assert (lse[:, 0].double().cpu() - torch.log1p(w)).abs().max() <= 20 * D.U
