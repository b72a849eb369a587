"""The operators over a paged cache at the ends of their ranges, against their definitions in 64 bits."""
import pytest
import torch

import decode as D                                        # (beside this file)
import paper_2505_12065_amd as ann
from test_gpu_decode import attend, close, dev            # noqa: F401

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
