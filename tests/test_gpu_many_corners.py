"""Calls of the operators that take many tokens at once which their documentation allows and that meet a corner of how work is dealt or numbers are held."""
import pytest
import torch

import decode as D                                        # (beside this file)
import many as M
import paper_2505_12065_amd as ann
from test_gpu_many import chunk, dev, shared

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
MOST = 2 ** 31 - 1


# ---- requests in no group -------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("sizes,common,starts,of", [([1, 4], [0, 400], [1, 5], [1]), ([2, 4, 2], [0, 400, 0], [2, 6], [1]), ([3, 2, 4], [0, 320, 800], [3, 5, 9], [1, 2]),
                                                    ([1, 5], [480, 0], [0, 0, 0, 1], [None, None, 0]), ([20, 1, 30], [0, 160, 0], [5, 5, 20, 21], [None, None, 1])])
@pytest.mark.parametrize("heads", [1, 4])
def test_leading_requests_in_no_group(dtype, sizes, common, starts, of, heads):
    """A group's number is that of a request that is in none; own slots in several parts, and bounds as close as they may be."""
    own = [(97 * b) % 700 + 300 for b in range(sum(sizes))]
    group = {b: of[g] for g in range(len(of)) for b in range(starts[g], starts[g + 1])}
    together = [0 if g is None else common[g] for g in of]
    of_request = [g for g, n in enumerate(sizes) for _ in range(n)]
    lengths = [common[of_request[b]] + own[b] for b in range(len(own))]
    most_own = max(n - (common[group[b]] if group.get(b) is not None else 0) for b, n in enumerate(lengths))

    def edit(q, k, v, table, lengths, *_):
        return q, k, v, table, lengths, starts, together
    for kw in (dict(), dict(max_shared=max(common), max_own=most_own)):
        shared(dtype, common, own, sizes, 4 * heads, heads, 64, 16, edit=edit, **kw)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_leading_requests_in_no_group_and_many_rows_in_common(dtype):
    """The same where slots in common go by tiles of 128 rows."""
    own = [(53 * b) % 500 + 200 for b in range(42)]

    def edit(q, k, v, table, lengths, *_):
        return q, k, v, table, lengths, [2, 42], [3504]
    shared(dtype, [0, 3504], own, [2, 40], 32, 4, 128, 16, edit=edit, max_shared=3504, max_own=max(own))


# ---- windows as large as there are ----------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("window", [40, 1000, MOST - 100, MOST])
def test_windows_where_some_tokens_have_no_slot(dtype, window):
    """Lengths below the number of new tokens: what a tile's first token has no slot for does not matter to its others; by many rows, and by few."""
    def edit(*lengths):
        return lambda q, k, v, table, _: (q, k, v, table, list(lengths))
    chunk(dtype, [180], [0], 4, 2, 64, 16, window=window, edit=edit(150))
    chunk(dtype, [300, 128, 70], [0, 0, 0], 2, 2, 128, 16, window=window, edit=edit(290, 100, 1), max_length=280)
    chunk(dtype, [60] + [1] * 9, [0] + [40] * 9, 1, 1, 64, 16, window=window, edit=edit(50, *[41] * 9))


# ---- small values ---------------------------------------------------------------------------------

def small(v, exponent):
    """v becomes values of sizes 1 to 2 times a power of two, which both types of 8 bits of exponent hold."""
    return torch.where(v < 0, -1.0, 1.0).to(v.dtype) * (1 + v.abs().clamp(max=7) / 8) * 2.0 ** exponent


@pytest.mark.parametrize("dtype,exponent", [(BF16, -105), (F32, -104)])
def test_small_values_behind_a_wide_table(dtype, exponent):
    """What a page table could hold, and slots that a window leaves out, cost no digits of small values."""
    width = (MOST - 65536) // 1024

    def wide(q, k, v, table, *rest):
        return q, k, v.copy_(small(v, exponent)), torch.cat([table, torch.full((len(table), width - table.shape[1]), -1, dtype=torch.int32)], 1), *rest
    chunk(dtype, [3, 1], [2500, 90], 4, 2, 64, 1024, window=100, edit=wide)
    chunk(dtype, [150, 40], [1000, 0], 4, 2, 64, 1024, window=100, edit=wide)
    shared(dtype, [2048], [300, 600, 20], [3], 4, 2, 64, 1024, max_shared=2048, max_own=600, edit=wide)
    shared(dtype, [2048], [300, 600, 20], [3], 4, 2, 64, 1024, max_shared=0, max_own=2648, edit=wide)


@pytest.mark.parametrize("T", [2, 90])
def test_small_values_that_have_all_the_weight(T):
    """fp32, near its smallest normal number (2^-126): of 9000 slots, which take 14 bits of the sums' range and one is left, one has all the weight."""
    n, d, page = 9000, 64, 64
    g = torch.Generator().manual_seed(T)
    pages = (n + page - 1) // page
    k, v = torch.zeros(pages, 1, page, d), small(torch.randn(pages, 1, page, d, generator=g), -115)
    k[77, 0, 5, 0] = 1
    q = torch.zeros(T, 2, d)
    q[..., 0] = 100                                       # (e^-100 2^13 is below 2^-130)
    table = torch.arange(pages, dtype=torch.int32).view(1, -1)
    out, _ = ann.ann_chunk_attention(dev(q), dev(k), dev(v), dev(table), dev(M.ints([n])), dev(M.ints([0, T])), scale=1.0, max_length=n)
    want = v[77, 0, 5].double()
    # a tile's sum, its factor, the row's sum, a joined part's factor and sum: numbers from 2^-115 2^-15 on, whose last place is 2^-149; weight, sums, division and product 2^-24 each
    assert ((out.double().cpu() - want).abs() <= 5 * 2.0 ** (-150 + 15) + 16 * D.U * want.abs()).all()


# ---- fp32 values near the largest -----------------------------------------------------------------

@pytest.mark.parametrize("T,common", [(9, None), (70, None), (5, 160), (130, 160)])
def test_values_near_the_largest_and_large_scores(T, common):
    """fp32: scores near 100 000, which exponents hold to 2^-7, so that weights of the largest score are up to 2^(2^-7) times what they are by it.  A row's scores are all the same, and so are its weights."""
    n, d, page = 200, 64, 16
    value = torch.finfo(F32).max * 0.999
    k, v = torch.zeros(13, 1, page, d, device=DEV), torch.full((13, 1, page, d), value, device=DEV)
    k[..., 0] = 1
    q = torch.zeros(T, 2, d, device=DEV)
    q[..., 0] = torch.arange(2 * T, device=DEV).view(T, 2) + 100_000
    table = torch.arange(13, dtype=torch.int32, device=DEV)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    if common is None:
        out, _ = ann.ann_chunk_attention(q, k, v, table.view(1, -1), ints(n), ints(0, T), scale=1.0, max_length=n)
    else:
        out, _ = ann.ann_shared_attention(q, k, v, table.repeat(T, 1), ints(*[n] * T), ints(0, T), ints(common), max_shared=common, max_own=n - common, scale=1.0)
    # sums of up to 200 products and of 200 weights, in any order, a division and a product: 2^-24 each
    assert bool(torch.isfinite(out).all()) and (out.double() / value - 1).abs().max() <= (2 * n + 8) * D.U


# ---- lse ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_lse_of_equal_scores(dtype):
    """Scores of 0: weights are one power of two and sums of them exact, so lse is the logarithm of a whole number, off by 2 units in the last place of a logarithm at most (2^-22 of it): by many
    rows, by few, in parts and with slots in common."""
    d, page = 64, 16
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731

    def near(lse, slots):
        want = torch.tensor(slots, dtype=torch.float64, device=DEV).log()[:, None]
        assert bool(((lse.double() - want).abs() <= 2.0 ** -22 * want).all()), (lse.double() - want).abs().max()

    k = torch.randn(600, 1, page, d, device=DEV).to(dtype)
    for T, n in ((2048, 2048), (300, 9000), (4, 9000), (1, 1)):
        table = torch.arange(600, dtype=torch.int32, device=DEV).view(1, -1)
        q = torch.zeros(T, 2, d, dtype=dtype, device=DEV)
        near(ann.ann_chunk_attention(q, k, k, table, ints([n]), ints([0, T]), max_length=n)[1], list(range(n - T + 1, n + 1)))
    for B in (7, 60, 300):
        lengths = [1 + 31 * b for b in range(B)]
        table = torch.arange(600, dtype=torch.int32, device=DEV).repeat(B, 1)
        q = torch.zeros(B, 2, d, dtype=dtype, device=DEV)
        near(ann.ann_chunk_attention(q, k, k, table, ints(lengths), ints(list(range(B + 1))))[1], lengths)
        for common in (0, 160, 4000):
            near(ann.ann_shared_attention(q, k, k, table, ints(lengths), ints([0, B]), ints([common]), max_shared=common)[1], lengths)


# ---- more requests than a wave has lanes -----------------------------------------------------------

@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("common,most_own", [(48, 1000), (16, 993), (80, 1024)])
def test_own_slots_of_more_than_64_requests_in_parts(dtype, common, most_own):
    """Own slots that begin off a multiple of 32 and are as many as may count: the last part holds what the beginning was moved by."""
    own = [most_own + common % 16 if b % 3 == 0 else (37 * b) % most_own for b in range(70)]
    shared(dtype, [common], own, [70], 2, 1, 64, 16, max_shared=common, max_own=most_own)
    # by the same plan, with all requests in no group but one
    shared(dtype, [common], own, [70], 2, 1, 64, 16, max_shared=common, max_own=most_own, edit=lambda *x: (*x[:5], [69, 70], x[6]))


# ---- outputs in the place of inputs ----------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("new,held", [([180, 3], [100, 700]), ([2, 5], [3000, 10]), ([1] * 80, [100] * 80)])
def test_attention_in_the_place_of_queries(dtype, new, held):
    """By many rows and by few, in parts and whole; a token's q where its rows of qkv begin."""
    lengths = [n + h for n, h in zip(new, held)]
    k, v, table = D.paged(lengths, 16, 2, 64, dtype, 3)
    q = D.rows(sum(new), 4, 64, dtype=dtype, seed=4).to(DEV)
    args = dev(k), dev(v), dev(table), dev(M.ints(lengths))
    want, want_lse = ann.ann_chunk_attention(q, *args, dev(M.starts_of(new)))
    own = q.clone()
    out, lse = ann.ann_chunk_attention(own, *args, dev(M.starts_of(new)), out=own)
    assert out is own and torch.equal(out, want) and torch.equal(lse, want_lse)
    B = len(new)
    groups = dev(M.ints([0, B])), dev(M.ints([0]))
    want, want_lse = ann.ann_shared_attention(q[:B], *args, *groups)
    own = q[:B].clone()
    out, lse = ann.ann_shared_attention(own, *args, *groups, out=own)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_append_of_one_token_in_the_place_of_its_rows():
    x = torch.randn(1, 8, 64, device=DEV)
    i = lambda *a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    frequencies, _ = ann.ann_rotation_frequencies(64, device=DEV)
    caches = [torch.zeros(1, 2, 16, 64, device=DEV) for _ in range(4)]
    want = ann.ann_rotate_append(x, i(0, 1), i(8), i(0).view(1, 1), frequencies, *caches[:2])
    own = x.clone()
    q = ann.ann_rotate_append(own, i(0, 1), i(8), i(0).view(1, 1), frequencies, *caches[2:], q=own[:, :4])
    assert torch.equal(q, want) and torch.equal(own[:, 4:], x[:, 4:]) and torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])
