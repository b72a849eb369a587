"""Argument errors of the operators that take many tokens at once, through the C ABI without a device; frequencies of a rotation."""
import ctypes
import math

import pytest
import torch

import paper_2505_12065_amd as ann
from paper_2505_12065_amd import binding
from test_decode_abi import A, BAD_CACHE, E, P, cache, call

APPEND = dict(qkv=P, token=512, head=64, T=3, q_heads=4, starts=P, B=2, lengths=P, table=P, width=5, positions=P, frequencies=P, rot=64, amplitude=1.0, pairs=0,
              cache=None, q=P, stream=None)
CHUNK = dict(q=P, row=256, head=64, T=3, q_heads=4, starts=P, B=2, cache=None, table=P, width=5, lengths=P, most=80, scale=0.1, window=0, out=P, lse=P, stream=None)
SHARED = dict(q=P, row=256, head=64, B=3, q_heads=4, cache=None, table=P, width=5, lengths=P, group_starts=P, shared=P, groups=2, max_shared=64, max_own=80, scale=0.1,
              out=P, lse=P, stream=None)


@pytest.mark.parametrize("fields,code", BAD_CACHE)
def test_a_cache_that_is_none(fields, code):
    for name, base in (("ann_rotate_append", APPEND), ("ann_chunk_attention", CHUNK), ("ann_shared_attention", SHARED)):
        assert call(name, base, cache=cache(**fields)) == code, (name, fields)
        assert binding.ann_last_error()


@pytest.mark.parametrize("name,base,kw,code", [
    *[("ann_rotate_append", APPEND, kw, code) for kw, code in (
        (dict(qkv=None), E), (dict(starts=None), E), (dict(lengths=None), E), (dict(table=None), E), (dict(frequencies=None), E), (dict(q=None), E), (dict(T=-1), E),
        (dict(T=2 ** 23), E), (dict(B=0), E), (dict(B=65537), E), (dict(q_heads=0), E), (dict(q_heads=65537), E), (dict(width=0), E), (dict(width=2 ** 27), E),
        (dict(rot=24), E), (dict(rot=80), E), (dict(rot=-16), E), (dict(amplitude=float("nan")), E), (dict(amplitude=float("inf")), E), (dict(token=-512), E),
        (dict(token=2 ** 60), E), (dict(head=60), A), (dict(qkv=P + 4), A), (dict(q=P + 8), A), (dict(starts=P + 2), A), (dict(positions=P + 1), A),
        (dict(frequencies=P + 4), A), (dict(lengths=P + 2), A), (dict(table=P + 3), A))],
    *[("ann_chunk_attention", CHUNK, kw, code) for kw, code in (
        (dict(q=None), E), (dict(table=None), E), (dict(lengths=None), E), (dict(out=None), E), (dict(starts=None), E), (dict(T=-1), E), (dict(T=2 ** 23), E), (dict(B=0), E),
        (dict(B=65537), E), (dict(q_heads=3), E), (dict(q_heads=0), E), (dict(q_heads=8194), E), (dict(T=2 ** 16, q_heads=2048), E), (dict(width=0), E), (dict(width=2 ** 28), E),
        (dict(most=0), E), (dict(most=81), E), (dict(scale=float("inf")), E), (dict(scale=float("nan")), E), (dict(window=-1), E), (dict(row=260), A), (dict(q=P + 8), A),
        (dict(out=P + 2), A), (dict(lse=P + 2), A), (dict(starts=P + 1), A), (dict(lengths=P + 2), A), (dict(row=-256), E))],
    *[("ann_shared_attention", SHARED, kw, code) for kw, code in (
        (dict(q=None), E), (dict(table=None), E), (dict(lengths=None), E), (dict(out=None), E), (dict(group_starts=None), E), (dict(shared=None), E), (dict(B=-1), E),
        (dict(B=65537), E), (dict(groups=0), E), (dict(groups=65537), E), (dict(q_heads=3), E), (dict(B=60000, q_heads=128), E), (dict(width=0), E), (dict(width=2 ** 28), E),
        (dict(max_shared=-1), E), (dict(max_shared=81), E), (dict(max_own=0), E), (dict(max_own=81), E), (dict(scale=float("inf")), E), (dict(row=260), A), (dict(q=P + 8), A),
        (dict(out=P + 2), A), (dict(lse=P + 2), A), (dict(group_starts=P + 2), A), (dict(shared=P + 1), A))],
])
def test_argument_errors(name, base, kw, code):
    assert call(name, base, **kw) == code, kw
    assert binding.ann_last_error()


def test_more_slots_than_a_sum_takes():
    for most, window, code in ((2 ** 26 + 1, 0, E), (2 ** 27, 2 ** 26 + 1, E)):
        assert call("ann_chunk_attention", CHUNK, width=2 ** 23, most=most, window=window) == code
        assert binding.ann_last_error()
        assert binding.lib().ann_chunk_attention_workspace_bytes(1, 1, 8, 2, 64, 0, most, window) == code
    for kw in (dict(max_shared=2 ** 26 + 1), dict(max_own=2 ** 26 + 1)):
        assert call("ann_shared_attention", SHARED, width=2 ** 23, **kw) == E
        assert binding.lib().ann_shared_attention_workspace_bytes(1, 1, 8, 2, 64, 0, kw.get("max_shared", 64), kw.get("max_own", 80)) == E
    assert binding.lib().ann_chunk_attention_workspace_bytes(1, 1, 8, 2, 64, 0, 2 ** 26, 0) > 0
    assert binding.lib().ann_chunk_attention_workspace_bytes(1, 1, 8, 2, 64, 0, 2 ** 30, 2 ** 20) > 0


def test_nothing_to_do():
    assert call("ann_rotate_append", APPEND, T=0) == 0 and call("ann_chunk_attention", CHUNK, T=0) == 0 and call("ann_shared_attention", SHARED, B=0) == 0


def test_workspace_of_sizes_that_are_none():
    w = binding.lib().ann_chunk_attention_workspace_bytes
    for args in ((0, 1, 8, 2, 64, 0, 100, 0), (1, 0, 8, 2, 64, 0, 100, 0), (1, 1, 7, 2, 64, 0, 100, 0), (1, 1, 8, 2, 264, 0, 100, 0), (1, 1, 8, 2, 64, 3, 100, 0), (1, 1, 8, 2, 64, 0, 0, 0),
                 (1, 1, 8, 2, 64, 0, 100, -1)):
        assert w(*args) == E, args
    w = binding.lib().ann_shared_attention_workspace_bytes
    for args in ((0, 1, 8, 2, 64, 0, 100, 9), (1, 0, 8, 2, 64, 0, 100, 9), (1, 1, 7, 2, 64, 0, 100, 9), (1, 1, 8, 2, 4, 0, 100, 9), (1, 1, 8, 2, 64, 3, 100, 9), (1, 1, 8, 2, 64, 0, -1, 9),
                 (1, 1, 8, 2, 64, 0, 100, 0)):
        assert w(*args) == E, args


def test_the_binding_refuses_what_is_not_on_a_device():
    x, i = torch.zeros(3, 8, 64), torch.zeros(3, dtype=torch.int32)
    c = torch.zeros(4, 2, 16, 64)
    for f in (lambda: ann.ann_rotate_append(x, i, i[:2], i.view(3, 1), None, c, c), lambda: ann.ann_chunk_attention(x, c, c, i.view(3, 1), i, i),
              lambda: ann.ann_shared_attention(x, c, c, i.view(3, 1), i, i, i)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(ValueError):
        ann.ann_chunk_attention_workspace_bytes(2 ** 32 + 1, 1, 8, 2, 64, torch.float16, 100)
    with pytest.raises(ValueError):
        ann.ann_shared_attention_workspace_bytes(1, 2 ** 32 + 1, 8, 2, 64, torch.float16, 100, 100)


# ---- frequencies ---------------------------------------------------------------------------------

def definition(rot, base, scaling="none", factor=1.0, original=0, low=1.0, high=32.0):
    def pair(r):
        return rot * math.log(original / (2 * math.pi * r)) / (2 * math.log(base))
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2))
    out = []
    for i in range(rot // 2):
        f = base ** (-2 * i / rot)
        if scaling == "linear":
            f = f / factor
        elif scaling == "ramp":
            a, b = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rot - 1)
            g = (i - a) / ((b - a) if b > a else 0.001)
            g = min(max(g, 0.0), 1.0)
            f = f * (1 - g) + f / factor * g
        elif scaling == "smooth":
            r = original * f / (2 * math.pi)
            u = (r - low) / (high - low)
            f = f / factor if r < low else f if r > high else (1 - u) * f / factor + u * f
        out.append(f)
    return out, 0.1 * math.log(factor) + 1 if scaling == "ramp" else 1.0


@pytest.mark.parametrize("rot", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("kw", [dict(), dict(base=500_000.0), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0), dict(scaling="ramp", factor=16.0, original=4096),
                                dict(scaling="ramp", factor=1.0, original=8), dict(scaling="ramp", factor=4.0, original=100_000, low=2.0, high=2.1, base=500_000.0),
                                dict(scaling="smooth", factor=8.0, original=8192, high=4.0, base=500_000.0)])
def test_frequencies(rot, kw):
    got, amplitude = ann.ann_rotation_frequencies(rot, **kw)
    want, size = definition(rot, **dict(dict(base=10_000.0), **kw))
    # powers of numbers up to 2^20 in binary64: an exponent of up to 20 bits is off by 2^-52 of itself, ten operations by 2^-53 each
    assert got.dtype == torch.float64 and got.shape == (rot // 2,)
    assert ((got - torch.tensor(want, dtype=torch.float64)) / torch.tensor(want, dtype=torch.float64)).abs().max() < 2.0 ** -46
    assert abs(amplitude - size) < 2.0 ** -50


def test_frequencies_at_their_ends():
    """What a scaling leaves alone and what it divides: fast pairs and slow ones."""
    plain, _ = ann.ann_rotation_frequencies(128)
    for scaling, high in (("ramp", 32.0), ("smooth", 4.0)):
        f, _ = ann.ann_rotation_frequencies(128, scaling=scaling, factor=8.0, original=4096, high=high)
        assert torch.equal(f[:5], plain[:5]) and torch.equal(f[-5:] * 8, plain[-5:]) and bool((f.diff() < 0).all())


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=24), dict(rot=272), dict(rot=-16), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(scaling="linear", factor=0.5),
                                dict(scaling="base", factor=float("inf")), dict(scaling="ramp", factor=2.0), dict(scaling="ramp", factor=2.0, original=10, low=0.0),
                                dict(scaling="smooth", factor=2.0, original=10, low=4.0, high=4.0)])
def test_frequencies_that_are_refused(kw):
    with pytest.raises(ann.AnnError) as e:
        ann.ann_rotation_frequencies(**dict(dict(rot=64), **kw))
    assert e.value.code == E


def test_frequencies_of_other_arguments():
    with pytest.raises(ValueError):
        ann.ann_rotation_frequencies(64, scaling="other")
    with pytest.raises(ValueError):
        ann.ann_rotation_frequencies(2 ** 32 + 64)
    d = ctypes.c_double()
    f = binding.lib().ann_rotation_frequencies
    assert f(64, 1e4, 5, 1.0, 0, 1.0, 2.0, ctypes.addressof(d), ctypes.addressof(d)) == E
    assert f(64, 1e4, -1, 1.0, 0, 1.0, 2.0, ctypes.addressof(d), ctypes.addressof(d)) == E
    assert f(64, 1e4, 0, 1.0, 0, 1.0, 2.0, None, ctypes.addressof(d)) == E and f(64, 1e4, 0, 1.0, 0, 1.0, 2.0, ctypes.addressof(d), None) == E


def test_constants_match_the_header():
    import re
    from test_abi import HEADER
    for name, value in binding.ROTATIONS.items():
        assert int(re.search(r"#define\s+ANN_ROTATION_%s\s+(\d+)" % name.upper(), HEADER).group(1)) == value
