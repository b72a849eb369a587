"""How the operators that take many tokens at once divide a call, decided without a GPU: the host rules of plan.hpp, compiled with the C++ compiler alone."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = r"""
#include "plan.hpp"
using namespace ann;
static void put(const ChunkPlan &p, int64_t *out) {
    int64_t *o = out;
    for (const ChunkPass *q : {&p.first, &p.own}) {
        const int64_t v[] = {q->mode, q->rows, q->items, q->fill, q->most_parts, q->least, q->part0, q->tiles, q->chunk};
        for (int64_t x : v) *o++ = x;
    }
    *o++ = p.splits;
    *o++ = (int64_t)p.bytes;
}
extern "C" void chunk(int cus, int eb, int d, int q_heads, int heads, int64_t T, int64_t B, int64_t length, int64_t window, int64_t most, int64_t *out) {
    put(chunk_plan(cus, eb, d, q_heads, heads, T, B, length, window, (size_t)most), out);
}
extern "C" void shared(int cus, int eb, int d, int q_heads, int heads, int64_t B, int64_t groups, int64_t max_shared, int64_t max_own, int64_t most, int64_t *out) {
    put(shared_plan(cus, eb, d, q_heads, heads, B, groups, max_shared, max_own, (size_t)most), out);
}
extern "C" int64_t enough(int64_t B, int64_t q_heads, int64_t d) { return (int64_t)shared_most(B, q_heads, d); }
extern "C" float lift(int dtype, int64_t slots) { return chunk_lift(dtype, slots); }
extern "C" int lds(int eb, int ve, int mt) { return (int)attend_lds_bytes(eb, ve, mt, 16 * mt, 0); }
"""
FIELDS = ("mode", "rows", "items", "fill", "most_parts", "least", "part0", "tiles", "chunk")
NEW, COMMON, OWN, ALL = range(4)
MOST = 2 ** 31 - 65537


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    folder = tmp_path_factory.mktemp("plans")
    (folder / "shim.cpp").write_text(SHIM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2505_12065_amd", "csrc"),
                           str(folder / "shim.cpp"), "-o", str(folder / "shim.so")])
    lib = ctypes.CDLL(str(folder / "shim.so"))
    i, n, p = ctypes.c_int, ctypes.c_int64, ctypes.POINTER(ctypes.c_int64)
    lib.chunk.argtypes = lib.shared.argtypes = [i] * 5 + [n] * 5 + [p]
    lib.enough.argtypes, lib.enough.restype = [n] * 3, n
    lib.lift.argtypes, lib.lift.restype = [i, n], ctypes.c_float
    return lib


def plan(f, *args):
    out = (ctypes.c_int64 * 20)()
    f(256, *args, out)
    first, own = (dict(zip(FIELDS, out[9 * k:9 * k + 9])) for k in range(2))
    return first, own, out[18], out[19]


def log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def check(p, heads, rows, sequences, length, splits):
    """Tiles and parts fit a launch and each other."""
    assert 1 <= p["most_parts"] <= 64 and p["part0"] + p["most_parts"] <= splits <= 128
    least = p["tiles"]
    per = -(-rows // sequences)
    tiles = sequences * -(-per // p["rows"]) if p["mode"] >= OWN else rows // p["rows"] + sequences
    assert least == tiles and p["items"] >= (tiles if p["most_parts"] == 1 else 1)
    assert p["items"] * heads < 2 ** 24
    if sequences > 64:
        assert p["items"] == tiles * p["most_parts"] and p["chunk"] * p["most_parts"] >= length and p["chunk"] % 64 == 0 and p["chunk"] < 2 ** 31
    else:
        # parts are evened out to at most fill or 2 fill workgroups, or are one to a tile
        assert p["items"] >= min(tiles * p["most_parts"], p["fill"])


def test_new_tokens(plans):
    rng = random.Random(1)
    for _ in range(6000):
        heads, G = log(rng, 1, 64), log(rng, 1, 100)
        if heads * G > 8192:
            continue
        T, B, d, eb = log(rng, 1, 4_000_000), log(rng, 1, 65536), 8 * rng.randint(1, 32), rng.choice([2, 4])
        if T * heads * G > 2 ** 26 or B * heads > 2 ** 22:
            continue
        length = rng.choice([log(rng, 1, 100_000), MOST])
        window = rng.choice([0, 0, 1, 100, 2 ** 31 - 1])
        most = rng.choice([1 << 30, log(rng, 1, 1 << 30)])
        first, own, splits, size = plan(plans.chunk, eb, d, heads * G, heads, T, B, length, window, most)
        assert own["items"] == 0 and first["mode"] == NEW and size <= most and (size == 0) == (splits == 1)
        check(first, heads, T * G, B, min(length, window + 160) if window else length, splits)


def test_groups(plans):
    rng = random.Random(2)
    for _ in range(6000):
        heads, G = log(rng, 1, 64), log(rng, 1, 100)
        if heads * G > 8192:
            continue
        B, groups, d, eb = log(rng, 1, 65536), log(rng, 1, 65536), 8 * rng.randint(1, 32), rng.choice([2, 4])
        if B * heads * G > 2 ** 22 or groups * heads > 2 ** 22:
            continue
        shared, own_slots = rng.choice([0, log(rng, 1, 100_000), MOST]), rng.choice([log(rng, 1, 10_000), MOST])
        enough = plans.enough(B, heads * G, d)
        most = rng.choice([enough, log(rng, 1, enough)])
        first, own, splits, size = plan(plans.shared, eb, d, heads * G, heads, B, groups, shared, own_slots, most)
        assert size <= most and (size == 0) == (splits == 1)
        if most == enough and shared:
            assert first["mode"] == COMMON and own["mode"] == OWN
        if first["mode"] == COMMON:
            assert own["part0"] == first["most_parts"] and splits == first["most_parts"] + own["most_parts"]
            assert first["rows"] in (own["rows"], 128)
            check(first, heads, B * G, groups, shared, splits)
            check(own, heads, B * G, B, own_slots, splits)
        else:
            assert first["mode"] == ALL and own["items"] == 0
            check(first, heads, B * G, B, min(shared + own_slots, MOST), splits)


def test_nothing_is_divided_where_there_is_enough_to_do(plans):
    assert plan(plans.chunk, 2, 128, 32, 8, 16384, 1, 16384, 0, 1 << 30)[2:] == (1, 0)
    assert plan(plans.chunk, 2, 128, 28, 4, 24 * 170, 24, 8400, 0, 1 << 30)[2:] == (1, 0)
    assert plan(plans.shared, 2, 128, 32, 8, 64, 1, 8096, 1004, 1 << 30)[1]["most_parts"] == 1
    assert plan(plans.chunk, 2, 128, 32, 8, 100, 1, 1600, 0, 1 << 30)[2] > 1


def test_weights_stay_within_their_types(plans):
    """A weight may be 2^8 times what it is by the score it goes by: fp16's largest is 65504, and bf16's and fp32's sums of as many values near the largest as there are slots stay below it."""
    assert 2.0 ** (plans.lift(0, 2 ** 31 - 1) + 8) <= 65504 and plans.lift(0, 1) == plans.lift(0, 2 ** 31 - 1)
    for dtype in (1, 2):
        for n in (1, 2, 3, 63, 64, 65, 1000, 2 ** 20, MOST):
            assert n * 2.0 ** (plans.lift(dtype, n) + 8) <= 1 and plans.lift(dtype, n) >= -40


def test_few_rows_fit_a_compute_unit(plans):
    for eb in (2, 4):
        for ve in (4, 8, 16):
            for mt in (1, 2):
                assert plans.lds(eb, ve, mt) <= 160 * 1024


def test_sums_of_weights_leave_room_for_roundings(plans):
    """Weights are as far above their power of two as the exponent of the score they go by is rounded down (2^(2^-7) at scores of 100 000), and sums are rounded too: sums stay below half of the largest value."""
    for n in (1, 63, 64, 4095, 65_535, 2 ** 20, 2 ** 26):
        assert n * 2.0 ** (plans.lift(1, n) + 8) <= 0.5


def test_parts_of_own_slots_cover_where_they_begin(plans):
    """A request's own slots are read from a multiple of 32 on, up to 31 below the first: parts of more than 64 requests, whose length the host says, have to hold these too."""
    rng = random.Random(3)
    divided = 0
    for _ in range(6000):
        heads, G, B, groups = log(rng, 1, 16), log(rng, 1, 32), log(rng, 65, 2000), log(rng, 1, 2000)
        if heads * G > 8192 or B * heads * G > 2 ** 22:
            continue
        shared, own_slots, d, eb = log(rng, 1, 100_000), rng.choice([64, 65, 512, log(rng, 1, 100_000)]), 8 * rng.randint(1, 32), rng.choice([2, 4])
        first, own, _, _ = plan(plans.shared, eb, d, heads * G, heads, B, groups, shared, own_slots, plans.enough(B, heads * G, d))
        assert own["chunk"] * own["most_parts"] >= own_slots + 31
        divided += own["most_parts"] > 1
    assert divided > 100
