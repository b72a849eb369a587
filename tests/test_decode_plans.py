"""How the operators over a paged cache divide a call, decided without a GPU: the host rules of plan.hpp, compiled with the C++ compiler alone."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = r"""
#include "plan.hpp"
using namespace ann;
// out: groups, splits, chunk, pad, part, once, bytes of a request, step, head tiles, LDS bytes, floats from head to head of scores in LDS
extern "C" void attend(int cus, int B, int q_heads, int heads, int d, int eb, int max_length, int window, int mass, int64_t most, int64_t *out) {
    const AttendPlan p = attend_plan(cus, B, q_heads, heads, d, eb, max_length, window, mass != 0, (size_t)most);
    const int G = q_heads / heads, mt = attend_head_tiles(eb, attend_ve(d), G);
    const int64_t v[] = {p.groups, p.splits, p.chunk, p.pad, p.part, p.once, (int64_t)p.one, attend_step(eb, d), mt, (int64_t)attend_lds_bytes(eb, attend_ve(d), mt, G, p.keep), p.keep};
    for (int i = 0; i < 11; ++i) out[i] = v[i];
}
extern "C" int64_t workspace(int cus, int B, int q_heads, int heads, int d, int eb, int max_length, int mass, int64_t most) {
    return (int64_t)attend_workspace(cus, B, q_heads, heads, d, eb, max_length, mass != 0, (size_t)most);
}
extern "C" int chunk(int cus, int B, int V) { return rules_chunk(cus, B, V); }
extern "C" int rows(int T, int heads, int groups) { return rotate_rows(T, heads, groups); }
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    folder = tmp_path_factory.mktemp("plans")
    (folder / "shim.cpp").write_text(SHIM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2505_12065_amd", "csrc"),
                           str(folder / "shim.cpp"), "-o", str(folder / "shim.so")])
    lib = ctypes.CDLL(str(folder / "shim.so"))
    lib.workspace.restype = ctypes.c_int64
    lib.workspace.argtypes = [ctypes.c_int] * 8 + [ctypes.c_int64]
    lib.attend.argtypes = [ctypes.c_int] * 9 + [ctypes.c_int64, ctypes.POINTER(ctypes.c_int64)]
    return lib


NAMES = ("groups", "splits", "chunk", "pad", "part", "once", "one", "step", "tiles", "lds", "keep")


def attend(lib, *args, most=1 << 30):
    out = (ctypes.c_int64 * len(NAMES))()
    lib.attend(256, *args, most, out)
    return dict(zip(NAMES, out))


def log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def test_attention_covers_every_slot_and_head(plans):
    rng = random.Random(1)
    for _ in range(4000):
        heads, G = log(rng, 1, 64), log(rng, 1, 100)
        B, d, eb, length = log(rng, 1, 4000), 8 * rng.randint(1, 32), rng.choice([2, 4]), log(rng, 1, 3_000_000)
        if heads * G > 8192:
            continue
        window, mass, most = rng.choice([0, 0, log(rng, 1, 100_000)]), rng.randint(0, 1), rng.choice([1 << 30, 1 << 30, 1 << 22])
        p = attend(plans, B, heads * G, heads, d, eb, length, window, mass, most=most)
        reach = min(length, window + 15) if window else length
        assert p["chunk"] % p["step"] == 0 and 1 <= p["splits"] <= 256 and p["pad"] == p["splits"] * p["chunk"]
        assert (p["splits"] - 1) * p["chunk"] < reach <= p["pad"]           # nothing left out, no part empty by construction
        assert p["groups"] * 16 * p["tiles"] >= G and (p["groups"] - 1) * 16 * p["tiles"] < G
        assert p["lds"] <= 160 * 1024 and 1 <= p["part"] <= B
        assert (p["one"] > 0) == (p["splits"] > 1 or (bool(mass) and not p["keep"]))
        if p["keep"]:                                     # all scores of a cache head, and room for a second workgroup
            assert mass and p["splits"] == p["groups"] == 1 and p["keep"] >= reach and p["keep"] * G * 4 <= 64 * 1024
        assert p["one"] * p["part"] <= most or p["part"] == 1
        assert p["part"] == 1 or p["part"] * heads * p["splits"] * p["groups"] <= 1 << 22


def test_attention_workspace_is_enough_for_all_that_is_shorter(plans):
    rng = random.Random(2)
    for _ in range(3000):
        heads, G = log(rng, 1, 32), log(rng, 1, 40)
        B, d, eb, length = log(rng, 1, 500), 8 * rng.randint(1, 32), rng.choice([2, 4]), log(rng, 1, 300_000)
        mass = rng.randint(0, 1)
        told = plans.workspace(256, B, heads * G, heads, d, eb, length, mass, 1 << 30)
        for shorter, window in ((length, 0), (rng.randint(1, length), 0), (length, rng.randint(1, length)), (log(rng, 1, length), log(rng, 1, length))):
            p = attend(plans, B, heads * G, heads, d, eb, shorter, window, mass)
            assert p["one"] * p["part"] <= told, (B, heads, G, d, eb, length, shorter, window, mass)


def test_only_what_is_read_once_and_large_is_read_past_the_cache(plans):
    assert attend(plans, 64, 64, 8, 128, 2, 9216, 0, 0)["once"] and not attend(plans, 1, 32, 8, 128, 2, 1500, 0, 0)["once"]
    assert not attend(plans, 64, 64, 8, 128, 2, 9216, 100, 0)["once"]       # a window of it is small
    assert attend(plans, 64, 128, 4, 128, 2, 9216, 0, 0)["once"] and not attend(plans, 64, 128, 2, 128, 2, 9216, 0, 0)["once"]   # 32 heads, 64 heads


def test_parts_of_the_logits_and_rows_of_a_token(plans):
    for B, V in ((1, 32_000), (33, 50_001), (192, 128_000), (1, 1), (513, 2049)):
        c = plans.chunk(256, B, V)
        assert c in (2048, 4096, 8192)
        assert c == 2048 or B * -(-V // c) >= 256
        assert c == 8192 or B * -(-V // (2 * c)) < 256
    for heads in range(3, 300):
        for groups in (8, 16, 32):
            few, many = plans.rows(511, heads, groups), plans.rows(512, heads, groups)
            assert few == 1 and 1 <= many <= 4
            parts = -(-heads // (groups * many))
            assert parts == -(-heads // (4 * groups))     # as few workgroups as with 4, evenly
