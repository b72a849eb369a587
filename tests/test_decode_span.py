"""Which slots of a request attention goes through, decided without a GPU: the arithmetic of plan.hpp that the kernels run too, compiled with the C++
compiler alone and checked over the whole range of lengths and windows."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = r"""
#include "plan.hpp"
extern "C" void span(int length, int max_length, int window, int chunk, int *out) {
    const ann::AttendSpan s = ann::attend_span(length, max_length, window, chunk);
    out[0] = s.n, out[1] = s.lo, out[2] = s.start, out[3] = s.parts;
}
// of all lengths up to `longest`: the most LDS that a workgroup is to have, and how many plans keep scores there
extern "C" void lds(int B, int heads, int G, int d, int elem_bytes, int longest, int64_t *out) {
    out[0] = out[1] = 0;
    for (int length = 1; length <= longest; ++length) {
        const ann::AttendPlan p = ann::attend_plan(256, B, heads * G, heads, d, elem_bytes, length, 0, true, (size_t)1 << 30);
        const int ve = ann::attend_ve(d);
        const int64_t bytes = ann::attend_lds_bytes(elem_bytes, ve, ann::attend_head_tiles(elem_bytes, ve, G), G, p.keep);
        out[0] = out[0] < bytes ? bytes : out[0], out[1] += p.keep > 0;
    }
}
extern "C" int end(int n, int first, int chunk) { return ann::attend_end(n, first, chunk); }
extern "C" void plan(int heads, int G, int d, int elem_bytes, int max_length, int window, int mass, int64_t *out) {
    const ann::AttendPlan p = ann::attend_plan(256, 1, heads * G, heads, d, elem_bytes, max_length, window, mass != 0, (size_t)1 << 30);
    out[0] = p.chunk, out[1] = p.splits, out[2] = p.pad, out[3] = p.grid, out[4] = ann::ATTEND_GRID_ONE, out[5] = p.keep;
}
"""
LEAST, MOST = -2 ** 31, 2 ** 31 - 1
LONGEST = MOST - 65536                                    # what a page table may hold
LENGTHS = [LEAST, LEAST + 1, LEAST + 1000, -65536, -1000, -3, -1, 0, 1, 2, 15, 16, 17, 100, 1499, 1500, 1501, 65536, MOST - 1, MOST]
WINDOWS = [0, 1, 2, 15, 16, 17, 999, 1001, 1500, 65535, 2 ** 30, MOST - 1, MOST]


@pytest.fixture(scope="module")
def span(tmp_path_factory):
    folder = tmp_path_factory.mktemp("span")
    (folder / "shim.cpp").write_text(SHIM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fwrapv", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2505_12065_amd", "csrc"),
                           str(folder / "shim.cpp"), "-o", str(folder / "shim.so")])
    lib = ctypes.CDLL(str(folder / "shim.so"))
    out = (ctypes.c_int * 4)()

    def call(*args):
        lib.span(*args, out)
        return list(out)
    call.lib = lib
    return call


@pytest.mark.parametrize("max_length,chunk", [(1, 128), (1500, 128), (1500, 256), (65536, 1024), (1_000_000, 3328)])
def test_span(span, max_length, chunk):
    """No length and no window reaches a slot before the first or behind the last; a negative length is none."""
    for length in LENGTHS:
        for window in WINDOWS:
            n, lo, start, parts = span(length, max_length, window, chunk)
            assert n == max(0, min(length, max_length)), (length, window)
            assert lo == (max(0, n - window) if window else 0), (length, window)
            assert start == lo - lo % 16 and parts == -(-(n - start) // chunk), (length, window)


@pytest.mark.parametrize("d,elem_bytes", [(8, 2), (64, 4), (128, 2), (128, 4), (256, 2), (256, 4)])
def test_parts_of_the_longest_contexts(span, d, elem_bytes):
    """Every slot is in one part, for contexts whose length and part together pass 2^31."""
    out = (ctypes.c_int64 * 6)()
    for max_length in (LONGEST, LONGEST - 1, LONGEST - 15, LONGEST - 8_000_000, 2 ** 30, 2 ** 30 + 1):
        for window in (0, max_length, max_length - 1, max_length - 17, 2 ** 30, MOST):
            span.lib.plan(1, 4, d, elem_bytes, max_length, window, 1, out)
            chunk, splits, pad = out[:3]
            assert pad == splits * chunk <= MOST - 2048
            for length in (max_length, max_length - 1, max_length - 16, max_length - chunk):
                n, lo, start, parts = span(length, max_length, window, chunk)
                assert n == length and parts == -(-(n - start) // chunk) <= splits, (max_length, window, length)
                assert start + (splits - 1) * chunk <= MOST               # (parts that this request has not are looked at too)
                reached = start
                for part in range(parts):
                    end = span.lib.end(n, reached, chunk)
                    assert end == min(n, reached + chunk) > reached
                    reached = end
                assert reached == n


def test_launches_of_one_request(span):
    """The second launch has a workgroup for 1024 slots of a cache head, so the most heads and the longest contexts together are more than a launch may have:
    what the plan counts is never less than either launch, and a call is refused from where 256 threads to a workgroup would pass 2^32."""
    out, refused = (ctypes.c_int64 * 6)(), 0
    for heads in (1, 7, 8, 9, 64, 1024, 8192):
        for length in (1, 1500, 2 ** 20, 2 ** 28, LONGEST):
            for mass in (0, 1):
                span.lib.plan(heads, 1, 128, 2, length, 0, mass, out)
                chunk, splits, pad, grid, most, keep = out
                assert grid >= heads * splits and grid >= (heads if splits > 1 else 0) + (heads * -(-pad // 1024) if mass and not keep else 0)
                assert most * 256 < 2 ** 32
                refused += grid > most
                assert mass or grid <= most
    assert 0 < refused < 20


@pytest.mark.parametrize("elem_bytes", [2, 4])
@pytest.mark.parametrize("B,heads", [(1, 1), (64, 8)])
def test_no_workgroup_has_more_lds_than_there_is(span, elem_bytes, B, heads):
    """Over all numbers of query heads that one workgroup may take and beyond, all sizes of a head, and all lengths whose scores may stay in LDS."""
    out, kept = (ctypes.c_int64 * 2)(), 0
    for G in range(1, 41):
        for d in range(8, 257, 8):
            span.lib.lds(B, heads, G, d, elem_bytes, 4400, out)
            assert out[0] <= 160 * 1024, (G, d)
            kept += out[1]
    assert kept > 0
