// Tokens of several requests one behind the other: request b has tokens starts[b] to starts[b + 1] - 1.
#pragma once

#include "common.hpp"

namespace ann {

// By a wave: how many of value(0), ..., value(n - 1), which ascend, are at most x.  64 of them are looked at at once, so one read tells for up to 64, two for up
// to 4096.  (Whatever the values are, the answer is in [0, n].)
template <class F>
__device__ __forceinline__ int count_up_to(F &&value, int n, int x) {
    const int lane = threadIdx.x & (WAVE - 1);
    int first = 0;
    while (n > 0) {
        const int step = (n + WAVE - 1) / WAVE, at = (lane + 1) * step - 1;
        const int c = (int)__popcll(__ballot(at < n && value(first + at) <= x));
        first += c * step;
        n = min(n - c * step, step - 1);
    }
    return first;
}

// starts[b] as far as it can be one
__device__ __forceinline__ int packed_start(const int32_t *starts, int b, int tokens) { return min(max(starts[b], 0), tokens); }

struct PackedToken {
    int request;                                          // -1: none
    int left;                                             // tokens of the request from this one on
};
__device__ __forceinline__ PackedToken packed_token(const int32_t *starts, int requests, int tokens, int t) {
    const int b = count_up_to([&](int i) { return packed_start(starts, i, tokens); }, requests + 1, t) - 1;
    if (b < 0 || b >= requests) return {-1, 0};
    return {b, packed_start(starts, b + 1, tokens) - t};
}

}  // namespace ann
