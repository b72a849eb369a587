// Attention of many rows (query heads of tokens) over paged caches.
#pragma once

#include "launch.hpp"
#include "packed.hpp"
#include "paged.hpp"

namespace ann {

constexpr int CHUNK_THREADS = 256;

// The slots lo .. hi - 1 that a token attends to, of request `request` (-1: it is none's).
struct ChunkSpan { int request, lo, hi; };
__device__ __forceinline__ ChunkSpan chunk_span(const ChunkArgs &a, int t) {
    if (a.starts) {
        const PackedToken token = packed_token(a.starts, a.requests, a.tokens, t);
        if (token.request < 0) return {-1, 0, 0};
        const int slot = max(a.lengths[token.request], 0) - token.left;
        if (slot < 0 || slot >= a.max_length) return {token.request, 0, 0};
        return {token.request, a.window > 0 ? max(slot + 1 - a.window, 0) : 0, slot + 1};
    }
    const int n = min(max(a.lengths[t], 0), a.max_length);
    const int g = count_up_to([&](int i) { return a.group_starts[i]; }, a.groups + 1, t) - 1;
    const int common = g < 0 || g >= a.groups ? 0 : min(min(max(a.shared[g], 0), a.max_shared), n);
    return {t, 0, common + min(n - common, a.max_own)};
}

// A wave to a row, a slot at a time.  Weights are as small as the number of slots is large before they meet the values: sums of the largest would overflow before they are divided.
constexpr float LIFT = 0x1p-32f;
template <class T>
__global__ __launch_bounds__(CHUNK_THREADS) void chunk_attention_kernel(ChunkArgs a) {
    const int lane = threadIdx.x & (WAVE - 1), e = 8 * lane, d = a.cache.d, mask = (1 << a.cache.slots_log) - 1;
    const int64_t rows = (int64_t)a.tokens * a.q_heads;
    for (int64_t r = (int64_t)blockIdx.x * (CHUNK_THREADS / WAVE) + threadIdx.x / WAVE; r < rows; r += (int64_t)gridDim.x * (CHUNK_THREADS / WAVE)) {
        const int t = (int)(r / a.q_heads), hq = (int)(r % a.q_heads), h = hq / (a.q_heads / a.cache.heads);
        const ChunkSpan span = chunk_span(a, t);
        if (span.request < 0) continue;
        Eight<T> x;
        float q[8], o[8] = {}, most = -INFINITY, total = 0.f;
        x.zero();
        if (e < d) x.load(static_cast<const char *>(a.q) + t * a.q_row + hq * a.q_head + e * T::bytes);
        x.get(q);
        for (int j = span.lo; j < span.hi; ++j) {
            const int page = a.table[(int64_t)span.request * a.width + (j >> a.cache.slots_log)];
            if ((unsigned)page >= (unsigned)a.cache.pages) continue;
            float k[8], v[8], s = 0.f;
            x.zero();
            if (e < d) x.load(a.cache.k + (int64_t)page * a.cache.k_page + h * a.cache.k_head + (j & mask) * a.cache.k_slot + e * T::bytes);
            x.get(k);
            x.zero();
            if (e < d) x.load(a.cache.v + (int64_t)page * a.cache.v_page + h * a.cache.v_head + (j & mask) * a.cache.v_slot + e * T::bytes);
            x.get(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(q[i], k[i], s);
#pragma unroll
            for (int i = 1; i < WAVE; i *= 2) s += __shfl_xor(s, i);
            s *= a.scale;
            const float now = fmaxf(most, s), base = now == -INFINITY ? 0.f : now, keep = exp2f(most - base), w = exp2f(s - base);
            most = now;
            total = total * keep + w;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = fmaf(w * LIFT, v[i], o[i] * keep);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = total == 0.f ? 0.f : o[i] / (total * LIFT);
        x.set(o);
        if (e < d) x.store(static_cast<char *>(a.out) + (r * d + e) * T::bytes);
        if (lane == 0 && a.lse) a.lse[r] = total == 0.f ? -INFINITY : (most == -INFINITY ? 0.f : most) * 0.6931471805599453f + logf(total);
    }
}

template <class T>
hipError_t launch_chunk(const ChunkArgs &a, hipStream_t stream) {
    const int64_t groups = ((int64_t)a.tokens * a.q_heads + CHUNK_THREADS / WAVE - 1) / (CHUNK_THREADS / WAVE);
    hipLaunchKernelGGL((chunk_attention_kernel<T>), dim3((unsigned)(groups < (1 << 20) ? groups : 1 << 20)), dim3(CHUNK_THREADS), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ann
