// Norms of queries and keys for each head, the rotation by position, and the write of keys and values into the cache.
#include "launch.hpp"
#include "paged.hpp"

namespace ann {

namespace {

constexpr int THREADS = 256;

// LPR lanes for a row (a head of a token), eight elements a lane; a workgroup's rows are heads of one token.
template <class T, int LPR, bool INTERLEAVED>
__global__ __launch_bounds__(THREADS) void qk_rotate_kernel(RotateArgs a) {
    const int d = a.cache.d, group = threadIdx.x / LPR, lane = threadIdx.x % LPR, e = 8 * lane;
    const int heads = a.q_heads + 2 * a.cache.heads, h = blockIdx.y * (THREADS / LPR) + group;
    const int64_t t = blockIdx.x;
    if (h >= heads) return;                               // (whole rows: lanes that exchange values stay together)
    const int p = a.positions[t], slot = a.slots[t];
    const bool pad = (unsigned)p >= (unsigned)a.max_positions, mine = e < d;
    const int page = slot >> a.cache.slots_log, off = slot & ((1 << a.cache.slots_log) - 1);
    const bool stored = !pad && slot >= 0 && page < a.cache.pages;
    const bool is_q = h < a.q_heads, is_k = !is_q && h < a.q_heads + a.cache.heads;
    Eight<T> x;
    x.zero();
    if (mine && !pad) x.load(static_cast<const char *>(a.qkv) + t * a.token + h * a.head + e * T::bytes);
    if (is_q || is_k) {
        float y[8], w[8] = {}, sum = 0.f;
        x.get(y);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(y[i], y[i], sum);
#pragma unroll
        for (int s = 1; s < LPR; s *= 2) sum += __shfl_xor(sum, s);
        const float r = 1.f / sqrtf(sum / (float)d + a.eps);
        if (mine) {
            Eight<T> wx;
            wx.load(static_cast<const char *>(is_q ? a.q_weight : a.k_weight) + e * T::bytes);
            wx.get(w);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = y[i] * r * w[i];
        const bool turns = e < a.rot && !pad;
        const float *table = a.cos_sin + (int64_t)(pad ? 0 : p) * a.rot;
        if (INTERLEAVED) {
            if (turns) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float c = table[e / 2 + i], s = table[a.rot / 2 + e / 2 + i], u = y[2 * i], v = y[2 * i + 1];
                    y[2 * i] = u * c - v * s;
                    y[2 * i + 1] = v * c + u * s;
                }
            }
        } else {
            const bool low = e < a.rot / 2;
            const int other = turns ? lane + (low ? a.rot / 16 : -(a.rot / 16)) : lane, i0 = low ? e : e - a.rot / 2;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float z = __shfl(y[i], other, LPR);
                if (turns) {
                    const float c = table[i0 + i], s = table[a.rot / 2 + i0 + i];
                    y[i] = low ? y[i] * c - z * s : y[i] * c + z * s;
                }
            }
        }
        x.set(y);
    }
    if (!mine) return;
    if (is_q) {
        if (pad) x.zero();
        x.store(static_cast<char *>(a.q) + ((t * a.q_heads + h) * d + e) * T::bytes);
    } else if (stored) {
        char *to = is_k ? a.cache.k + (int64_t)page * a.cache.k_page + (h - a.q_heads) * a.cache.k_head + off * a.cache.k_slot
                        : a.cache.v + (int64_t)page * a.cache.v_page + (h - a.q_heads - a.cache.heads) * a.cache.v_head + off * a.cache.v_slot;
        x.store(to + e * T::bytes);
    }
}

template <class T, int LPR>
hipError_t launch(const RotateArgs &a, int T_, hipStream_t stream) {
    const int heads = a.q_heads + 2 * a.cache.heads, per = THREADS / LPR;
    const dim3 grid(T_, (heads + per - 1) / per);
    if (a.interleaved) hipLaunchKernelGGL((qk_rotate_kernel<T, LPR, true>), grid, dim3(THREADS), 0, stream, a);
    else hipLaunchKernelGGL((qk_rotate_kernel<T, LPR, false>), grid, dim3(THREADS), 0, stream, a);
    return hipGetLastError();
}
template <class T>
hipError_t launch(const RotateArgs &a, int T_, hipStream_t stream) {
    return a.cache.d <= 64 ? launch<T, 8>(a, T_, stream) : a.cache.d <= 128 ? launch<T, 16>(a, T_, stream) : launch<T, 32>(a, T_, stream);
}

}  // namespace

hipError_t launch_qk_rotate(int dtype, const RotateArgs &a, int T, hipStream_t stream) {
    return dtype == ANN_F16 ? launch<F16>(a, T, stream) : dtype == ANN_BF16 ? launch<BF16>(a, T, stream) : launch<F32>(a, T, stream);
}

}  // namespace ann
