// Norms of queries and keys for each head, the rotation by position, and the write of keys and values into the cache.
//
// Every row is read once and written once, where it is wanted: some ten operations an element, so bytes bound it where there are many tokens, and the launch where
// there are few.  16000 tokens of 32 + 8 + 8 heads of 128, bf16 (0.40 GB): 75 us, 5.4 TB/s (a copy of as much: 4.9); 8 tokens: 2.9 us on the GPU, 5.2 a call.
#include "launch.hpp"
#include "paged.hpp"

namespace ann {

namespace {

constexpr int THREADS = 256;

// LPR lanes for a row (a head of a token), eight elements a lane.  A group of LPR lanes takes NR rows of one token, LANES / LPR heads apart:
// all are asked for at once, and what belongs to the token and the lane (cosines and sines, four times the bytes of a row at 16 bits) or to the lane
// alone (weights) is read once for all of them.
template <class T, int LPR, int NR, bool INTERLEAVED>
__global__ __launch_bounds__(THREADS) void qk_rotate_kernel(RotateArgs a) {
    constexpr int GROUPS = THREADS / LPR;
    const int d = a.cache.d, group = threadIdx.x / LPR, lane = threadIdx.x % LPR, e = 8 * lane;
    const int heads = a.q_heads + 2 * a.cache.heads, h0 = blockIdx.y * (GROUPS * NR) + group;
    const int64_t t = blockIdx.x;
    const int p = a.positions[t], slot = a.slots[t];
    const bool pad = (unsigned)p >= (unsigned)a.max_positions, mine = e < d;
    const int page = slot >> a.cache.slots_log, off = slot & ((1 << a.cache.slots_log) - 1);
    const bool stored = !pad && slot >= 0 && page < a.cache.pages;
    Eight<T> x[NR], wq, wk;
    const char *in = static_cast<const char *>(a.qkv) + t * a.token + e * T::bytes;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        x[r].zero();
        const int h = h0 + r * GROUPS;
        if (mine && !pad && h < heads) x[r].load(in + h * a.head);
    }
    wq.zero();
    wk.zero();
    if (mine) {
        wq.load(static_cast<const char *>(a.q_weight) + e * T::bytes);
        wk.load(static_cast<const char *>(a.k_weight) + e * T::bytes);
    }
    // cosine and sine of the lane's pairs; for pairs of halves its own eight, and the sine's sign is that of its half
    constexpr int PAIRS = INTERLEAVED ? 4 : 8;
    const bool turns = e < a.rot && !pad, low = e < a.rot / 2;
    float c[PAIRS], s[PAIRS];
    if (turns) {
        const float *table = a.cos_sin + (int64_t)p * a.rot + (INTERLEAVED ? e / 2 : low ? e : e - a.rot / 2);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            c[i] = table[i];
            s[i] = table[a.rot / 2 + i];
            if (!INTERLEAVED && low) s[i] = -s[i];
        }
    }
    const int other = turns ? lane + (low ? a.rot / 16 : -(a.rot / 16)) : lane;
    const float per_d = 1.f / (float)d;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int h = h0 + r * GROUPS;
        if (h >= heads) break;                            // (whole groups: lanes that exchange values stay together)
        const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.cache.heads;
        if (!is_v) {
            float y[8], w[8], sum = 0.f;
            x[r].get(y);
            (is_q ? wq : wk).get(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(y[i], y[i], sum);
#pragma unroll
            for (int k = 1; k < LPR; k *= 2) sum += __shfl_xor(sum, k);
            const float f = rsqrtf(fmaf(sum, per_d, a.eps));
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = y[i] * f * w[i];
            if (INTERLEAVED) {
                if (turns) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float u = y[2 * i], v = y[2 * i + 1];
                        y[2 * i] = u * c[i % PAIRS] - v * s[i % PAIRS];
                        y[2 * i + 1] = v * c[i % PAIRS] + u * s[i % PAIRS];
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float z = __shfl(y[i], other, LPR);
                    if (turns) y[i] = y[i] * c[i % PAIRS] + z * s[i % PAIRS];
                }
            }
            x[r].set(y);
        }
        if (!mine) continue;
        if (is_q) {
            if (pad) x[r].zero();
            x[r].store(static_cast<char *>(a.q) + ((t * a.q_heads + h) * d + e) * T::bytes);
        } else if (stored) {
            char *to = is_v ? a.cache.v + (int64_t)page * a.cache.v_page + (h - a.q_heads - a.cache.heads) * a.cache.v_head + off * a.cache.v_slot
                            : a.cache.k + (int64_t)page * a.cache.k_page + (h - a.q_heads) * a.cache.k_head + off * a.cache.k_slot;
            x[r].store(to + e * T::bytes);
        }
    }
}

template <class T, int LPR, int NR>
hipError_t launch(const RotateArgs &a, int T_, hipStream_t stream) {
    const int heads = a.q_heads + 2 * a.cache.heads, per = THREADS / LPR * NR;
    const dim3 grid(T_, (heads + per - 1) / per);
    if (a.interleaved) hipLaunchKernelGGL((qk_rotate_kernel<T, LPR, NR, true>), grid, dim3(THREADS), 0, stream, a);
    else hipLaunchKernelGGL((qk_rotate_kernel<T, LPR, NR, false>), grid, dim3(THREADS), 0, stream, a);
    return hipGetLastError();
}
template <class T, int LPR>
hipError_t launch(const RotateArgs &a, int T_, hipStream_t stream) {
    const int rows = rotate_rows(T_, a.q_heads + 2 * a.cache.heads, THREADS / LPR);
    return rows == 1 ? launch<T, LPR, 1>(a, T_, stream) : rows == 2 ? launch<T, LPR, 2>(a, T_, stream)
           : rows == 3 ? launch<T, LPR, 3>(a, T_, stream) : launch<T, LPR, 4>(a, T_, stream);
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
