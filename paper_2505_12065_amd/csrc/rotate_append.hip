// The position rotation of queries and keys, angles from frequencies, and keys and values put behind what each request holds in a paged cache.
//
// Every row is read once and written once: bytes bound it where there are many tokens, the launch and a chain of dependent reads (the token's request, its length, its
// page) where there are few: 14039 tokens, 32 + 8 + 8 heads of 128, bf16, 67.7 us (345 MB, 5.1 TB/s; a copy reaches 4.7 to 5.0), 8 tokens 3.2 us, 5.1 with the host's launch.  An angle is a
// product in 64 bits, taken in turns and less its whole ones before it is rounded: in 32 bits position 100 000 would be off by 2^-8.
#include "launch.hpp"
#include "packed.hpp"
#include "paged.hpp"

namespace ann {

namespace {

constexpr int THREADS = 256;

// A workgroup takes heads of one token, LPR lanes a row of eight elements a lane, NR rows for each group of lanes, which are asked for at once.  The cosines and sines of the token
// are made once, one pair to a thread, and shared in LDS.
template <class T, int LPR, int NR, bool INTERLEAVED>
__global__ __launch_bounds__(THREADS) void rotate_append_kernel(AppendArgs a) {
    constexpr int GROUPS = THREADS / LPR;
    __shared__ float s_cos[128], s_sin[128];
    const int d = a.cache.d, group = threadIdx.x / LPR, lane = threadIdx.x % LPR, e = 8 * lane;
    const int heads = a.q_heads + 2 * a.cache.heads, h0 = blockIdx.y * (GROUPS * NR) + group;
    const int64_t t = blockIdx.x;
    const bool mine = e < d;
    Eight<T> x[NR];
    const char *in = static_cast<const char *>(a.qkv) + t * a.token + e * T::bytes;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        x[r].zero();
        const int h = h0 + r * GROUPS;
        if (mine && h < heads) x[r].load(in + h * a.head);
    }
    const PackedToken token = packed_token(a.starts, a.requests, a.tokens, (int)t);
    if (token.request < 0) return;                        // (the whole workgroup: it is not a request's)
    const int64_t slot = (int64_t)max(a.lengths[token.request], 0) - token.left;
    const int p = a.positions ? a.positions[t] : (int)max(slot, (int64_t)-1);
    // (without positions of their own, tokens before the first slot have none)
    const bool pad = p < 0;
    int page = -1;
    if (!pad && slot >= 0 && (slot >> a.cache.slots_log) < a.width) page = a.table[(int64_t)token.request * a.width + (slot >> a.cache.slots_log)];
    const bool stored = (unsigned)page < (unsigned)a.cache.pages;
    const int off = (int)(slot & ((1 << a.cache.slots_log) - 1));
    if (threadIdx.x < a.rot / 2) {
        const double turns = (double)p * a.frequencies[threadIdx.x] * 0.15915494309189535;
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        s_cos[threadIdx.x] = c * a.amplitude;
        s_sin[threadIdx.x] = s * a.amplitude;
    }
    __syncthreads();
    constexpr int PAIRS = INTERLEAVED ? 4 : 8;
    const bool turns = e < a.rot, low = e < a.rot / 2;
    float c[PAIRS], s[PAIRS];
    if (turns) {
        const int first = INTERLEAVED ? e / 2 : low ? e : e - a.rot / 2;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            c[i] = s_cos[first + i];
            s[i] = s_sin[first + i];
            if (!INTERLEAVED && low) s[i] = -s[i];
        }
    }
    const int other = turns ? lane + (low ? a.rot / 16 : -(a.rot / 16)) : lane;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int h = h0 + r * GROUPS;
        if (h >= heads) break;                            // (whole groups: lanes that exchange values stay together)
        const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.cache.heads;
        if (!is_v) {
            float y[8];
            x[r].get(y);
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
            if (turns) x[r].set(y);                       // (the others keep their bits)
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
hipError_t launch(const AppendArgs &a, hipStream_t stream) {
    const int heads = a.q_heads + 2 * a.cache.heads, per = THREADS / LPR * NR;
    const dim3 grid(a.tokens, (heads + per - 1) / per);
    if (a.interleaved) hipLaunchKernelGGL((rotate_append_kernel<T, LPR, NR, true>), grid, dim3(THREADS), 0, stream, a);
    else hipLaunchKernelGGL((rotate_append_kernel<T, LPR, NR, false>), grid, dim3(THREADS), 0, stream, a);
    return hipGetLastError();
}
template <class T, int LPR>
hipError_t launch(const AppendArgs &a, hipStream_t stream) {
    const int rows = rotate_rows(a.tokens, a.q_heads + 2 * a.cache.heads, THREADS / LPR);
    return rows == 1 ? launch<T, LPR, 1>(a, stream) : rows == 2 ? launch<T, LPR, 2>(a, stream)
           : rows == 3 ? launch<T, LPR, 3>(a, stream) : launch<T, LPR, 4>(a, stream);
}
template <class T>
hipError_t launch(const AppendArgs &a, hipStream_t stream) {
    return a.cache.d <= 64 ? launch<T, 8>(a, stream) : a.cache.d <= 128 ? launch<T, 16>(a, stream) : launch<T, 32>(a, stream);
}

}  // namespace

hipError_t launch_rotate_append(int dtype, const AppendArgs &a, hipStream_t stream) {
    return dtype == ANN_F16 ? launch<F16>(a, stream) : dtype == ANN_BF16 ? launch<BF16>(a, stream) : launch<F32>(a, stream);
}

}  // namespace ann
