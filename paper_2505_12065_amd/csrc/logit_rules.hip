// Penalties for repeated tokens, biases and grammar masks on logits.
//
// The logits are read and written once.  What decides about a token is gathered beside them in LDS: a workgroup takes THREADS * 8 * R
// tokens of the vocabulary of one request, asks for their logits (eight of a lane lie together), goes through the request's history and
// biases while those are under way, and notes in a word for each token how often it was generated, whether it was seen, and its last bias.
// Every workgroup of a request reads the whole history, so there are as few as keep the machine busy (rules_chunk).
//
// Bytes are the bound, and the histories' share of instructions comes on top.  192 rows of 128000 bf16 logits, a mask each, histories of up to 8100 tokens, 64 biases (0.11 GB): 27 us, 3.9 TB/s;
// without histories and biases 16.5.  One row of 32000 fp32 logits: 4.5 us on the GPU, 5.6 a call.
#include <type_traits>

#include "launch.hpp"
#include "paged.hpp"

namespace ann {

namespace {

// the same 16 bytes from any address that its element may have
template <int ALIGN> struct Any;
template <> struct Any<2> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Any<4> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4))); };

template <class T> struct Scalar;
template <> struct Scalar<F16> { typedef _Float16 type; };
template <> struct Scalar<BF16> { typedef __bf16 type; };
template <> struct Scalar<F32> { typedef float type; };

template <class T>
__device__ __forceinline__ Eight<T> load_any(const void *p) {
    typedef typename Any<T::bytes>::type A;
    Eight<T> e;
    if constexpr (T::bytes == 2) {
        e.raw = *static_cast<const A *>(p);
    } else {
        e.raw[0] = static_cast<const A *>(p)[0];
        e.raw[1] = static_cast<const A *>(p)[1];
    }
    return e;
}
template <class T>
__device__ __forceinline__ void store_any(void *p, const Eight<T> &e) {
    typedef typename Any<T::bytes>::type A;
    if constexpr (T::bytes == 2) {
        *static_cast<A *>(p) = e.raw;
    } else {
        static_cast<A *>(p)[0] = e.raw[0];
        static_cast<A *>(p)[1] = e.raw[1];
    }
}

// -inf in the place of the elements whose bit is 0
template <class T>
__device__ __forceinline__ Eight<T> masked(Eight<T> x, uint32_t bits) {
    if constexpr (T::bytes == 2) {
        const uint32_t none = std::is_same_v<T, F16> ? 0xfc00fc00u : 0xff80ff80u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t low = (uint32_t)((int32_t)(bits << (31 - 2 * j)) >> 31), high = (uint32_t)((int32_t)(bits << (30 - 2 * j)) >> 31);
            const uint32_t keep = (low & 0xffffu) | (high & 0xffff0000u);
            x.raw[j] = (x.raw[j] & keep) | (none & ~keep);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x.raw[j / 4][j % 4] = (bits >> j) & 1 ? x.raw[j / 4][j % 4] : 0xff800000u;
    }
    return x;
}

// The word of a token: its count in the lowest CB bits, the mark of a token that was seen above them, and above that the number of its
// last bias plus 1, in the same word (LONG: in a word of its own, for histories whose counts leave no room).
template <class T, int THREADS, int R, bool LONG>
__global__ __launch_bounds__(THREADS) void logit_rules_kernel(RulesArgs a, int parts) {
    typedef typename Scalar<T>::type E;
    constexpr int CHUNK = THREADS * 8 * R, CB = LONG ? 24 : RULES_COUNT_BITS;
    constexpr uint32_t SEEN = 1u << CB, COUNT = SEEN - 1;
    extern __shared__ __align__(16) uint32_t word[];
    uint32_t *bias = LONG ? word + CHUNK : word;
    __shared__ float first_values[THREADS];               // of the first biases
    const int id = xcd_block(), b = id / parts, v0 = id % parts * CHUNK, m = min(CHUNK, a.V - v0), tid = threadIdx.x;
    const E *in = static_cast<const E *>(a.logits) + b * a.row + v0;
    E *out = static_cast<E *>(a.out) + b * a.out_row + v0;
    const int mask_row = a.masks ? a.mask_rows[b] : -1;
    // (bit v % 32 of word v / 32 is bit v % 8 of byte v / 8)
    const uint8_t *mask = (unsigned)mask_row < (unsigned)a.n_masks
                              ? reinterpret_cast<const uint8_t *>(a.masks + (int64_t)mask_row * ((a.V + 31) / 32)) + v0 / 8 : nullptr;
    Eight<T> x[R];
    uint32_t bits[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = (r * THREADS + tid) * 8;
        bits[r] = 0xffu;
        if (i + 8 <= m) {
            x[r] = load_any<T>(in + i);
            if (mask) bits[r] = mask[i / 8];
        }
    }
    const int n = max(0, min(a.lengths[b], a.T)), prompt = max(0, a.prompt[b]);
    const int32_t *tokens = a.tokens + (int64_t)b * a.T, *bias_tokens = a.bias_tokens + (int64_t)b * a.K;
    const float *bias_values = a.bias_values + (int64_t)b * a.K;
    const float repetition = a.repetition[b], presence = a.presence[b], frequency = a.frequency[b];
    constexpr int AHEAD = 2;                              // loads of the history under way at a time
    u4 told[AHEAD];
    auto ask = [&](int t0) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int t = t0 + u * 4 * THREADS;
            told[u] = u4{~0u, ~0u, ~0u, ~0u};             // (no token)
            if (t + 4 <= n) told[u] = *reinterpret_cast<const Any<4>::type *>(tokens + t);
        }
    };
    int rest = -1, biased = -1;                           // what the last whole four leave; the first biases
    if ((n & ~3) + tid < n) rest = tokens[(n & ~3) + tid];
    float worth = 0.f;
    if (tid < a.K) {
        biased = bias_tokens[tid];
        worth = bias_values[tid];
    }
    ask(4 * tid);
    for (int i = tid * 4; i < (LONG ? 2 * CHUNK : CHUNK); i += THREADS * 4) *reinterpret_cast<u4 *>(word + i) = zero_chunk();
    __syncthreads();
    if (a.K > 0) {
        first_values[tid] = worth;
        auto note_bias = [&](int i, int token) {
            if (token >= v0 && token - v0 < m) atomicMax(&bias[token - v0], LONG ? (uint32_t)i + 1 : (uint32_t)(i + 1) << (CB + 1));
        };
        note_bias(tid, biased);
        for (int i = tid + THREADS; i < a.K; i += THREADS) note_bias(i, bias_tokens[i]);
        if (!LONG) __syncthreads();                       // (a maximum of what the counts have not been added to)
    }
    // (a token below 0 is beyond the last of the part as an unsigned number: V < 2^31 - 2^15)
    auto note_seen = [&](uint32_t token) {
        if (token - (uint32_t)v0 < (uint32_t)m) atomicOr(&word[token - v0], SEEN);
    };
    auto note_told = [&](uint32_t token) {
        if (token - (uint32_t)v0 < (uint32_t)m) atomicAdd(&word[token - v0], 1u);
    };
    for (int t0 = 4 * tid; t0 < n; t0 += AHEAD * 4 * THREADS) {
        u4 w[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) w[u] = told[u];
        if (t0 + AHEAD * 4 * THREADS < n) ask(t0 + AHEAD * 4 * THREADS);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int t = t0 + u * 4 * THREADS;
            if (t >= prompt) {
#pragma unroll
                for (int i = 0; i < 4; ++i) note_told(w[u][i]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) t + i < prompt ? note_seen(w[u][i]) : note_told(w[u][i]);
            }
        }
    }
    (n & ~3) + tid < prompt ? note_seen((uint32_t)rest) : note_told((uint32_t)rest);
    __syncthreads();
    auto ruled = [&](float y, uint32_t w, uint32_t k, bool allowed) {
        if (w & (SEEN | COUNT)) {
            y = y > 0.f ? y / repetition : y * repetition;
            if (w & COUNT) y = y - frequency * (float)(w & COUNT) - presence;
        }
        if (k) y += k <= THREADS ? first_values[k - 1] : bias_values[k - 1];
        return allowed ? y : -INFINITY;
    };
    auto number = [&](int i) { return LONG ? bias[i] : word[i] >> (CB + 1); };
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = (r * THREADS + tid) * 8;
        if (i + 8 <= m) {
            const u4 w0 = *reinterpret_cast<const u4 *>(word + i), w1 = *reinterpret_cast<const u4 *>(word + i + 4);
            u4 k0 = zero_chunk(), k1 = zero_chunk();
            if (LONG) {
                k0 = *reinterpret_cast<const u4 *>(bias + i);
                k1 = *reinterpret_cast<const u4 *>(bias + i + 4);
            }
            const u4 any = w0 | w1 | k0 | k1;
            if (any[0] | any[1] | any[2] | any[3]) {
                float y[8];
                x[r].get(y);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t w = j < 4 ? w0[j & 3] : w1[j & 3], k = LONG ? (j < 4 ? k0[j & 3] : k1[j & 3]) : w >> (CB + 1);
                    y[j] = ruled(y[j], w, k, true);
                }
                x[r].set(y);
            }
            x[r] = masked<T>(x[r], bits[r]);
            store_any<T>(out + i, x[r]);
        } else {
            for (int j = i; j < m; ++j) out[j] = (E)ruled((float)in[j], word[j], number(j), !mask || ((mask[j / 8] >> (j & 7)) & 1));
        }
    }
}

template <class T, int THREADS, int R, bool LONG>
hipError_t launch(const RulesArgs &a, int B, hipStream_t stream) {
    constexpr int CHUNK = THREADS * 8 * R;
    constexpr size_t bytes = (size_t)CHUNK * (LONG ? 8 : 4);
    static_assert(bytes + THREADS * 4 <= 64 * 1024, "what a launch may take unasked");
    const int parts = (a.V + CHUNK - 1) / CHUNK;
    hipLaunchKernelGGL((logit_rules_kernel<T, THREADS, R, LONG>), dim3(parts * B), dim3(THREADS), bytes, stream, a, parts);
    return hipGetLastError();
}
template <class T>
hipError_t launch(const RulesArgs &a, int cus, int B, hipStream_t stream) {
    if (a.T >= 1 << RULES_COUNT_BITS) return launch<T, 512, 1, true>(a, B, stream);
    const int chunk = rules_chunk(cus, B, a.V);
    return chunk == 2048 ? launch<T, 256, 1, false>(a, B, stream) : chunk == 4096 ? launch<T, 512, 1, false>(a, B, stream)
           : launch<T, 512, 2, false>(a, B, stream);
}

}  // namespace

hipError_t launch_logit_rules(int dtype, int cus, const RulesArgs &a, int B, hipStream_t stream) {
    return dtype == ANN_F16 ? launch<F16>(a, cus, B, stream) : dtype == ANN_BF16 ? launch<BF16>(a, cus, B, stream) : launch<F32>(a, cus, B, stream);
}

}  // namespace ann
