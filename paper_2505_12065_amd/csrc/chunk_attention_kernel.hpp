// Attention of many rows (query heads of tokens) that read the same keys and values, on the matrix cores:
//     x_j = scale q k_j        out = sum over j of e^(x_j - m) v_j / sum over j of e^(x_j - m)        lse = m + ln(sum over j of e^(x_j - m)),
// in one pass over the slots j with a running m, by powers of 2: scale holds 1 / ln 2.
//
// A workgroup takes R rows of one request (or group of requests) and cache head and a part of the slots, KT of them at a time, in LDS.  Both products are turned so that
// rows of queries are the columns of every tile:
//     S^T [32 slots x 32 rows] = K Q^T          O^T [d x 32 rows] += V^T P^T
// Lane 32 h + m then has the scores of row m and slots 8 a + 4 h + i (a, i < 4), which is where the second product wants its operand P^T if its 16 columns are
// numbered 8 h + 4 a + i for slot 8 a + 4 h + i: nothing passes between lanes but a maximum, and maxima, sums and factors belong to the lane's own row.  V^T comes from the rows of V as they
// lie, by reads of LDS that turn 4 x 16 elements.
//
// What bounds it is the matrix cores, and the power that they and the exponentials draw: 16384 tokens from nothing, 32 heads of 128 to 8, bf16, take 2.09 to 2.23 ms by the card (1.05 to 0.99 PFLOP/s;
// a large library product reaches 1.36 on such data), at a clock of 1.8 GHz, the matrix cores busy for half of the time and the vector units for somewhat more; 24 passages of up to 300 tokens behind
// up to 8100 slots 347 to 388 us (0.82 to 0.73 PFLOP/s: a tenth goes to rows and slots that masks leave out, another to the last workgroups), d = 256 0.54 PFLOP/s, fp32 0.08 to 0.1 (a library product
// 0.15). With all values 0 the prompt takes 1880 us: the clock.
// Why so and not otherwise, the same prompt: 64 rows a wave do not fit its registers (3.5 ms); 256 rows a workgroup, 8 waves: no faster; four tiles of 32 slots in flight for two of 64: 2.75 ms; a
// tile's sums by dot products of packed weights for sums of 32 bits: 2145 us; a word of each line of the tile behind the next read ahead into the second cache: 2460.
#pragma once

#include <type_traits>

#include "chunk_rows.hpp"
#include "launch.hpp"
#include "paged.hpp"
#include "paged_attention_kernel.hpp"

namespace ann {

typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef unsigned short us2 __attribute__((ext_vector_type(2)));

#define ANN_LDS(p) ((__attribute__((address_space(3))) void *)(p))
#define ANN_ROW_TO_LDS(gptr, lptr) \
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(gptr), ANN_LDS(lptr), 16, 0, 0)

template <class T>
__device__ __forceinline__ void store_four(char *to, f4 y);
template <>
__device__ __forceinline__ void store_four<F32>(char *to, f4 y) { *reinterpret_cast<f4 *>(to) = y; }
template <>
__device__ __forceinline__ void store_four<F16>(char *to, f4 y) {
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<h4 *>(to) = h4{(_Float16)y[0], (_Float16)y[1], (_Float16)y[2], (_Float16)y[3]};
}
template <>
__device__ __forceinline__ void store_four<BF16>(char *to, f4 y) {
    typedef __bf16 b4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<b4 *>(to) = b4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
}
// From what the weights' exponents are less (the largest score as an exponent of 2, or one near it, less the lift) and their sum.  The sum's exponent is added to them before the product with ln 2: the lift is in
// both, and of two logarithms of its size that cancel each other lse would keep the roundings (16 bits, up to 2048 slots, scores of deviations from 0.3 to 2: off by 2.0e-6 to 2.8e-6 at most, 0.4e-6 to 1.4e-6 so).
__device__ __forceinline__ float chunk_lse(float less, float total) {
    int exponent;
    const float fraction = frexpf(total, &exponent);
    return total == 0.f ? -INFINITY : fmaf(less == -INFINITY ? 0.f : less + (float)exponent, 0.6931471805599453f, logf(fraction));
}

// until at most n of this wave's loads are outstanding
template <int n>
__device__ __forceinline__ void wait_outstanding() {
    static_assert(n >= 0 && n < 64, "vmcnt is a field of 6 bits");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (n & 15) | ((n >> 4) << 14));
    asm volatile("" ::: "memory");
}

// ---- the kernel ----------------------------------------------------------------------------------------------

template <class T, int DP_>
struct ChunkShape {
    static constexpr int DP = DP_, RB = DP * T::bytes;                  // largest d; bytes of a row in LDS
    static constexpr int KT = chunk_slots(RB, chunk_per_simd(DP)), WAVES = CHUNK_WAVES;
    static constexpr int CPR = RB / 16, RPI = 64 / CPR;                 // chunks of a row, rows that a load brings
    static constexpr int LOADS = KT * RB / 1024 / WAVES;                // of K, and of V, that a wave issues for a tile of slots
    static constexpr int TILE = KT * RB, LDS = 4 * TILE;                // K and V, twice
    static constexpr int NS = RB / 32, NC = DP / 32, NU = KT / 32;      // steps of 32 bytes of a row; tiles of 32 elements; tiles of 32 slots
};

// Where chunk c of row r lies in its row: 16 rows that an operand is read of lie in 16 places of the 256 bytes that the banks hold, and so do four rows of 64 bytes that are turned.
template <int RB>
__device__ __forceinline__ int chunk_swizzle(int r) {
    return RB == 128 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 3) : (r & 3) << 2 | ((r >> 2) & 3);
}

__device__ __forceinline__ f16v zero16() {
    f16v z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
}

template <class T>
__device__ __forceinline__ u4 pack_weights(const float *p);
template <>
__device__ __forceinline__ u4 pack_weights<BF16>(const float *p) {
    b8 x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (__bf16)p[i];
    return __builtin_bit_cast(u4, x);
}
template <>
__device__ __forceinline__ u4 pack_weights<F16>(const float *p) {
    h8 x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (_Float16)p[i];
    return __builtin_bit_cast(u4, x);
}

// Largest size among the words' elements, as bits, kept in `most`; whether that is none of a finite number.
template <class T>
__device__ __forceinline__ void most_bits(uint32_t w, uint32_t &most) {
    if constexpr (T::bytes == 2) {
        const us2 a = __builtin_bit_cast(us2, w & 0x7fff7fffu), b = __builtin_bit_cast(us2, most);
        most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(a, b));
    } else {
        most = max(most, w & 0x7fffffffu);
    }
}
template <class T>
__device__ __forceinline__ bool not_finite(uint32_t most) {
    constexpr uint32_t INF = std::is_same_v<T, F16> ? 0x7c00u : std::is_same_v<T, BF16> ? 0x7f80u : 0x7f800000u;
    if constexpr (T::bytes == 2) return (most & 0xffffu) >= INF || (most >> 16) >= INF;
    else return most >= INF;
}

// The elements of a word, 0 where they are not finite
template <class T>
__device__ __forceinline__ uint32_t finite_of(uint32_t w) {
    constexpr uint32_t INF = std::is_same_v<T, F16> ? 0x7c00u : std::is_same_v<T, BF16> ? 0x7f80u : 0x7f800000u;
    if constexpr (T::bytes == 2) return ((w & 0x7fffu) < INF ? w & 0xffffu : 0u) | (((w >> 16) & 0x7fffu) < INF ? w & 0xffff0000u : 0u);
    else return (w & 0x7fffffffu) < INF ? w : 0u;
}
// Four elements of a row, 0 where they are finite
template <class T>
__device__ __forceinline__ f4 not_finite_four(const char *p) {
    f4 y;
    if constexpr (T::bytes == 4) {
        y = *reinterpret_cast<const f4 *>(p);
    } else if constexpr (std::is_same_v<T, F16>) {
        typedef _Float16 h4 __attribute__((ext_vector_type(4)));
        const h4 x = *reinterpret_cast<const h4 *>(p);
        y = f4{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
    } else {
        typedef __bf16 b4 __attribute__((ext_vector_type(4)));
        const b4 x = *reinterpret_cast<const b4 *>(p);
        y = f4{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (__float_as_uint(y[i]) & 0x7fffffffu) < 0x7f800000u ? 0.f : y[i];
    return y;
}

// Slots of one row of a deal, of token t, the i-th of its sequence
__device__ __forceinline__ ChunkSpan chunk_row_span(const ChunkArgs &a, int mode, const ChunkDeal &deal, int t, int i) {
    if (mode == CHUNK_NEW) return chunk_span(a, deal.k.length, deal.k.q.tokens - i);
    return {deal.range.lo, mode == CHUNK_COMMON ? min(deal.range.hi, chunk_length(a, t)) : deal.range.hi};
}
// A row without other parts is divided and written; else what joins the parts reads its elements, its statistics, how many parts there are and whether it is of a group.
__device__ __forceinline__ bool chunk_whole(const ChunkArgs &a, const ChunkDeal &deal) { return a.splits == 1 || deal.alone; }
// Weights are 2^lift times what they are.  16 bits: by their exponents, before they are rounded, which are off by 2^-19 at most so (2^-8 and 2^-11 are the weights' own roundings).  fp32: exponents would be rounded to the lift's last place (20: 2^-20, and not the 2^-23 of those that count, which
// left outputs and statistics twice as far off): they are less by 2^-7, so that 64 slots' products are half as large as the largest value, and sums of these are multiplied by the rest.  (Half:
// weights are as far above 2^-7 as the largest score's exponent is rounded down, by 2^(2^-7) at scores of 100 000.)
constexpr float CHUNK_LIFT_F32 = -7.f;
// (a weight of 16 bits may pass the one of the score it goes by by 2^8, one of fp32 by nothing)
constexpr int CHUNK_ROOM_F32 = 8;
template <class T>
__device__ __forceinline__ float chunk_lift_exponent(const ChunkArgs &a) { return T::bytes == 4 ? CHUNK_LIFT_F32 : a.lift; }
template <class T>
__device__ __forceinline__ float chunk_lift_factor(const ChunkArgs &a) {
    return T::bytes == 4 ? __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((127 + CHUNK_ROOM_F32 + (int)(a.lift - CHUNK_LIFT_F32)) << 23)) : 1.f;
}
template <class T>
__device__ __forceinline__ float chunk_by(const ChunkArgs &a, float total) { return total == 0.f ? 0.f : 1.f / (total * chunk_lift_factor<T>(a)); }
__device__ __forceinline__ f4 chunk_divided(f4 y, float by) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = by == 0.f ? 0.f : y[i] * by;
    return y;
}
__device__ __forceinline__ int64_t chunk_place(const ChunkArgs &a, const ChunkPass &pass, const ChunkDeal &deal, int row) { return (int64_t)row * a.splits + pass.part0 + deal.part; }
__device__ __forceinline__ void chunk_statistics(const ChunkArgs &a, const ChunkPass &pass, const ChunkDeal &deal, int row, float most, float total) {
    if (a.splits > 1) *reinterpret_cast<f4 *>(a.stats + 4 * chunk_place(a, pass, deal, row)) = f4{most, total, __int_as_float(deal.parts), __int_as_float(deal.k.grouped)};
    if (a.lse && chunk_whole(a, deal)) a.lse[row] = chunk_lse(most, total);
}
// Four elements of a row: divided and written if the row has no other parts, else left for what joins them.
template <class T>
__device__ __forceinline__ void chunk_write(const ChunkArgs &a, const ChunkPass &pass, const ChunkDeal &deal, int row, int at, f4 y, float by) {
    if (!chunk_whole(a, deal)) {
        *reinterpret_cast<f4 *>(a.partial + chunk_place(a, pass, deal, row) * a.cache.d + at) = y;
        return;
    }
    store_four<T>(static_cast<char *>(a.out) + ((int64_t)row * a.cache.d + at) * T::bytes, chunk_divided(y, by));
}
// Row `in` of a deal, among those of all tokens.
__device__ __forceinline__ int chunk_row(const ChunkArgs &a, const ChunkDeal &deal, int head, int G, int in) {
    const int r = deal.r0 + in;
    return (deal.k.q.token0 + r / G) * a.q_heads + head * G + r % G;
}

// ---- 128 rows -------------------------------------------------------------------------------------------------

template <class T, int DP>
__global__ __launch_bounds__(CHUNK_WAVES * WAVE, chunk_per_simd(DP)) void chunk_attention_kernel(ChunkArgs a, ChunkPass pass) {
    typedef ChunkShape<T, DP> Sh;
    constexpr int KT = Sh::KT, RB = Sh::RB, NS = Sh::NS, NC = Sh::NC, NU = Sh::NU, LOADS = Sh::LOADS, CPR = Sh::CPR, RPI = Sh::RPI, WAVES = Sh::WAVES;
    constexpr bool WIDE = T::bytes == 4;
    constexpr float RISE = WIDE ? 0.f : 8.f;
    constexpr int AHEAD = DP == 128 ? 6 : 4;              // reads of LDS in flight before a product
    extern __shared__ __align__(16) unsigned char chunk_lds[];
    __shared__ int s_lo[WAVES], s_hi[WAVES], s_bad[2];
    const int lane = threadIdx.x & (WAVE - 1), m = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int G = a.q_heads / a.cache.heads, head = blockIdx.x % a.cache.heads;
    const ChunkDeal deal = chunk_deal(a, pass, blockIdx.x / a.cache.heads, G);
    if (deal.count <= 0) return;
    const int first = deal.first, end = deal.end;
    const int32_t *table = a.table + (int64_t)deal.k.q.request * a.width;
    const int slots_log = a.cache.slots_log, mask = (1 << slots_log) - 1;
    // the page of slot k0 + lane % KT, or -1
    auto look_up = [&](int k0) {
        const int key = k0 + (lane & (KT - 1));
        int page = -1;
        if (key < end) page = table[key >> slots_log];
        return (unsigned)page < (unsigned)a.cache.pages ? page : -1;
    };
    int pages = look_up(first), pages_next = look_up(first + KT);           // (asked for before the queries: they are waited for first)

    // this lane's row: its query and the slots that it attends to
    u4 q[NS];
    int lo = 0, hi = INT_MAX, hi_most = 0;
    const uint32_t flip = a.scale < 0.f ? (WIDE ? 0x80000000u : 0x80008000u) : 0u;
    const float scale = fmaxf(fabsf(a.scale), 1e-37f);    // (not 0: a score of -infinity stays one)
    const int row0 = wave * 32, row_bytes = a.cache.d * T::bytes;
    {
        const int in = row0 + m, r = deal.r0 + in, t = deal.k.q.token0 + r / G;
        const bool there = in < deal.count;
        const char *from = static_cast<const char *>(a.q) + t * a.q_row + (head * G + r % G) * a.q_head;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int at = (2 * s + h) * 16;
            q[s] = zero_chunk();
            if (there && at < row_bytes) q[s] = load_chunk(from + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) q[s][i] ^= flip;
        }
        if (there) {
            const ChunkSpan span = chunk_row_span(a, pass.mode, deal, t, r / G);
            lo = span.lo;
            hi = span.hi;
            hi_most = hi;
        }
    }
    int lo_most = lo, hi_least = hi;                      // of all rows of the wave
    lo_most = __builtin_amdgcn_readfirstlane(wave_max_of(lo_most));
    hi_least = __builtin_amdgcn_readfirstlane(-wave_max_of(-hi_least));
    hi_most = __builtin_amdgcn_readfirstlane(wave_max_of(hi_most));
    int all_lo = lo_most, all_hi = hi_least;              // ... of all waves that read the same slots
    {
        if (lane == 0) { s_lo[wave] = lo_most; s_hi[wave] = hi_least; }
        if (threadIdx.x == 0) { s_bad[0] = INT_MAX; s_bad[1] = -1; }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) { all_lo = max(all_lo, s_lo[w]); all_hi = min(all_hi, s_hi[w]); }
        all_lo = __builtin_amdgcn_readfirstlane(all_lo);
        all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    }

    unsigned char *const mine = chunk_lds;
    const char *k_head = a.cache.k + head * a.cache.k_head, *v_head = a.cache.v + head * a.cache.v_head;
    // Slots without a row take one of the first page's: their scores do not count, and of their values only that they are finite.
    const int first_row = wave * LOADS * RPI, in_load = lane / CPR, first_at = ((lane & (CPR - 1)) ^ chunk_swizzle<RB>(first_row + in_load)) * 16;
    auto issue = [&](int k0, int pages, unsigned char *to) __attribute__((always_inline)) {
        to += first_row * RB;
        auto coarse = [&](auto full) __attribute__((always_inline)) {       // the 16 rows from a multiple of 16 on are of one page, and a load's rows lie within 32 bits
#pragma unroll
            for (int e = 0; e < LOADS; ++e) {
                const int row = first_row + e * RPI, page = max(__builtin_amdgcn_readlane(pages, row & ~15), 0);
                const int64_t place = (k0 + row) & mask;
                const char *k = k_head + page * a.cache.k_page + place * a.cache.k_slot, *v = v_head + page * a.cache.v_page + place * a.cache.v_slot;
                // (the chunk's place goes by bits of the row: those of the first load's, turned by those of e)
                const uint32_t at = first_at ^ (chunk_swizzle<RB>(e * RPI) * 16);
                if (decltype(full)::value || (int)at < row_bytes) {
                    ANN_ROW_TO_LDS(k + (in_load * (uint32_t)a.cache.k_slot + at), to + e * 1024);
                    ANN_ROW_TO_LDS(v + (in_load * (uint32_t)a.cache.v_slot + at), to + Sh::TILE + e * 1024);
                }
            }
        };
        if (a.coarse) {
            if (row_bytes == RB) coarse(std::true_type{});
            else coarse(std::false_type{});
            return;
        }
#pragma unroll
        for (int e = 0; e < LOADS; ++e) {
            const int row = first_row + e * RPI + in_load, at = ((lane & (CPR - 1)) ^ chunk_swizzle<RB>(row)) * 16;
            const int page = max(__shfl(pages, row), 0);
            const int64_t place = (k0 + row) & mask;
            const char *k = k_head + page * a.cache.k_page + place * a.cache.k_slot + at, *v = v_head + page * a.cache.v_page + place * a.cache.v_slot + at;
            if (at < row_bytes) {
                ANN_ROW_TO_LDS(k, to + e * 1024);
                ANN_ROW_TO_LDS(v, to + Sh::TILE + e * 1024);
            }
        }
    };
    if (row_bytes < RB) {                                 // what lies behind the end of a row in LDS is never loaded
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int e = 0; e < LOADS; ++e) *reinterpret_cast<u4 *>(mine + b * Sh::TILE + first_row * RB + e * 1024 + lane * 16) = zero_chunk();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }

    f16v o[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) o[c] = zero16();
    // What exponents are less, of a score that the weights go by; the sum of this lane's slots alone.  (Everything that compares weights goes by this one rounded number, not by the score: they would differ by
    // its rounding, 2^-24 of a score times 1 / ln 2.)
    float off = -INFINITY, sum = 0.f;
    const int k_lane = m * RB, k_turn_of_lane = (h ^ chunk_swizzle<RB>(m)) << 4;    // a lane's part of the places of its operands
    const int i16 = lane & 15, v_row = 4 * h + (i16 >> 2), v_lane = v_row * RB;
    const int v_turn = ((2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) ^ chunk_swizzle<RB>(v_row)) << 4 | (i16 & 1) << 3;
    constexpr uint64_t ALL = KT == 64 ? ~0ull : (1ull << (KT & 63)) - 1;

    auto scores = [&](unsigned char *at_k, int k0, uint64_t seen, f16v (&x)[NU]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NU; ++u) x[u] = zero16();
        int k_turn = k_turn_of_lane;
        if constexpr (WIDE) asm volatile("" : "+v"(k_turn));   // (or the places of all operands stay in registers from tile to tile: at d = 256 93 were spilled, and 2 x 1024 tokens of 4096 took 2601 us, 1647 so)
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            if (WIDE && 32 * s >= row_bytes) break;       // (uniform; a product of 32 bits takes 16 times as long)
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const u4 k = *reinterpret_cast<const u4 *>(at_k + u * 32 * RB + k_lane + ((32 * s) ^ k_turn));
                if constexpr (WIDE) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[u] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[i]), __uint_as_float(q[s][i]), x[u], 0, 0, 0);
                } else {
                    x[u] = mfma32<T>(k, q[s], x[u]);
                }
            }
        }
        if constexpr (!WIDE) {                            // reads of K ahead of the products
            __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
            for (int r = 0; r < NU * NS - AHEAD; ++r) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
        }
        if (seen == ALL && k0 >= lo_most && k0 + KT <= hi_least) return;
#pragma unroll
        for (int u = 0; u < NU; ++u) {                    // which of this lane's slots its row attends to: bit 8 a + i for slot 8 a + 4 h + i
            const int from = lo - (k0 + 32 * u), to = hi - (k0 + 32 * u);
            uint32_t bits = (uint32_t)(seen >> (32 * u));
            bits = from <= 0 ? bits : from >= 32 ? 0u : bits & (~0u << from);
            bits = to >= 32 ? bits : to <= 0 ? 0u : bits & ~(~0u << to);
            bits >>= 4 * h;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (!((bits >> (8 * (i / 4) + i % 4)) & 1)) x[u][i] = -INFINITY;
        }
    };
    // Scores become weights; 16 bits: in p, as operands, rounded once.  (Two operands, what rounding the first leaves being the second, as where there are few rows and the matrix cores wait, would make the
    // matrix instructions that bound this loop half as many again.)
    auto weights = [&](f16v (&x)[NU], u4 (&p)[NU][2]) __attribute__((always_inline)) {
        float most = x[0][0];
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, x[u][i]);
        uint32_t b0, b1;
        row_pair<32>(__float_as_uint(most), b0, b1);
        most = fmaxf(__uint_as_float(b0), __uint_as_float(b1));
        // 16 bits: the largest score may pass the one that the weights go by by a factor of 2^8 before all that there is of the row is scaled again.
        const float next = fmaf(most, scale, -chunk_lift_exponent<T>(a));
        const bool rise = next - off > RISE;
        if (__ballot(rise)) {
            const float keep = rise ? exp2_fast(off - next) : 1.f;
            if (rise) off = next;
            sum *= keep;
#pragma unroll
            for (int c = 0; c < NC; ++c) o[c] *= keep;
        }
        const float less = off == -INFINITY ? 0.f : off;
        float tile = 0.f;                                 // (summed alone: a weight at a time, a sum of n of them may be off by n 2^-24)
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            float w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                w[i] = exp2_fast(fmaf(x[u][i], scale, -less));
                tile += w[i];
                if constexpr (WIDE) x[u][i] = w[i];
            }
            if constexpr (!WIDE) {
                p[u][0] = pack_weights<T>(w);
                p[u][1] = pack_weights<T>(w + 8);
            }
        }
        sum += tile;
    };
    auto times_v = [&](unsigned char *at_v, const f16v (&x)[NU], const u4 (&p)[NU][2]) __attribute__((always_inline)) {
        int m = lane & 31;
        if constexpr (WIDE) asm volatile("" : "+v"(m));
        // fp32: a tile's products are summed alone, as its weights are, since the matrix cores add two slots at a time to a sum: equal weights over 8192 slots left it 1.2e-4 off without (a
        // library product 3e-5).
        // (2 x 1024 tokens of 4096: d = 128 742 us, 667 without; d = 64 357 and 340.)
        if constexpr (WIDE) {
            const float up = chunk_lift_factor<T>(a);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if (32 * c >= a.cache.d) break;           // (uniform)
                f16v y = zero16();
#pragma unroll
                for (int u = 0; u < NU; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int row = 32 * u + 8 * (i / 4) + 4 * h + i % 4;
                        const float v = *reinterpret_cast<const float *>(at_v + row * RB + (((8 * c + (m >> 2)) ^ chunk_swizzle<RB>(row)) << 4) + (m & 3) * 4);
                        y = __builtin_amdgcn_mfma_f32_32x32x2f32(v, x[u][i], y, 0, 0, 0);
                    }
                o[c] += y * up;
            }
        } else {
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    unsigned char *from = at_v + (32 * u + 16 * j) * RB + v_lane;
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        typedef __attribute__((address_space(3))) s4 *Turned;
                        const u2 v0 = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Turned)ANN_LDS(from + ((64 * c) ^ v_turn))));
                        const u2 v1 = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Turned)ANN_LDS(from + 8 * RB + ((64 * c) ^ v_turn ^ 32))));
                        o[c] = mfma32<T>(u4{v0[0], v0[1], v1[0], v1[1]}, p[u][j], o[c]);
                    }
                }
        }
    };
    // Rows of V that some rows of queries attend to and others do not must be finite, or they would go into all: 0 times NaN is no 0.  What this wave loaded that is not is taken
    // out, and given to the rows that attend to it at the end.
    auto take_out = [&](unsigned char *at_v, int k0) __attribute__((always_inline)) {
        unsigned char *loaded = at_v + first_row * RB + lane * 16;
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < LOADS; ++e) {
            const u4 x = *reinterpret_cast<const u4 *>(loaded + e * 1024);
#pragma unroll
            for (int i = 0; i < 4; ++i) most_bits<T>(x[i], most);
        }
        if (!__ballot(not_finite<T>(most))) return;
#pragma unroll 1
        for (int e = 0; e < LOADS; ++e) {
            u4 x = *reinterpret_cast<const u4 *>(loaded + e * 1024);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = finite_of<T>(x[i]);
            *reinterpret_cast<u4 *>(loaded + e * 1024) = x;
        }
        if (lane == 0) {
            atomicMin(&s_bad[0], k0);
            atomicMax(&s_bad[1], k0);
        }
    };

    int k0 = first;
    int buffer = 0;
    uint64_t valid = 0;
    if (k0 < end) {
        issue(k0, pages, mine);
        valid = __ballot(pages >= 0) & ALL;
        pages = pages_next;
    }
    for (; k0 < end; k0 += KT, buffer ^= 1) {
        unsigned char *at_k = mine + buffer * 2 * Sh::TILE;
        wait_outstanding<0>();
        if (!(valid == ALL && k0 >= all_lo && k0 + KT <= all_hi)) take_out(at_k + Sh::TILE, k0);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // all waves' loads are there, and nobody reads the other buffer any more
        const uint64_t seen = valid;
        if (k0 + KT < end) {
            issue(k0 + KT, pages, mine + (buffer ^ 1) * 2 * Sh::TILE);
            valid = __ballot(pages >= 0) & ALL;
            pages = look_up(k0 + 2 * KT);
        }
        if (k0 >= hi_most) continue;                  // (no row of this wave's attends to it)
        f16v x[NU];
        u4 p[NU][2];
        scores(at_k, k0, seen, x);
        // Weights and their products go before another wave's scores, which need the matrix cores alone: of two waves on a SIMD one has something for each unit.  (A prompt of 16384 tokens, 32 heads of 128 to 8,
        // bf16: 2216 us without and 2105 with it; of 8192, 16 heads to 8, fp32: d = 128 2619 and 2550, d = 64 1309 and 1174; d = 64, bf16, 4 x 1024 of 8192 206 and 199, but 24 x 170 of 4400 235 and 241.)
        constexpr bool FIRST = chunk_per_simd(DP) > 1;
        if constexpr (FIRST) __builtin_amdgcn_s_setprio(1);
        weights(x, p);
        times_v(at_k + Sh::TILE, x, p);
        if constexpr (FIRST) __builtin_amdgcn_s_setprio(0);
    }
    __syncthreads();
    const int bad_first = s_bad[0], bad_last = s_bad[1];
#pragma unroll 1
    for (int k = bad_first; k <= bad_last; k += KT)
#pragma unroll 1
        for (int key = k; key < k + KT && key < end; ++key) {
            const int page = table[key >> slots_log];
            if ((unsigned)page >= (unsigned)a.cache.pages) continue;
            const char *from = v_head + page * a.cache.v_page + (key & mask) * a.cache.v_slot;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int at = 32 * c + 2 * i + 4 * h;
                    if (at >= a.cache.d || key < lo || key >= hi) continue;
                    const f4 v = not_finite_four<T>(from + at * T::bytes);
#pragma unroll
                    for (int b = 0; b < 4; ++b) o[c][i + b] += v[b];
                }
        }

    {
        uint32_t b0, b1;
        row_pair<32>(__float_as_uint(sum), b0, b1);
        sum = __uint_as_float(b0) + __uint_as_float(b1);
    }
    // Written by way of LDS, 32 or 64 elements of all the wave's rows at a time, so that eight lanes write 128 bytes of a row.  (A workgroup alone on its compute unit, two tiles: 2 us
    // of 9, instructions for the most part; 3 while every element's place, division and statistics were worked out where it was written.)
    constexpr int PER = WAVE / 8, CH = NC > 1 && WAVES * 32 * 68 * 4 <= Sh::LDS ? 2 : 1, LD = 32 * CH + 4;
    float *turn = reinterpret_cast<float *>(chunk_lds) + wave * 32 * LD;
    const int my_row = chunk_row(a, deal, head, G, min(row0 + m, deal.count - 1));
    const float my_by = chunk_by<T>(a, sum);
    if (h == 0 && row0 + m < deal.count) chunk_statistics(a, pass, deal, my_row, off, sum);
    auto write = [&](auto whole) __attribute__((always_inline)) {
        constexpr int BYTES = decltype(whole)::value ? T::bytes : 4;
        char *to[32 / PER];
        float by[32 / PER];
#pragma unroll
        for (int k = 0; k < 32 / PER; ++k) {
            const int in = k * PER + lane / 8, row = __shfl(my_row, in);
            by[k] = __shfl(my_by, in);
            if constexpr (decltype(whole)::value) to[k] = static_cast<char *>(a.out) + (int64_t)row * a.cache.d * BYTES;
            else to[k] = reinterpret_cast<char *>(a.partial + chunk_place(a, pass, deal, row) * a.cache.d);
            to[k] += lane % 8 * 4 * BYTES;
        }
#pragma unroll
        for (int c = 0; c < NC; c += CH) {
            if (32 * c >= a.cache.d) break;
#pragma unroll
            for (int cc = 0; cc < CH; ++cc)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<f4 *>(turn + m * LD + 32 * cc + 2 * i + 4 * h) = f4{o[c + cc][i], o[c + cc][i + 1], o[c + cc][i + 2], o[c + cc][i + 3]};
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");          // (what the wave itself wrote)
#pragma unroll
            for (int k = 0; k < 32 / PER; ++k) {
                const int in = k * PER + lane / 8;
#pragma unroll
                for (int cc = 0; cc < CH; ++cc) {
                    f4 y = *reinterpret_cast<const f4 *>(turn + in * LD + 32 * cc + lane % 8 * 4);
                    if (row0 + in >= deal.count || 32 * (c + cc) + lane % 8 * 4 >= a.cache.d) continue;
                    if constexpr (decltype(whole)::value) store_four<T>(to[k] + 32 * (c + cc) * BYTES, chunk_divided(y, by[k]));
                    else *reinterpret_cast<f4 *>(to[k] + 32 * (c + cc) * BYTES) = y;
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    };
    if (chunk_whole(a, deal)) write(std::true_type{});
    else write(std::false_type{});
}

// ---- few rows -------------------------------------------------------------------------------------------------
//
// Up to 16 MT rows: the waves share the slots out, K and V go from memory to registers, and the tiles are of 16 slots and 16 rows, as in paged_attention_kernel: reading K and V once bounds it
// (128 requests of 4096 slots, 64 heads of 128 to 8, bf16: 330 us, 6.5 TB/s; ragged ones of up to 2048 4.9 TB/s; fp32, 64 of 2048, 173 us, 6.1 TB/s);
// with little to read it is a chain of dependent reads (five requests behind 2000 slots in common, 32 heads to 8: 10 us).  A passage of 100 tokens, 400 rows of a cache head, takes 26.9 us
// so and 19.8 by 128 rows.
// Lane 16 g + m has the scores of row m and slots 4 g .. 4 g + 3 of a tile; weights are operands of two parts.  Both passes of groups go in one launch where both have few rows.
template <class T, int VE, int MT, bool FINE>
__global__ __launch_bounds__(CHUNK_WAVES * WAVE, chunk_few_per_simd(T::bytes, VE, MT)) void chunk_few_kernel(ChunkArgs a, ChunkPass first_pass, ChunkPass own_pass) {
    typedef AttendShape<T, VE> Sh;
    typedef typename Words<Sh::CW>::type VChunk;
    constexpr int NT = Sh::NT, NS = Sh::NS, NU = Sh::NU, CE = Sh::CE, WAVES = CHUNK_WAVES, STEP = 16 * NT * WAVES, ROWS = 16 * MT, LD = attend_lds_row(VE);
    extern __shared__ __align__(16) float few_lds[];
    __shared__ int s_row[ROWS];
    __shared__ float s_by[ROWS];
    const int lane = threadIdx.x & (WAVE - 1), g = lane >> 4, m = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int G = a.q_heads / a.cache.heads, head = blockIdx.x % a.cache.heads, item = blockIdx.x / a.cache.heads;
    const bool is_own = item >= first_pass.items;
    const ChunkPass &pass = is_own ? own_pass : first_pass;
    const ChunkDeal deal = chunk_deal(a, pass, is_own ? item - first_pass.items : item, G);
    if (deal.count <= 0) return;
    const int first = deal.first, end = deal.end, row_bytes = a.cache.d * T::bytes;
    const bool full = a.cache.d == 16 * VE;
    const uint32_t flip = a.scale < 0.f ? (T::bytes == 4 ? 0x80000000u : 0x80008000u) : 0u;
    const float scale = fmaxf(fabsf(a.scale), 1e-37f);

    float *s_top = few_lds, *s_sum = few_lds + WAVES * ROWS, *s_o = few_lds + 2 * WAVES * ROWS;
    constexpr bool Q_LDS = attend_q_in_lds(VE);
    u4 *s_q = reinterpret_cast<u4 *>(s_o), q[Q_LDS ? 1 : MT][Q_LDS ? 1 : NS];
    int lo[MT], hi[MT], lo_most = 0, hi_least = INT_MAX;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int in = 16 * mt + m, r = deal.r0 + in, t = deal.k.q.token0 + r / G;
        const bool there = in < deal.count;
        const char *from = static_cast<const char *>(a.q) + t * a.q_row + (head * G + r % G) * a.q_head;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int at = (4 * s + g) * 16;
            u4 x = zero_chunk();
            if (there && at < row_bytes) x = load_chunk(from + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] ^= flip;
            if constexpr (!Q_LDS) q[mt][s] = x;
            else if ((mt * NS + s) % WAVES == wave) s_q[(mt * NS + s) * WAVE + lane] = x;
        }
        lo[mt] = 0;
        hi[mt] = INT_MAX;
        if (there) {
            const ChunkSpan span = chunk_row_span(a, pass.mode, deal, t, r / G);
            lo[mt] = span.lo;
            hi[mt] = span.hi;
        }
        lo_most = max(lo_most, lo[mt]);
        hi_least = min(hi_least, hi[mt]);
    }
#pragma unroll
    for (int i = 1; i < 16; i *= 2) {
        lo_most = max(lo_most, __shfl_xor(lo_most, i));
        hi_least = min(hi_least, __shfl_xor(hi_least, i));
    }
    lo_most = __builtin_amdgcn_readfirstlane(lo_most);
    hi_least = __builtin_amdgcn_readfirstlane(hi_least);

    const int32_t *table = a.table + (int64_t)deal.k.q.request * a.width;
    const int slots_log = a.cache.slots_log, mask = (1 << slots_log) - 1;
    const char *k_head = a.cache.k + head * a.cache.k_head, *v_head = a.cache.v + head * a.cache.v_head;
    auto row_page = [&](int key) {
        int page = -1;
        if (key < end) page = table[key >> slots_log];
        return (unsigned)page < (unsigned)a.cache.pages ? page : -1;
    };
    // pages of tiles, looked up a step ahead; -1: none.  FINE: of the lane's row of K, and of its four rows of V
    struct Pages { int k[NT], v[NT][FINE ? 4 : 1]; };
    Pages page, page_next;
    u4 kr[NT][NS];
    auto pages_of = [&](int k0, Pages &out) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (!FINE) {
                out.k[t] = __builtin_amdgcn_readfirstlane(row_page(k0 + 16 * t));
                continue;
            }
            out.k[t] = row_page(k0 + 16 * t + m);
#pragma unroll
            for (int i = 0; i < (FINE ? 4 : 1); ++i) out.v[t][i] = row_page(k0 + 16 * t + 4 * g + i);
        }
    };
    auto load_k = [&](int k0, const Pages &pg) __attribute__((always_inline)) {
        auto load = [&](auto whole, auto once) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int p = max(pg.k[t], 0);
                const char *row = k_head + (int64_t)p * a.cache.k_page + ((k0 + 16 * t + m) & mask) * a.cache.k_slot;
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const int at = (4 * s + g) * 16;
                    if (decltype(whole)::value || at < row_bytes) kr[t][s] = stream_load<decltype(once)::value>(reinterpret_cast<const u4 *>(row + at));
                    else kr[t][s] = zero_chunk();
                }
            }
        };
        if (full && pass.once) load(std::true_type{}, std::true_type{});
        else if (full) load(std::true_type{}, std::false_type{});
        else load(std::false_type{}, std::false_type{});
    };

    f4 o[MT][VE];
    float top[MT], sum[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int c = 0; c < VE; ++c) o[mt][c] = f4{0.f, 0.f, 0.f, 0.f};
        top[mt] = -INFINITY;
        sum[mt] = 0.f;
    }
    int k0 = first + wave * 16 * NT, bad_first = INT_MAX, bad_last = -1;
    if (k0 < end) {
        pages_of(k0, page);
        load_k(k0, page);
    }
    if constexpr (Q_LDS) __syncthreads();
    for (; k0 < end; k0 += STEP) {
        const bool more = k0 + STEP < end;
        if (more) pages_of(k0 + STEP, page_next);
        VChunk vr[NT][4][NU];
        auto load_v = [&](auto whole, auto once) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int p = max(FINE ? page.v[t][FINE ? i : 0] : page.k[t], 0);
                    const char *row = v_head + (int64_t)p * a.cache.v_page + ((k0 + 16 * t + 4 * g + i) & mask) * a.cache.v_slot;
#pragma unroll
                    for (int u = 0; u < NU; ++u) {
                        const int at = (u * 16 + m) * CE;
                        if (decltype(whole)::value || at < a.cache.d) vr[t][i][u] = stream_load<decltype(once)::value>(reinterpret_cast<const VChunk *>(row + at * T::bytes));
                        else vr[t][i][u] = VChunk(0);
                    }
                }
        };
        if (full && pass.once) load_v(std::true_type{}, std::true_type{});
        else if (full) load_v(std::true_type{}, std::false_type{});
        else load_v(std::false_type{}, std::false_type{});
        if constexpr (Q_LDS) asm volatile("" ::: "memory");                 // (the queries stay where they are)
        f4 x[MT][NT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                x[mt][t] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < NS; ++s) x[mt][t] = scores_step<T>(kr[t][s], Q_LDS ? s_q[(mt * NS + s) * WAVE + lane] : q[Q_LDS ? 0 : mt][Q_LDS ? 0 : s], x[mt][t]);
            }
        if (more) load_k(k0 + STEP, page_next);
        bool whole = k0 >= lo_most && k0 + 16 * NT <= hi_least && k0 + 16 * NT <= end;
#pragma unroll
        for (int t = 0; t < NT; ++t) whole = whole && page.k[t] >= 0;
        if (FINE || !whole) {                             // slots that do not count, for all rows or for some: no score, and values that are numbers
            uint32_t most = 0;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = k0 + 16 * t + 4 * g + i;
                    const bool there = (FINE ? page.v[t][FINE ? i : 0] : page.k[t]) >= 0 && key < end;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
                        if (!there || key < lo[mt] || key >= hi[mt]) x[mt][t][i] = -INFINITY;
#pragma unroll
                    for (int u = 0; u < NU; ++u) {
                        if (!there) vr[t][i][u] = VChunk(0);
#pragma unroll
                        for (int w = 0; w < Sh::CW; ++w) most_bits<T>(vr[t][i][u][w], most);
                    }
                }
            // (infinities and NaN are given to the rows that attend to them at the end: 0 times NaN is no 0)
            if (__ballot(not_finite<T>(most))) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int u = 0; u < NU; ++u)
#pragma unroll
                            for (int w = 0; w < Sh::CW; ++w) vr[t][i][u][w] = finite_of<T>(vr[t][i][u][w]);
                bad_first = min(bad_first, k0);
                bad_last = k0;
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {                 // x becomes the weights
            float most = x[mt][0][0];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) most = fmaxf(most, x[mt][t][i]);
            const float now = fmaxf(top[mt], fmaf(column_max(most), scale, -chunk_lift_exponent<T>(a))), keep = top[mt] == now ? 1.f : exp2_fast(top[mt] - now), less = now == -INFINITY ? 0.f : now;
            top[mt] = now;                                // (as by many rows: what exponents are less)
            float tile = 0.f;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[mt][t][i] = exp2_fast(fmaf(x[mt][t][i], scale, -less));
                    tile += x[mt][t][i];
                }
            sum[mt] = sum[mt] * keep + tile;
#pragma unroll
            for (int c = 0; c < VE; ++c) o[mt][c] *= keep;
        }
        if constexpr (T::bytes == 2) {
#pragma unroll
            for (int t = 0; t < NT; t += 2) {
                u4 high[MT], low[MT];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const f4 x0 = x[mt][t], x1 = x[mt][t + 1];
                    const float w[8] = {x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]};
                    split_weights<T>(w, high[mt], low[mt]);
                }
#pragma unroll
                for (int u = 0; u < NU; ++u)
#pragma unroll
                    for (int c = 0; c < CE; ++c) {
                        u4 v;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            v[k] = __builtin_amdgcn_perm(vr[t + k / 2][2 * (k & 1) + 1][u][c / 2], vr[t + k / 2][2 * (k & 1)][u][c / 2], c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            f4 &acc = o[mt][u * CE + c];
                            acc = mfma16<T>(v, high[mt], acc);
                            acc = mfma16<T>(v, low[mt], acc);
                        }
                    }
            }
        } else {                                          // (a step's products summed alone, as by many rows)
            static_assert(16 * NT <= 64, "as the lift is for");
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
                for (int c = 0; c < CE; ++c)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        f4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int i = 0; i < 4; ++i) y = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[t][i][u][c]), x[mt][t][i], y, 0, 0, 0);
                        o[mt][u * CE + c] += y * chunk_lift_factor<T>(a);
                    }
        }
        page = page_next;
    }
#pragma unroll 1
    for (int k = bad_first; k <= bad_last; k += STEP)
#pragma unroll 1
        for (int key = k; key < k + 16 * NT && key < end; ++key) {
            const int p = row_page(key);
            if (p < 0) continue;
            const char *from = v_head + (int64_t)p * a.cache.v_page + (key & mask) * a.cache.v_slot;
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < CE; c += 4) {
                        const int at = (u * 16 + 4 * g + i) * CE + c;
                        if (at >= a.cache.d) continue;
                        const f4 v = not_finite_four<T>(from + at * T::bytes);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
                            if (key >= lo[mt] && key < hi[mt]) {
#pragma unroll
                                for (int b = 0; b < 4; ++b) o[mt][u * CE + c + b][i] += v[b];
                            }
                    }
        }

    // the waves' sums, joined (of those that had a slot): lane 16 g + m holds elements CE (4 g + i) .. of every 16 CE, row 16 mt + m
    const int used = min(WAVES, (max(end - first, 1) + 16 * NT - 1) / (16 * NT));
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        sum[mt] = column_sum(sum[mt]);
        if (g == 0) {
            s_top[wave * ROWS + 16 * mt + m] = top[mt];
            s_sum[wave * ROWS + 16 * mt + m] = sum[mt];
        }
    }
    __syncthreads();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int in = 16 * mt + m;
        float all = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) all = fmaxf(all, s_top[w * ROWS + in]);
        const float f = top[mt] == -INFINITY ? 1.f : exp2_fast(top[mt] - all);          // (a row without a score has zeros, or NaN)
        if (in < deal.count && wave < used) {
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < CE; c += 4) {
                        const int at = (u * 16 + 4 * g + i) * CE + c, e = u * CE + c;
                        *reinterpret_cast<f4 *>(s_o + (wave * deal.count + in) * LD + at) = f4{o[mt][e][i], o[mt][e + 1][i], o[mt][e + 2][i], o[mt][e + 3][i]} * f;
                    }
        }
    }
    if ((int)threadIdx.x < deal.count) {                  // (wave 0: what belongs to a row)
        const int in = threadIdx.x, row = chunk_row(a, deal, head, G, in);
        float most = -INFINITY, total = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = fmaxf(most, s_top[w * ROWS + in]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float t = s_top[w * ROWS + in];
            total += s_sum[w * ROWS + in] * (t == -INFINITY ? 1.f : exp2_fast(t - most));
        }
        s_row[in] = row;
        s_by[in] = chunk_by<T>(a, total);
        chunk_statistics(a, pass, deal, row, most, total);
    }
    __syncthreads();
    const int per_row = a.cache.d / 4;
    for (int i = threadIdx.x; i < deal.count * per_row; i += WAVES * WAVE) {
        const int in = i / per_row, at = i % per_row * 4;
        f4 y = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < used; ++w) y += *reinterpret_cast<const f4 *>(s_o + (w * deal.count + in) * LD + at);
        chunk_write<T>(a, pass, deal, s_row[in], at, y, s_by[in]);
    }
}

// What the parts of a row left, joined by a wave (bytes, or the launch: 34 MB of parts 8.6 us, the smallest 3.5; a join by the last workgroup of a row would want memory that is cleared
// beforehand), whose lanes share the parts out where a row takes fewer than there are.  The first part of a pass says how many there are, and the one of own slots whether
// the row is in a group.
template <class T>
__global__ __launch_bounds__(256) void chunk_join_kernel(ChunkArgs a, int own_part0, bool new_tokens) {
    const int lane = threadIdx.x & (WAVE - 1), d = a.cache.d;
    const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / WAVE;
    if (row >= (int64_t)a.tokens * a.q_heads) return;
    const f4 *stats = reinterpret_cast<const f4 *>(a.stats) + row * a.splits;
    // (of parts that are not there too, which are at most 128; what they hold is not looked at)
    const f4 s0 = lane < a.splits ? stats[lane] : f4{0.f, 0.f, 0.f, 0.f}, s1 = lane + WAVE < a.splits ? stats[lane + WAVE] : f4{0.f, 0.f, 0.f, 0.f};
    if (new_tokens && packed_token(a.starts, a.requests, a.tokens, (int)(row / a.q_heads)).request < 0) return;
    auto word = [&](int s, int i) { return __builtin_amdgcn_readlane(__float_as_int(s < WAVE ? s0[i] : s1[i]), s & (WAVE - 1)); };
    // (no more than there is room for, whatever the groups' starts are)
    auto parts = [&](int s, int most) { return min(max(word(s, 2), 0), most); };
    int parts0 = 0, parts1 = 0;
    if (new_tokens) {
        parts0 = parts(0, a.splits);
        if (parts0 == 1) return;                          // (it is written)
    } else {
        parts1 = parts(own_part0, a.splits - own_part0);
        if (own_part0 > 0 && word(own_part0, 3)) parts0 = parts(0, own_part0);
    }
    auto there = [&](int s) { return s < parts0 || (s >= own_part0 && s < own_part0 + parts1); };
    float most = fmaxf(there(lane) ? s0[0] : -INFINITY, there(lane + WAVE) ? s1[0] : -INFINITY);
    most = wave_max(most);
    // (a part without a score has a sum of 0, or NaN, and counts as it is)
    const float f0 = !there(lane) ? 0.f : s0[0] == -INFINITY ? 1.f : exp2_fast(s0[0] - most), f1 = !there(lane + WAVE) ? 0.f : s1[0] == -INFINITY ? 1.f : exp2_fast(s1[0] - most);
    const float total = wave_sum((there(lane) ? s0[1] * f0 : 0.f) + (there(lane + WAVE) ? s1[1] * f1 : 0.f));
    // lanes of a row: the power of two from d / 4 on
    const int per = d <= 32 ? 8 : d <= 64 ? 16 : d <= 128 ? 32 : 64, at = 4 * (lane % per), n = parts0 + parts1;
    const float *from = a.partial + row * a.splits * d + at;
    f4 y = {0.f, 0.f, 0.f, 0.f};
    constexpr int AHEAD = 8;
    for (int i0 = 0; i0 < n; i0 += AHEAD * WAVE / per) {
        f4 z[AHEAD];
        float f[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = i0 + k * (WAVE / per) + lane / per, s = i < parts0 ? i : own_part0 + i - parts0;
            const float g0 = __shfl(f0, s & (WAVE - 1)), g1 = __shfl(f1, s & (WAVE - 1));
            const bool ok = i < n && at < d;
            z[k] = ok ? *reinterpret_cast<const f4 *>(from + (int64_t)s * d) : f4{0.f, 0.f, 0.f, 0.f};
            f[k] = !ok ? 0.f : s < WAVE ? g0 : g1;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) y += z[k] * f[k];
    }
    for (int i = per; i < WAVE; i *= 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] += __shfl_xor(y[j], i);
    }
    if (lane >= per || at >= d) return;
    store_four<T>(static_cast<char *>(a.out) + (row * d + at) * T::bytes, chunk_divided(y, chunk_by<T>(a, total)));
    if (lane == 0 && a.lse) a.lse[row] = chunk_lse(most, total);
}

template <class T, int DP>
hipError_t chunk_more(const ChunkArgs &a, const ChunkPass &pass, hipStream_t stream) {
    static size_t granted = 0;
    constexpr int bytes = ChunkShape<T, DP>::LDS;
    if (hipError_t e = allow_big_lds(reinterpret_cast<const void *>(chunk_attention_kernel<T, DP>), bytes, &granted)) return e;
    hipLaunchKernelGGL((chunk_attention_kernel<T, DP>), dim3((unsigned)((int64_t)pass.items * a.cache.heads)), dim3(CHUNK_WAVES * WAVE), bytes, stream, a, pass);
    return hipGetLastError();
}
template <class T, int VE, int MT, bool FINE>
hipError_t chunk_few(const ChunkArgs &a, const ChunkPass &first, const ChunkPass &own, hipStream_t stream) {
    static size_t granted = 0;
    const size_t bytes = attend_lds_bytes(T::bytes, VE, MT, 16 * MT, 0);
    if (hipError_t e = allow_big_lds(reinterpret_cast<const void *>(chunk_few_kernel<T, VE, MT, FINE>), bytes, &granted)) return e;
    hipLaunchKernelGGL((chunk_few_kernel<T, VE, MT, FINE>), dim3((unsigned)((int64_t)(first.items + own.items) * a.cache.heads)), dim3(CHUNK_WAVES * WAVE), bytes, stream, a, first, own);
    return hipGetLastError();
}
template <class T, int VE>
hipError_t chunk_few(const ChunkArgs &a, const ChunkPass &first, const ChunkPass &own, int rows, hipStream_t stream) {
    const bool fine = a.cache.slots_log < 4;
    if constexpr (chunk_few_rows(T::bytes, VE, 32) == 32)
        if (rows == 32) return fine ? chunk_few<T, VE, 2, true>(a, first, own, stream) : chunk_few<T, VE, 2, false>(a, first, own, stream);
    return fine ? chunk_few<T, VE, 1, true>(a, first, own, stream) : chunk_few<T, VE, 1, false>(a, first, own, stream);
}
template <class T, int VE>
hipError_t chunk_launch(const ChunkArgs &a, const ChunkPlan &pl, hipStream_t stream) {
    if (pl.first.rows <= 32) return chunk_few<T, VE>(a, pl.first, pl.own, pl.first.rows, stream);
    if (hipError_t e = chunk_more<T, 16 * VE>(a, pl.first, stream)) return e;
    return pl.own.items ? chunk_few<T, VE>(a, ChunkPass{}, pl.own, pl.own.rows, stream) : hipSuccess;
}
template <class T>
hipError_t launch_chunk(const ChunkArgs &a, const ChunkPlan &pl, hipStream_t stream) {
    const int ve = attend_ve(a.cache.d);
    if (hipError_t e = ve == 4 ? chunk_launch<T, 4>(a, pl, stream) : ve == 8 ? chunk_launch<T, 8>(a, pl, stream) : chunk_launch<T, 16>(a, pl, stream)) return e;
    if (a.splits == 1) return hipSuccess;
    const int64_t rows = (int64_t)a.tokens * a.q_heads;
    hipLaunchKernelGGL((chunk_join_kernel<T>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, a, pl.own.part0, pl.first.mode == CHUNK_NEW);
    return hipGetLastError();
}

}  // namespace ann
