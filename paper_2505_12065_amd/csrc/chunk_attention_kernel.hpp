// Attention of many rows (query heads of tokens) that read the same keys and values, on the matrix cores.
//
// A workgroup takes R rows of one request (or group of requests) and cache head and a part of the slots, KT of them at a time, in LDS.  Both products are turned so that
// rows of queries are the columns of every tile:
//     S^T [32 slots x 32 rows] = K Q^T          O^T [d x 32 rows] += V^T P^T
// Lane 32 h + m then has the scores of row m and slots 8 a + 4 h + i (a, i < 4), which is where the second product wants its operand P^T if its 16 columns are
// numbered 8 h + 4 a + i for slot 8 a + 4 h + i: nothing passes between lanes but a maximum, and maxima, sums and factors belong to the lane's own row.  V^T comes from the rows of V as they
// lie, by reads of LDS that turn 4 x 16 elements.
#pragma once

#include <type_traits>

#include "launch.hpp"
#include "packed.hpp"
#include "paged.hpp"

namespace ann {

typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef unsigned short us2 __attribute__((ext_vector_type(2)));

#define ANN_LDS(p) ((__attribute__((address_space(3))) void *)(p))
#define ANN_ROW_TO_LDS(gptr, lptr) \
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(gptr), ANN_LDS(lptr), 16, 0, 0)

// ---- which rows and slots ---------------------------------------------------------------------------------

// A tile: rows r0 .. r0 + count - 1 of a sequence of tokens (a request's new ones, the one of each request of a group, or one), the first of which is token0; a token has a row for
// each query head of the cache head.  `request`: whose page table is read.
struct ChunkTile { int token0, tokens, sequence, request, r0, count; };

__device__ __forceinline__ int chunk_start(const ChunkArgs &a, int i) { return packed_start(a.mode == CHUNK_NEW ? a.starts : a.group_starts, i, a.tokens); }
// The tile of sequence i that row r of it is in.
__device__ __forceinline__ ChunkTile chunk_tile(const ChunkArgs &a, int i, int64_t r, int G, int R) {
    const int s0 = a.mode == CHUNK_OWN ? i : chunk_start(a, i), s1 = a.mode == CHUNK_OWN ? i + 1 : chunk_start(a, i + 1);
    const int64_t r0 = r / R * R, rows = (int64_t)max(s1 - s0, 0) * G;
    return {s0, max(s1 - s0, 0), i, a.mode == CHUNK_COMMON ? min(s0, a.tokens - 1) : i, (int)r0, (int)max((int64_t)0, min((int64_t)R, rows - r0))};
}
// Tile number id.  A sequence of n tokens has at most as many tiles as there are numbers from start G / R + i up to the next one's.
__device__ __forceinline__ ChunkTile chunk_tile(const ChunkArgs &a, int id, int G, int R) {
    if (a.mode == CHUNK_OWN) {
        const int per = (G + R - 1) / R, i = id / per;
        return i < a.tokens ? chunk_tile(a, i, (int64_t)(id % per) * R, G, R) : ChunkTile{0, 0, 0, 0, 0, 0};
    }
    const int n = a.mode == CHUNK_NEW ? a.requests : a.groups;
    auto first = [&](int i) { return (int)((int64_t)chunk_start(a, i) * G / R) + i; };
    const int i = count_up_to(first, n + 1, id) - 1;
    return i >= 0 && i < n ? chunk_tile(a, i, (int64_t)(id - first(i)) * R, G, R) : ChunkTile{0, 0, 0, 0, 0, 0};
}
__device__ __forceinline__ int chunk_length(const ChunkArgs &a, int request) { return max(a.lengths[request], 0); }
// The group that request t is in, or -1.
__device__ __forceinline__ int chunk_group(const ChunkArgs &a, int t) {
    const int g = count_up_to([&](int i) { return packed_start(a.group_starts, i, a.tokens); }, a.groups + 1, t) - 1;
    return g < a.groups ? g : -1;
}
__device__ __forceinline__ int chunk_common(const ChunkArgs &a, int g) { return g < 0 ? 0 : min(max(a.shared[g], 0), a.max_shared); }

struct ChunkSpan { int lo, hi; };                         // slots lo .. hi - 1
// ... that the token `left` from the end of a request of `length` slots attends to
__device__ __forceinline__ ChunkSpan chunk_span(const ChunkArgs &a, int length, int left) {
    const int slot = length - left;
    if (slot < 0 || slot >= a.max_length) return {0, 0};
    return {a.window > 0 ? max(slot + 1 - a.window, 0) : 0, slot + 1};
}
// ... that all rows of a tile attend to something in
__device__ __forceinline__ ChunkSpan chunk_range(const ChunkArgs &a, const ChunkTile &tile, int G) {
    const int length = chunk_length(a, tile.request);
    if (a.mode == CHUNK_NEW) {
        const int first = length - (tile.tokens - tile.r0 / G), last = length - (tile.tokens - (tile.r0 + tile.count - 1) / G);
        return {a.window > 0 ? max(first + 1 - a.window, 0) : 0, min(max(last + 1, 0), a.max_length)};
    }
    if (a.mode == CHUNK_COMMON) return {0, chunk_common(a, tile.sequence)};
    const int n = min(length, a.max_length), common = min(n, chunk_common(a, chunk_group(a, tile.token0)));
    return {common, common + min(n - common, a.max_own)};
}
// Parts begin with multiples of 32 slots, so that the rows that a load brings are one page's or many's.
__device__ __forceinline__ int chunk_begin(const ChunkSpan &range) { return min(range.lo, range.hi) & ~31; }
__device__ __forceinline__ int chunk_parts(const ChunkSpan &range, int chunk) {
    return range.hi > chunk_begin(range) ? (range.hi - chunk_begin(range) - 1) / chunk + 1 : 1;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

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
// From the largest score, as an exponent of 2, and the sum of weights, 2^lift times as large.
__device__ __forceinline__ float chunk_lse(float most, float total, float lift) {
    return total == 0.f ? -INFINITY : ((most == -INFINITY ? 0.f : most) - lift) * 0.6931471805599453f + logf(total);
}

// ---- the kernel ----------------------------------------------------------------------------------------------

template <class T, int DP_, int NR_, bool SPLIT_>
struct ChunkShape {
    static constexpr int DP = DP_, NR = NR_, RB = DP * T::bytes;        // largest d; row tiles of a wave; bytes of a row in LDS
    static constexpr bool SPLIT = SPLIT_;                               // the waves take slots of their own of the same rows; else rows of their own of the same slots
    static constexpr int KT = chunk_slots(RB, SPLIT), WAVES = chunk_waves(RB, SPLIT), THREADS = WAVES * WAVE;
    static constexpr int R = 32 * NR * (SPLIT ? 1 : WAVES);             // rows of a workgroup
    static constexpr int CPR = RB / 16, RPI = 64 / CPR;                 // chunks of a row, rows that a load brings
    static constexpr int LOADS = KT * RB / 1024 / (SPLIT ? 1 : WAVES);  // of K, and of V, that a wave issues for a tile
    static constexpr int TILE = KT * RB, BUFFER = 2 * TILE;             // K, then V
    static constexpr int LDS = 2 * BUFFER * (SPLIT ? WAVES : 1);
    static constexpr int NS = RB / 32, NC = DP / 32, NU = KT / 32;      // steps of 32 bytes of a row; tiles of 32 elements; tiles of 32 slots
    static constexpr int SUB = NR == 1 ? NU : 1;                        // tiles of 32 slots at a time, as registers allow
    static constexpr int PER_SIMD = chunk_per_simd(T::bytes, DP);
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

template <class T, int DP, int NR, bool SPLIT>
__global__ __launch_bounds__((ChunkShape<T, DP, NR, SPLIT>::THREADS), (ChunkShape<T, DP, NR, SPLIT>::PER_SIMD)) void chunk_attention_kernel(ChunkArgs a) {
    typedef ChunkShape<T, DP, NR, SPLIT> Sh;
    constexpr int KT = Sh::KT, RB = Sh::RB, NS = Sh::NS, NC = Sh::NC, NU = Sh::NU, LOADS = Sh::LOADS, CPR = Sh::CPR, RPI = Sh::RPI, WAVES = Sh::WAVES, R = Sh::R, SUB = Sh::SUB;
    constexpr bool WIDE = T::bytes == 4;
    constexpr int AHEAD = DP == 128 && !SPLIT ? 6 : 4;    // reads of LDS in flight before a product
    extern __shared__ __align__(16) unsigned char chunk_lds[];
    __shared__ int s_lo[8], s_hi[8], s_bad[2];
    const int lane = threadIdx.x & (WAVE - 1), m = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int G = a.q_heads / a.cache.heads;
    const int head = blockIdx.x % a.cache.heads, item = blockIdx.x / a.cache.heads, part = item / a.tiles, id = a.tiles - 1 - item % a.tiles;
    const ChunkTile tile = chunk_tile(a, id, G, R);
    if (tile.count <= 0) return;
    const ChunkSpan range = chunk_range(a, tile, G);
    if (part >= chunk_parts(range, a.chunk)) return;      // (the first part of nothing says so)
    const int first = chunk_begin(range) + part * a.chunk, end = range.hi - first < a.chunk ? range.hi : first + a.chunk;

    // this lane's rows: their queries and the slots that they attend to
    u4 q[NR][NS];
    int lo[NR], hi[NR], lo_most = 0, hi_least = INT_MAX, hi_most = 0;
    const uint32_t flip = a.scale < 0.f ? (WIDE ? 0x80000000u : 0x80008000u) : 0u;
    const float scale = fmaxf(fabsf(a.scale), 1e-37f);    // (not 0: a score of -infinity stays one)
    const int row0 = SPLIT ? 0 : wave * NR * 32;          // of the tile
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
        const int in = row0 + rt * 32 + m, r = tile.r0 + in, t = tile.token0 + r / G;
        const bool there = in < tile.count;
        const char *from = static_cast<const char *>(a.q) + t * a.q_row + (head * G + r % G) * a.q_head;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int at = (2 * s + h) * 16;
            q[rt][s] = zero_chunk();
            if (there && at < a.cache.d * T::bytes) q[rt][s] = load_chunk(from + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) q[rt][s][i] ^= flip;
        }
        lo[rt] = 0;
        hi[rt] = INT_MAX;
        if (there) {
            ChunkSpan span = range;
            if (a.mode == CHUNK_NEW) span = chunk_span(a, chunk_length(a, tile.request), tile.tokens - r / G);
            if (a.mode == CHUNK_COMMON) span.hi = min(span.hi, chunk_length(a, t));
            lo[rt] = span.lo;
            hi[rt] = span.hi;
            hi_most = max(hi_most, span.hi);
        }
        lo_most = max(lo_most, lo[rt]);
        hi_least = min(hi_least, hi[rt]);
    }
#pragma unroll
    for (int i = 1; i < WAVE; i *= 2) {
        lo_most = max(lo_most, __shfl_xor(lo_most, i));
        hi_least = min(hi_least, __shfl_xor(hi_least, i));
        hi_most = max(hi_most, __shfl_xor(hi_most, i));
    }
    lo_most = __builtin_amdgcn_readfirstlane(lo_most);
    hi_least = __builtin_amdgcn_readfirstlane(hi_least);
    hi_most = __builtin_amdgcn_readfirstlane(hi_most);
    int all_lo = lo_most, all_hi = hi_least;              // of all waves that read the same slots
    if constexpr (!SPLIT) {
        if (lane == 0) { s_lo[wave] = lo_most; s_hi[wave] = hi_least; }
        if (threadIdx.x == 0) { s_bad[0] = INT_MAX; s_bad[1] = -1; }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) { all_lo = max(all_lo, s_lo[w]); all_hi = min(all_hi, s_hi[w]); }
        all_lo = __builtin_amdgcn_readfirstlane(all_lo);
        all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    }

    unsigned char *mine = chunk_lds + (SPLIT ? wave * 2 * Sh::BUFFER : 0);
    const int32_t *table = a.table + (int64_t)tile.request * a.width;
    const int slots_log = a.cache.slots_log, mask = (1 << slots_log) - 1, row_bytes = a.cache.d * T::bytes;
    const char *k_head = a.cache.k + head * a.cache.k_head, *v_head = a.cache.v + head * a.cache.v_head;
    // the page of slot k0 + lane % KT, or -1
    auto look_up = [&](int k0) {
        const int key = k0 + (lane & (KT - 1));
        int page = -1;
        if (key < end) page = table[key >> slots_log];
        return (unsigned)page < (unsigned)a.cache.pages ? page : -1;
    };
    // Slots without a row take one of the first page's: their scores do not count, and of their values only that they are finite.
    const int first_row = (SPLIT ? 0 : wave * LOADS) * RPI;
    const int in_load = lane / CPR, first_at = ((lane & (CPR - 1)) ^ chunk_swizzle<RB>(first_row + in_load)) * 16;
    const uint32_t k_load = in_load * (uint32_t)a.cache.k_slot, v_load = in_load * (uint32_t)a.cache.v_slot;
    auto issue = [&](int k0, int pages, int buffer) {
        unsigned char *to = mine + buffer * Sh::BUFFER + (SPLIT ? 0 : wave * LOADS * 1024);
        auto coarse = [&](auto full) __attribute__((always_inline)) {       // the 16 rows from a multiple of 16 on are of one page, and a load's rows lie within 32 bits
#pragma unroll
            for (int e = 0; e < LOADS; ++e) {
                const int row0 = first_row + e * RPI, page = max(__builtin_amdgcn_readlane(pages, row0 & ~15), 0);
                const int64_t place = (k0 + row0) & mask;
                const char *k = k_head + page * a.cache.k_page + place * a.cache.k_slot, *v = v_head + page * a.cache.v_page + place * a.cache.v_slot;
                // (the chunk's place goes by bits of the row: those of the first load's, turned by those of e)
                const uint32_t at = first_at ^ (chunk_swizzle<RB>(e * RPI) * 16);
                if (decltype(full)::value || (int)at < row_bytes) {
                    ANN_ROW_TO_LDS(k + (k_load + at), to + e * 1024);
                    ANN_ROW_TO_LDS(v + (v_load + at), to + Sh::TILE + e * 1024);
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
        for (int e = 0; e < 4 * LOADS; ++e)
            *reinterpret_cast<u4 *>(mine + (e / LOADS) * Sh::TILE + (first_row / RPI + e % LOADS) * 1024 + lane * 16) = zero_chunk();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }

    f16v o[NR][NC];
    float top[NR], sum[NR];                               // largest score so far, as the weights go by it; the sum of this lane's slots alone
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
#pragma unroll
        for (int c = 0; c < NC; ++c) o[rt][c] = zero16();
        top[rt] = -INFINITY;
        sum[rt] = 0.f;
    }
    const int sw = chunk_swizzle<RB>(m);
    const int k_lane = m * RB, k_turn = (h ^ sw) << 4;    // a lane's part of the places of its operands
    const int i16 = lane & 15, v_row = 4 * h + (i16 >> 2), v_lane = v_row * RB;
    const int v_turn = ((2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) ^ chunk_swizzle<RB>(v_row)) << 4 | (i16 & 1) << 3;

    constexpr int STEP = SPLIT ? WAVES * KT : KT;
    constexpr uint64_t ALL = KT == 64 ? ~0ull : (1ull << (KT & 63)) - 1;
    int k0 = first + (SPLIT ? wave * KT : 0), buffer = 0, pages = -1, bad_first = INT_MAX, bad_last = -1;
    uint64_t valid = 0;
    if (k0 < end) {
        pages = look_up(k0);
        issue(k0, pages, 0);
        valid = __ballot(pages >= 0) & ALL;
        pages = look_up(k0 + STEP);
    }
    for (; k0 < end; k0 += STEP, buffer ^= 1) {
        unsigned char *at_k = mine + buffer * Sh::BUFFER, *at_v = at_k + Sh::TILE;
        __builtin_amdgcn_s_waitcnt(0x0F70);               // this tile is there: vmcnt 0
        asm volatile("" ::: "memory");
        // Rows of V that some rows of queries attend to and others do not must be finite, or they would go into all: 0 times NaN is no 0.  What is not is taken
        // out, and given to the rows that attend to it at the end.
        if (!(valid == ALL && k0 >= all_lo && k0 + KT <= all_hi)) {
            unsigned char *loaded = at_v + (SPLIT ? 0 : wave * LOADS * 1024) + lane * 16;
            uint32_t most = 0;
#pragma unroll
            for (int e = 0; e < LOADS; ++e) {
                const u4 x = *reinterpret_cast<const u4 *>(loaded + e * 1024);
#pragma unroll
                for (int i = 0; i < 4; ++i) most_bits<T>(x[i], most);
            }
            if (__ballot(not_finite<T>(most))) {
#pragma unroll 1
                for (int e = 0; e < LOADS; ++e) {
                    u4 x = *reinterpret_cast<const u4 *>(loaded + e * 1024);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = finite_of<T>(x[i]);
                    *reinterpret_cast<u4 *>(loaded + e * 1024) = x;
                }
                if constexpr (SPLIT) {
                    bad_first = min(bad_first, k0);
                    bad_last = k0;
                } else if (lane == 0) {
                    atomicMin(&s_bad[0], k0);
                    atomicMax(&s_bad[1], k0);
                }
            }
        }
        if constexpr (SPLIT) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // (what was read of the other buffer is in registers)
        else asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const uint64_t seen = valid;
        if (k0 + STEP < end) {
            issue(k0 + STEP, pages, buffer ^ 1);
            valid = __ballot(pages >= 0) & ALL;
            pages = look_up(k0 + 2 * STEP);
        }
        if (k0 >= hi_most) continue;                      // (no row of this wave's attends to it)
        const bool whole = seen == ALL && k0 >= lo_most && k0 + KT <= hi_least;
#pragma unroll
        for (int u0 = 0; u0 < NU; u0 += SUB) {
            f16v x[SUB][NR];
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int rt = 0; rt < NR; ++rt) x[u][rt] = zero16();
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int u = 0; u < SUB; ++u) {
                    const u4 k = *reinterpret_cast<const u4 *>(at_k + (u0 + u) * 32 * RB + k_lane + ((32 * s) ^ k_turn));
#pragma unroll
                    for (int rt = 0; rt < NR; ++rt) {
                        if constexpr (WIDE) {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                x[u][rt] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[i]), __uint_as_float(q[rt][s][i]), x[u][rt], 0, 0, 0);
                        } else {
                            x[u][rt] = mfma32<T>(k, q[rt][s], x[u][rt]);
                        }
                    }
                }
            if constexpr (!WIDE) {                        // reads of K ahead of the products
                __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
                for (int r = 0; r < SUB * NS - AHEAD; ++r) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
            }
            // which of this lane's slots its rows attend to: bit 8 a + i of tile u for slot 8 a + 4 h + i
            if (!whole) {
#pragma unroll
                for (int rt = 0; rt < NR; ++rt)
#pragma unroll
                    for (int u = 0; u < SUB; ++u) {
                        const int from = lo[rt] - (k0 + 32 * (u0 + u)), to = hi[rt] - (k0 + 32 * (u0 + u));
                        uint32_t bits = (uint32_t)(seen >> (32 * (u0 + u)));
                        bits = from <= 0 ? bits : from >= 32 ? 0u : bits & (~0u << from);
                        bits = to >= 32 ? bits : to <= 0 ? 0u : bits & ~(~0u << to);
                        bits >>= 4 * h;
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (!((bits >> (8 * (i / 4) + i % 4)) & 1)) x[u][rt][i] = -INFINITY;
                    }
            }
            u4 p[SUB][NR][2];
#pragma unroll
            for (int rt = 0; rt < NR; ++rt) {
                float most = x[0][rt][0];
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i) most = fmaxf(most, x[u][rt][i]);
                uint32_t b0, b1;
                row_pair<32>(__float_as_uint(most), b0, b1);
                most = fmaxf(__uint_as_float(b0), __uint_as_float(b1));
                // Weights go by a score that the largest may pass by a factor of 2^8 before all that there is of the row is scaled again.
                const bool rise = (most - top[rt]) * scale > 8.f;
                if (__ballot(rise)) {
                    const float keep = rise ? exp2_fast((top[rt] - most) * scale) : 1.f;
                    if (rise) top[rt] = most;
                    sum[rt] *= keep;
#pragma unroll
                    for (int c = 0; c < NC; ++c) o[rt][c] *= keep;
                }
                const float off = (top[rt] == -INFINITY ? 0.f : top[rt] * scale) - a.lift;
#pragma unroll
                for (int u = 0; u < SUB; ++u) {
                    float w[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        w[i] = exp2_fast(fmaf(x[u][rt][i], scale, -off));
                        sum[rt] += w[i];
                        if constexpr (WIDE) x[u][rt][i] = w[i];
                    }
                    if constexpr (!WIDE) {
                        p[u][rt][0] = pack_weights<T>(w);
                        p[u][rt][1] = pack_weights<T>(w + 8);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                if constexpr (WIDE) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int row = 32 * (u0 + u) + 8 * (i / 4) + 4 * h + i % 4;
#pragma unroll
                        for (int c = 0; c < NC; ++c) {
                            const float v = *reinterpret_cast<const float *>(at_v + row * RB + (((8 * c + (m >> 2)) ^ chunk_swizzle<RB>(row)) << 4) + (m & 3) * 4);
#pragma unroll
                            for (int rt = 0; rt < NR; ++rt) o[rt][c] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, x[u][rt][i], o[rt][c], 0, 0, 0);
                        }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        unsigned char *from = at_v + (32 * (u0 + u) + 16 * j) * RB + v_lane;
#pragma unroll
                        for (int c = 0; c < NC; ++c) {
                            typedef __attribute__((address_space(3))) s4 *Turned;
                            const u2 v0 = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Turned)ANN_LDS(from + ((64 * c) ^ v_turn))));
                            const u2 v1 = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Turned)ANN_LDS(from + 8 * RB + ((64 * c) ^ v_turn ^ 32))));
#pragma unroll
                            for (int rt = 0; rt < NR; ++rt) o[rt][c] = mfma32<T>(u4{v0[0], v0[1], v1[0], v1[1]}, p[u][rt][j], o[rt][c]);
                        }
                    }
                }
            }
        }
    }

    // infinities and NaN of V that were taken out
    if constexpr (!SPLIT) {
        __syncthreads();
        bad_first = s_bad[0];
        bad_last = s_bad[1];
    }
#pragma unroll 1
    for (int k = bad_first; k <= bad_last; k += STEP)
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
                    if (at >= a.cache.d) continue;
                    const f4 v = not_finite_four<T>(from + at * T::bytes);
#pragma unroll
                    for (int rt = 0; rt < NR; ++rt)
                        if (key >= lo[rt] && key < hi[rt]) {
#pragma unroll
                            for (int b = 0; b < 4; ++b) o[rt][c][i + b] += v[b];
                        }
                }
        }

#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
        uint32_t b0, b1;
        row_pair<32>(__float_as_uint(sum[rt]), b0, b1);
        sum[rt] = __uint_as_float(b0) + __uint_as_float(b1);
        top[rt] *= scale;                                 // an exponent of 2
    }
    // four elements of a row: divided and written, or left for what joins the parts
    auto write = [&](int in, int at, f4 y, float most, float total) {
        const int r = tile.r0 + in;
        const int64_t row = (int64_t)(tile.token0 + r / G) * a.q_heads + head * G + r % G;
        if (a.splits > 1) {
            const int64_t slot = row * a.splits + a.part0 + part;
            *reinterpret_cast<f4 *>(a.partial + slot * a.cache.d + at) = y;
            if (at == 0) {
                a.stats[2 * slot] = most;
                a.stats[2 * slot + 1] = total;
            }
        } else {
            const float by = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = total == 0.f ? 0.f : y[i] * by;
            store_four<T>(static_cast<char *>(a.out) + (row * a.cache.d + at) * T::bytes, y);
            if (at == 0 && a.lse) a.lse[row] = chunk_lse(most, total, a.lift);
        }
    };
    if constexpr (!SPLIT) {
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            const int in = row0 + rt * 32 + m;
            if (in >= tile.count) continue;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int at = 32 * c + 2 * i + 4 * h;
                    if (at < a.cache.d) write(in, at, f4{o[rt][c][i], o[rt][c][i + 1], o[rt][c][i + 2], o[rt][c][i + 3]}, top[rt], sum[rt]);
                }
        }
    } else {
        // the waves' sums, joined
        constexpr int LD = DP + 4, ROWS = 32 * NR;
        __shared__ float s_top[WAVES][ROWS], s_sum[WAVES][ROWS];
        float *s_o = reinterpret_cast<float *>(chunk_lds);
        if (h == 0) {
#pragma unroll
            for (int rt = 0; rt < NR; ++rt) { s_top[wave][rt * 32 + m] = top[rt]; s_sum[wave][rt * 32 + m] = sum[rt]; }
        }
        __syncthreads();
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            float all = -INFINITY;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) all = fmaxf(all, s_top[w][rt * 32 + m]);
            const float f = top[rt] == -INFINITY ? 1.f : exp2_fast(top[rt] - all);      // (a row without a score has zeros, or NaN)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<f4 *>(s_o + (wave * ROWS + rt * 32 + m) * LD + 32 * c + 2 * i + 4 * h) =
                        f4{o[rt][c][i], o[rt][c][i + 1], o[rt][c][i + 2], o[rt][c][i + 3]} * f;
        }
        __syncthreads();
        const int per_row = a.cache.d / 4;
        for (int i = threadIdx.x; i < tile.count * per_row; i += WAVES * WAVE) {
            const int in = i / per_row, at = i % per_row * 4;
            float all = -INFINITY, total = 0.f;
            f4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) all = fmaxf(all, s_top[w][in]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float t = s_top[w][in];
                total += s_sum[w][in] * (t == -INFINITY ? 1.f : exp2_fast(t - all));
                y += *reinterpret_cast<const f4 *>(s_o + (w * ROWS + in) * LD + at);
            }
            write(in, at, y, all, total);
        }
    }
}

// What the parts of a row left, joined by a wave.  own: the parts behind the first launch's (CHUNK_COMMON) are the second one's (CHUNK_OWN).
template <class T>
__global__ __launch_bounds__(256) void chunk_join_kernel(ChunkArgs a, ChunkJoin j) {
    const int lane = threadIdx.x & (WAVE - 1), d = a.cache.d, G = a.q_heads / a.cache.heads;
    const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / WAVE;
    if (row >= (int64_t)a.tokens * a.q_heads) return;
    const int t = (int)(row / a.q_heads), in_head = (int)(row % a.q_heads) % G;
    int parts0 = 0, parts1 = 0;                           // of the first and of the second launch
    if (a.mode == CHUNK_NEW) {
        const PackedToken token = packed_token(a.starts, a.requests, a.tokens, t);
        if (token.request < 0) return;
        const int i = t - chunk_start(a, token.request);
        parts0 = chunk_parts(chunk_range(a, chunk_tile(a, token.request, (int64_t)i * G + in_head, G, j.rows), G), j.chunk);
    } else {
        const int g = chunk_group(a, t), common = chunk_common(a, g), n = min(chunk_length(a, t), a.max_length), mine = min(n, common);
        if (g >= 0 && j.first_parts > 0) parts0 = chunk_parts({0, common}, j.chunk);
        parts1 = chunk_parts({mine, mine + min(n - mine, a.max_own)}, j.own_chunk);
    }
    const int n = parts0 + parts1;
    auto slot = [&](int s) { return row * a.splits + (s < parts0 ? s : j.first_parts + s - parts0); };
    float most = -INFINITY, total = 0.f;
    for (int s = lane; s < n; s += WAVE) most = fmaxf(most, a.stats[2 * slot(s)]);
#pragma unroll
    for (int i = 1; i < WAVE; i *= 2) most = fmaxf(most, __shfl_xor(most, i));
    const int at = 4 * lane;
    f4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < n; ++s) {
        const float x = a.stats[2 * slot(s)], f = x == -INFINITY ? 1.f : exp2_fast(x - most);
        total += a.stats[2 * slot(s) + 1] * f;
        if (at < d) y += *reinterpret_cast<const f4 *>(a.partial + slot(s) * d + at) * f;
    }
    if (at >= d) return;
    const float by = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = total == 0.f ? 0.f : y[i] * by;
    store_four<T>(static_cast<char *>(a.out) + (row * d + at) * T::bytes, y);
    if (lane == 0 && a.lse) a.lse[row] = chunk_lse(most, total, a.lift);
}

template <class T, int DP, int NR, bool SPLIT>
hipError_t chunk_rows(const ChunkArgs &a, int parts, hipStream_t stream) {
    typedef ChunkShape<T, DP, NR, SPLIT> Sh;
    static size_t granted = 0;
    if (hipError_t e = allow_big_lds(reinterpret_cast<const void *>(chunk_attention_kernel<T, DP, NR, SPLIT>), Sh::LDS, &granted)) return e;
    hipLaunchKernelGGL((chunk_attention_kernel<T, DP, NR, SPLIT>), dim3((unsigned)((int64_t)a.tiles * parts * a.cache.heads)), dim3(Sh::THREADS), Sh::LDS, stream, a);
    return hipGetLastError();
}
template <class T, int DP>
hipError_t chunk_rows(const ChunkArgs &a, const ChunkPass &pass, hipStream_t stream) {
    if (pass.shape == CHUNK_FEW) return chunk_rows<T, DP, 1, true>(a, pass.parts, stream);
    if constexpr (chunk_most(T::bytes, DP) == 2)
        if (pass.shape == CHUNK_MANY) return chunk_rows<T, DP, 2, false>(a, pass.parts, stream);
    return chunk_rows<T, DP, 1, false>(a, pass.parts, stream);
}
template <class T>
hipError_t chunk_pass(ChunkArgs a, const ChunkPass &pass, int mode, int part0, hipStream_t stream) {
    a.mode = mode; a.tiles = pass.tiles; a.chunk = pass.chunk; a.part0 = part0;
    return a.cache.d <= 64 ? chunk_rows<T, 64>(a, pass, stream) : a.cache.d <= 128 ? chunk_rows<T, 128>(a, pass, stream) : chunk_rows<T, 256>(a, pass, stream);
}
template <class T>
hipError_t launch_chunk(const ChunkArgs &a, const ChunkPlan &pl, hipStream_t stream) {
    const bool shared = a.group_starts != nullptr;
    if (!shared || pl.first.parts > 0)
        if (hipError_t e = chunk_pass<T>(a, pl.first, shared ? CHUNK_COMMON : CHUNK_NEW, 0, stream)) return e;
    if (shared)
        if (hipError_t e = chunk_pass<T>(a, pl.own, CHUNK_OWN, pl.first.parts, stream)) return e;
    if (pl.splits == 1) return hipSuccess;
    ChunkArgs b = a;
    b.mode = shared ? CHUNK_COMMON : CHUNK_NEW;
    const ChunkJoin join{pl.first.chunk, pl.first.parts, pl.own.chunk, pl.first.rows};
    const int64_t rows = (int64_t)a.tokens * a.q_heads;
    hipLaunchKernelGGL((chunk_join_kernel<T>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, b, join);
    return hipGetLastError();
}

}  // namespace ann
