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

#include "chunk_rows.hpp"
#include "launch.hpp"
#include "paged.hpp"

namespace ann {

typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef unsigned short us2 __attribute__((ext_vector_type(2)));

#define ANN_LDS(p) ((__attribute__((address_space(3))) void *)(p))
#define ANN_ROW_TO_LDS(gptr, lptr) \
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(gptr), ANN_LDS(lptr), 16, 0, 0)

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

// until at most n of this wave's loads are outstanding
template <int n>
__device__ __forceinline__ void wait_outstanding() {
    static_assert(n >= 0 && n < 64, "vmcnt is a field of 6 bits");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (n & 15) | ((n >> 4) << 14));
    asm volatile("" ::: "memory");
}

// ---- the kernel ----------------------------------------------------------------------------------------------

// FEW: the waves take slots of their own, of 32 rows; else 32 rows each of their own, of the same slots.
template <class T, int DP_, bool FEW_>
struct ChunkShape {
    static constexpr int DP = DP_, RB = DP * T::bytes;                  // largest d; bytes of a row in LDS
    static constexpr bool FEW = FEW_;
    static constexpr int KT = chunk_slots(RB, FEW), WAVES = CHUNK_WAVES, SLOT_WAVES = chunk_slot_waves(RB);    // FEW: waves that take slots, as LDS allows
    static constexpr int R = chunk_rows(FEW);
    static constexpr int CPR = RB / 16, RPI = 64 / CPR;                 // chunks of a row, rows that a load brings
    static constexpr int LOADS = KT * RB / 1024 / (FEW ? 1 : WAVES);    // of K, and of V, that a wave issues for a tile of slots
    static constexpr int TILE = KT * RB;
    static constexpr int BUFFERS = FEW ? 1 : 2;                         // FEW: K of the next tile is loaded while the weights meet V, V while K meets the queries
    static constexpr int NS = RB / 32, NC = DP / 32, NU = KT / 32;      // steps of 32 bytes of a row; tiles of 32 elements; tiles of 32 slots
    static constexpr int LD = DP + 4;                                   // floats of a row where the waves' sums are joined
    static constexpr int LDS_TILES = BUFFERS * 2 * TILE * (FEW ? SLOT_WAVES : 1), LDS_JOIN = FEW ? WAVES * 32 * (LD + 2) * 4 : 0;
    static constexpr int LDS = LDS_TILES > LDS_JOIN ? LDS_TILES : LDS_JOIN;
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

template <class T, int DP, bool FEW>
__device__ __forceinline__ void chunk_body(const ChunkArgs &a, const ChunkPass &pass, int block, unsigned char *chunk_lds, int *s_scratch) {
    typedef ChunkShape<T, DP, FEW> Sh;
    constexpr int KT = Sh::KT, RB = Sh::RB, NS = Sh::NS, NC = Sh::NC, NU = Sh::NU, LOADS = Sh::LOADS, CPR = Sh::CPR, RPI = Sh::RPI, WAVES = Sh::WAVES;
    constexpr bool WIDE = T::bytes == 4;
    constexpr int AHEAD = DP == 128 && !FEW ? 6 : 4;      // reads of LDS in flight before a product
    int *s_lo = s_scratch, *s_hi = s_scratch + 4, *s_bad = s_scratch + 8;
    const int lane = threadIdx.x & (WAVE - 1), m = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int G = a.q_heads / a.cache.heads, head = block % a.cache.heads;
    const ChunkDeal deal = chunk_deal(a, pass, block / a.cache.heads, G);
    if (deal.count <= 0) return;
    const ChunkSpan range = chunk_range(a, pass.mode, deal.sequence, deal.q, deal.r0 / G, (deal.r0 + deal.count - 1) / G);
    if (deal.part >= chunk_parts(chunk_slots_of(range), deal.chunk)) return;
    const int first = chunk_begin(range) + deal.part * deal.chunk, end = range.hi - first < deal.chunk ? range.hi : first + deal.chunk;

    // this lane's row: its query and the slots that it attends to
    u4 q[NS];
    int lo = 0, hi = INT_MAX, hi_most = 0;
    const uint32_t flip = a.scale < 0.f ? (WIDE ? 0x80000000u : 0x80008000u) : 0u;
    const float scale = fmaxf(fabsf(a.scale), 1e-37f);    // (not 0: a score of -infinity stays one)
    const int row0 = FEW ? 0 : wave * 32, row_bytes = a.cache.d * T::bytes;
    {
        const int in = row0 + m, r = deal.r0 + in, t = deal.q.token0 + r / G;
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
            ChunkSpan span = range;
            if (pass.mode == CHUNK_NEW) span = chunk_span(a, chunk_length(a, deal.q.request), deal.q.tokens - r / G);
            if (pass.mode == CHUNK_COMMON) span.hi = min(span.hi, chunk_length(a, t));
            lo = span.lo;
            hi = span.hi;
            hi_most = hi;
        }
    }
    int lo_most = lo, hi_least = hi;                      // of all rows of the wave
#pragma unroll
    for (int i = 1; i < 32; i *= 2) {
        lo_most = max(lo_most, __shfl_xor(lo_most, i));
        hi_least = min(hi_least, __shfl_xor(hi_least, i));
        hi_most = max(hi_most, __shfl_xor(hi_most, i));
    }
    lo_most = __builtin_amdgcn_readfirstlane(lo_most);
    hi_least = __builtin_amdgcn_readfirstlane(hi_least);
    hi_most = __builtin_amdgcn_readfirstlane(hi_most);
    int all_lo = lo_most, all_hi = hi_least;              // ... of all waves that read the same slots
    if constexpr (!FEW) {
        if (lane == 0) { s_lo[wave] = lo_most; s_hi[wave] = hi_least; }
        if (threadIdx.x == 0) { s_bad[0] = INT_MAX; s_bad[1] = -1; }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) { all_lo = max(all_lo, s_lo[w]); all_hi = min(all_hi, s_hi[w]); }
        all_lo = __builtin_amdgcn_readfirstlane(all_lo);
        all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    }

    unsigned char *mine = chunk_lds + (FEW ? wave * 2 * Sh::TILE : 0);
    const int32_t *table = a.table + (int64_t)deal.q.request * a.width;
    const int slots_log = a.cache.slots_log, mask = (1 << slots_log) - 1;
    const char *k_head = a.cache.k + head * a.cache.k_head, *v_head = a.cache.v + head * a.cache.v_head;
    // the page of slot k0 + lane % KT, or -1
    auto look_up = [&](int k0) {
        const int key = k0 + (lane & (KT - 1));
        int page = -1;
        if (key < end) page = table[key >> slots_log];
        return (unsigned)page < (unsigned)a.cache.pages ? page : -1;
    };
    // Slots without a row take one of the first page's: their scores do not count, and of their values only that they are finite.
    const int first_row = (FEW ? 0 : wave * LOADS) * RPI, in_load = lane / CPR, first_at = ((lane & (CPR - 1)) ^ chunk_swizzle<RB>(first_row + in_load)) * 16;
    // K, V or both of the tile of slots from k0 on
    auto issue = [&](int k0, int pages, unsigned char *to, auto keys, auto values) __attribute__((always_inline)) {
        constexpr bool K = decltype(keys)::value, V = decltype(values)::value;
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
                    if constexpr (K) ANN_ROW_TO_LDS(k + (in_load * (uint32_t)a.cache.k_slot + at), to + e * 1024);
                    if constexpr (V) ANN_ROW_TO_LDS(v + (in_load * (uint32_t)a.cache.v_slot + at), to + Sh::TILE + e * 1024);
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
                if constexpr (K) ANN_ROW_TO_LDS(k, to + e * 1024);
                if constexpr (V) ANN_ROW_TO_LDS(v, to + Sh::TILE + e * 1024);
            }
        }
    };
    const bool loads = !FEW || wave < Sh::SLOT_WAVES;
    if (row_bytes < RB && loads) {                        // what lies behind the end of a row in LDS is never loaded
#pragma unroll
        for (int b = 0; b < 2 * Sh::BUFFERS; ++b)
#pragma unroll
            for (int e = 0; e < LOADS; ++e) *reinterpret_cast<u4 *>(mine + b * Sh::TILE + first_row * RB + e * 1024 + lane * 16) = zero_chunk();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }

    f16v o[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) o[c] = zero16();
    float top = -INFINITY, sum = 0.f;                     // a score that the weights go by; the sum of this lane's slots alone
    const int k_lane = m * RB, k_turn = (h ^ chunk_swizzle<RB>(m)) << 4;    // a lane's part of the places of its operands
    const int i16 = lane & 15, v_row = 4 * h + (i16 >> 2), v_lane = v_row * RB;
    const int v_turn = ((2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) ^ chunk_swizzle<RB>(v_row)) << 4 | (i16 & 1) << 3;
    constexpr uint64_t ALL = KT == 64 ? ~0ull : (1ull << (KT & 63)) - 1;
    int bad_first = INT_MAX, bad_last = -1;

    auto scores = [&](unsigned char *at_k, int k0, uint64_t seen, f16v (&x)[NU]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NU; ++u) x[u] = zero16();
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
    // scores become weights; 16 bits: in p, as operands
    auto weights = [&](f16v (&x)[NU], u4 (&p)[NU][2]) __attribute__((always_inline)) {
        float most = x[0][0];
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, x[u][i]);
        uint32_t b0, b1;
        row_pair<32>(__float_as_uint(most), b0, b1);
        most = fmaxf(__uint_as_float(b0), __uint_as_float(b1));
        // The largest score may pass the one that the weights go by by a factor of 2^8 before all that there is of the row is scaled again.
        const bool rise = (most - top) * scale > 8.f;
        if (__ballot(rise)) {
            const float keep = rise ? exp2_fast((top - most) * scale) : 1.f;
            if (rise) top = most;
            sum *= keep;
#pragma unroll
            for (int c = 0; c < NC; ++c) o[c] *= keep;
        }
        const float off = (top == -INFINITY ? 0.f : top * scale) - a.lift;
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            float w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                w[i] = exp2_fast(fmaf(x[u][i], scale, -off));
                sum += w[i];
                if constexpr (WIDE) x[u][i] = w[i];
            }
            if constexpr (!WIDE) {
                p[u][0] = pack_weights<T>(w);
                p[u][1] = pack_weights<T>(w + 8);
            }
        }
    };
    auto times_v = [&](unsigned char *at_v, const f16v (&x)[NU], const u4 (&p)[NU][2]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            if constexpr (WIDE) {
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    if (32 * c >= a.cache.d) break;       // (uniform)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int row = 32 * u + 8 * (i / 4) + 4 * h + i % 4;
                        const float v = *reinterpret_cast<const float *>(at_v + row * RB + (((8 * c + (m >> 2)) ^ chunk_swizzle<RB>(row)) << 4) + (m & 3) * 4);
                        o[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, x[u][i], o[c], 0, 0, 0);
                    }
                }
            } else {
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
        if constexpr (FEW) {
            bad_first = min(bad_first, k0);
            bad_last = k0;
        } else if (lane == 0) {
            atomicMin(&s_bad[0], k0);
            atomicMax(&s_bad[1], k0);
        }
    };

    constexpr int STEP = FEW ? Sh::SLOT_WAVES * KT : KT;
    constexpr std::true_type YES{};
    constexpr std::false_type NO{};
    int k0 = !loads ? end : first + (FEW ? wave * KT : 0);
    if constexpr (FEW) {
        uint64_t valid = 0;
        int pages = -1, next = -1;                        // of this tile, of the next
        if (k0 < end) {
            pages = look_up(k0);
            issue(k0, pages, mine, YES, NO);
            next = look_up(k0 + STEP);
            issue(k0, pages, mine, NO, YES);
        }
        for (; k0 < end; k0 += STEP) {
            const bool more = k0 + STEP < end;
            f16v x[NU];
            u4 p[NU][2];
            // K is there once no more than the loads of V are outstanding, which were issued behind it; V likewise
            wait_outstanding<LOADS>();
            valid = __ballot(pages >= 0) & ALL;
            scores(mine, k0, valid, x);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            pages = next;
            if (more) {
                issue(k0 + STEP, pages, mine, YES, NO);
                next = look_up(k0 + 2 * STEP);
            }
            weights(x, p);
            if (more) wait_outstanding<LOADS>();
            else wait_outstanding<0>();
            if (!(valid == ALL && k0 >= lo_most && k0 + KT <= hi_least)) take_out(mine + Sh::TILE, k0);
            times_v(mine + Sh::TILE, x, p);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more) issue(k0 + STEP, pages, mine, NO, YES);
        }
    } else {
        int pages = -1, buffer = 0;
        uint64_t valid = 0;
        if (k0 < end) {
            pages = look_up(k0);
            issue(k0, pages, mine, YES, YES);
            valid = __ballot(pages >= 0) & ALL;
            pages = look_up(k0 + STEP);
        }
        for (; k0 < end; k0 += STEP, buffer ^= 1) {
            unsigned char *at_k = mine + buffer * 2 * Sh::TILE;
            wait_outstanding<0>();
            if (!(valid == ALL && k0 >= all_lo && k0 + KT <= all_hi)) take_out(at_k + Sh::TILE, k0);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // all waves' loads are there, and nobody reads the other buffer any more
            const uint64_t seen = valid;
            if (k0 + STEP < end) {
                issue(k0 + STEP, pages, mine + (buffer ^ 1) * 2 * Sh::TILE, YES, YES);
                valid = __ballot(pages >= 0) & ALL;
                pages = look_up(k0 + 2 * STEP);
            }
            if (k0 >= hi_most) continue;                  // (no row of this wave's attends to it)
            f16v x[NU];
            u4 p[NU][2];
            scores(at_k, k0, seen, x);
            weights(x, p);
            times_v(at_k + Sh::TILE, x, p);
        }
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
        top *= scale;                                     // an exponent of 2
    }
    // four elements of a row: divided and written, or left for what joins the parts
    auto write = [&](int in, int at, f4 y, float most, float total) {
        const int r = deal.r0 + in;
        const int64_t row = (int64_t)(deal.q.token0 + r / G) * a.q_heads + head * G + r % G;
        if (a.splits > 1) {
            const int64_t place = row * a.splits + pass.part0 + deal.part;
            *reinterpret_cast<f4 *>(a.partial + place * a.cache.d + at) = y;
            if (at == 0) {
                a.stats[2 * place] = most;
                a.stats[2 * place + 1] = total;
            }
        } else {
            const float by = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = total == 0.f ? 0.f : y[i] * by;
            store_four<T>(static_cast<char *>(a.out) + (row * a.cache.d + at) * T::bytes, y);
            if (at == 0 && a.lse) a.lse[row] = chunk_lse(most, total, a.lift);
        }
    };
    if constexpr (!FEW) {
        const int in = row0 + m;
        if (in < deal.count) {
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int at = 32 * c + 2 * i + 4 * h;
                    if (at < a.cache.d) write(in, at, f4{o[c][i], o[c][i + 1], o[c][i + 2], o[c][i + 3]}, top, sum);
                }
        }
    } else {
        // the waves' sums, joined
        constexpr int LD = Sh::LD;
        float *s_o = reinterpret_cast<float *>(chunk_lds), *s_top = s_o + WAVES * 32 * LD, *s_sum = s_top + WAVES * 32;
        __syncthreads();
        if (h == 0) { s_top[wave * 32 + m] = top; s_sum[wave * 32 + m] = sum; }
        __syncthreads();
        float all = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) all = fmaxf(all, s_top[w * 32 + m]);
        const float f = top == -INFINITY ? 1.f : exp2_fast(top - all);      // (a row without a score has zeros, or NaN)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<f4 *>(s_o + (wave * 32 + m) * LD + 32 * c + 2 * i + 4 * h) = f4{o[c][i], o[c][i + 1], o[c][i + 2], o[c][i + 3]} * f;
        __syncthreads();
        const int per_row = a.cache.d / 4;
        for (int i = threadIdx.x; i < deal.count * per_row; i += WAVES * WAVE) {
            const int in = i / per_row, at = i % per_row * 4;
            float most = -INFINITY, total = 0.f;
            f4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) most = fmaxf(most, s_top[w * 32 + in]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float t = s_top[w * 32 + in];
                total += s_sum[w * 32 + in] * (t == -INFINITY ? 1.f : exp2_fast(t - most));
                y += *reinterpret_cast<const f4 *>(s_o + (w * 32 + in) * LD + at);
            }
            write(in, at, y, most, total);
        }
    }
}

// One pass, or two side by side: workgroups of either in turn, as long as there are both, so that a compute unit has some that wait for memory beside some that multiply.
template <class T, int DP, bool FEW, bool BOTH>
__global__ __launch_bounds__(CHUNK_WAVES * WAVE, chunk_per_simd(T::bytes, DP)) void chunk_attention_kernel(ChunkArgs a, ChunkPass first, ChunkPass own) {
    extern __shared__ __align__(16) unsigned char chunk_lds[];
    __shared__ int s_scratch[12];
    int block = blockIdx.x;
    if constexpr (BOTH) {
        const int n0 = first.items * a.cache.heads, n1 = own.items * a.cache.heads, both = 2 * min(n0, n1);
        const bool is_own = block < both ? block & 1 : n1 > n0;
        block = block < both ? block >> 1 : block - both / 2;
        if (is_own) return chunk_body<T, DP, true>(a, own, block, chunk_lds, s_scratch);
    }
    chunk_body<T, DP, FEW>(a, first, block, chunk_lds, s_scratch);
}

// What the parts of a row left, joined by a wave: lanes share the parts out where a row takes fewer than there are.
template <class T>
__global__ __launch_bounds__(256) void chunk_join_kernel(ChunkArgs a, ChunkPass first, ChunkPass own) {
    const int lane = threadIdx.x & (WAVE - 1), d = a.cache.d, G = a.q_heads / a.cache.heads;
    const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / WAVE;
    if (row >= (int64_t)a.tokens * a.q_heads) return;
    const int t = (int)(row / a.q_heads), in_head = (int)(row % a.q_heads) % G;
    int parts0 = 0, parts1 = 0;                           // of the two passes, or of the only one
    if (first.mode == CHUNK_NEW) {
        const PackedToken token = packed_token(a.starts, a.requests, a.tokens, t);
        if (token.request < 0) return;
        parts0 = chunk_parts_of(a, first, token.request, t, in_head, G);
    } else if (first.mode == CHUNK_OWN) {
        parts0 = chunk_parts_of(a, first, t, t, in_head, G);
    } else {
        const int g = chunk_group(a, t);
        if (g >= 0) parts0 = chunk_parts_of(a, first, g, t, in_head, G);
        parts1 = chunk_parts_of(a, own, t, t, in_head, G);
    }
    const int n = parts0 + parts1;
    auto place = [&](int s) { return row * a.splits + (s < parts0 ? s : own.part0 + s - parts0); };
    const float2 *stats = reinterpret_cast<const float2 *>(a.stats);
    float most = -INFINITY;
    for (int s = lane; s < n; s += WAVE) most = fmaxf(most, stats[place(s)].x);
#pragma unroll
    for (int i = 1; i < WAVE; i *= 2) most = fmaxf(most, __shfl_xor(most, i));
    // lanes of a row: the power of two from d / 4 on
    const int per = d <= 32 ? 8 : d <= 64 ? 16 : d <= 128 ? 32 : 64, at = 4 * (lane % per);
    float total = 0.f;
    f4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = lane / per; s < n; s += WAVE / per) {
        const int64_t p = place(s);
        const float2 st = stats[p];
        const float f = st.x == -INFINITY ? 1.f : exp2_fast(st.x - most);
        total += st.y * f;
        if (at < d) y += *reinterpret_cast<const f4 *>(a.partial + p * d + at) * f;
    }
    for (int i = per; i < WAVE; i *= 2) {
        total += __shfl_xor(total, i);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] += __shfl_xor(y[j], i);
    }
    if (lane >= per || at >= d) return;
    const float by = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = total == 0.f ? 0.f : y[i] * by;
    store_four<T>(static_cast<char *>(a.out) + (row * d + at) * T::bytes, y);
    if (lane == 0 && a.lse) a.lse[row] = chunk_lse(most, total, a.lift);
}

template <class T, int DP, bool FEW, bool BOTH>
hipError_t chunk_launch(const ChunkArgs &a, const ChunkPlan &pl, hipStream_t stream) {
    typedef ChunkShape<T, DP, FEW> Sh;
    typedef ChunkShape<T, DP, true> Own;
    constexpr int LDS = BOTH && Own::LDS > Sh::LDS ? Own::LDS : Sh::LDS;
    static size_t granted = 0;
    if (hipError_t e = allow_big_lds(reinterpret_cast<const void *>(chunk_attention_kernel<T, DP, FEW, BOTH>), LDS, &granted)) return e;
    const int64_t blocks = (int64_t)(pl.first.items + (BOTH ? pl.own.items : 0)) * a.cache.heads;
    hipLaunchKernelGGL((chunk_attention_kernel<T, DP, FEW, BOTH>), dim3((unsigned)blocks), dim3(CHUNK_WAVES * WAVE), LDS, stream, a, pl.first, pl.own);
    return hipGetLastError();
}
template <class T, int DP>
hipError_t chunk_launch(const ChunkArgs &a, const ChunkPlan &pl, hipStream_t stream) {
    if (pl.own.items) return pl.first.shape == CHUNK_FEW ? chunk_launch<T, DP, true, true>(a, pl, stream) : chunk_launch<T, DP, false, true>(a, pl, stream);
    return pl.first.shape == CHUNK_FEW ? chunk_launch<T, DP, true, false>(a, pl, stream) : chunk_launch<T, DP, false, false>(a, pl, stream);
}
template <class T>
hipError_t launch_chunk(const ChunkArgs &a, const ChunkPlan &pl, hipStream_t stream) {
    if (hipError_t e = a.cache.d <= 64 ? chunk_launch<T, 64>(a, pl, stream) : a.cache.d <= 128 ? chunk_launch<T, 128>(a, pl, stream) : chunk_launch<T, 256>(a, pl, stream)) return e;
    if (a.splits == 1) return hipSuccess;
    const int64_t rows = (int64_t)a.tokens * a.q_heads;
    hipLaunchKernelGGL((chunk_join_kernel<T>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, a, pl.first, pl.own);
    return hipGetLastError();
}

}  // namespace ann
