// Attention of one new token per request over a paged cache, on the matrix cores.
//
// A workgroup of four waves takes a part of one request's slots for at most 16 MT query heads of one cache head; a wave
// takes NT tiles of 16 slots at a time.  Both products are turned so that the query heads are the columns of every tile:
//     S^T [16 slots x 16 heads] = K Q^T          O^T [d x 16 heads] += V^T P^T
// Lane 16 g + m then holds the scores of slots 4 g .. 4 g + 3 and head m, which is where the second product wants its operand P^T if
// its 32 columns are numbered 8 g + 4 t + i for slot 4 g + i of tile t: nothing passes between lanes.  Its maximum, its sum
// and its factor belong to head m too, so the accumulators are scaled in place.  Rows of V come as they lie in memory, 16 lanes
// beside each other to a row, and are turned in registers, one byte permutation for two elements.
//
// Bound by reading K and V once: G = q_heads / heads query heads make G multiply-adds of a 16-bit element, a tenth of what the matrix cores do in the
// time even where 15 of 16 columns are empty (G = 1).  So the loop asks for V of these slots and K of the next before it needs either, 16 KB a wave at d = 128, three
// workgroups to a compute unit.  64 requests of 9216 slots, 8 cache heads of 128, bf16 (2.4 GB): 376 to 390 us, 6.4 to 6.2 TB/s, which is what a loop of loads reads; G = 1: 6.6,
// d = 256: 6.3, fp32: 6.4, pages of 8 slots 5.7, of one 5.4 (a look-up for each row).  One request of 131072 slots (0.54 GB): 103 to 107 us a call.
#pragma once

#include <type_traits>

#include "launch.hpp"
#include "paged.hpp"

namespace ann {

constexpr int ATTEND_THREADS = ATTEND_WAVES * WAVE;

template <class T, int VE_>
struct AttendShape {
    static constexpr int VE = VE_, DP = 16 * VE;                     // elements of a row of V a lane holds; largest d
    static constexpr int CE = T::bytes == 2 && VE > 4 ? 8 : 4;       // ... of which so many lie together
    static constexpr int NU = VE / CE, CW = CE * T::bytes / 4;       // such chunks, and their registers
    static constexpr int NS = DP * T::bytes / 64;                    // steps of 64 bytes of a row of K
    static constexpr int NT = attend_tiles(T::bytes, VE);
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// maximum, sum over the lanes with the same l % 16
__device__ __forceinline__ float column_max(float x) {
    uint32_t a, b;
    row_pair<16>(__float_as_uint(x), a, b);
    x = fmaxf(__uint_as_float(a), __uint_as_float(b));
    row_pair<32>(__float_as_uint(x), a, b);
    return fmaxf(__uint_as_float(a), __uint_as_float(b));
}
__device__ __forceinline__ float column_sum(float x) {
    uint32_t a, b;
    row_pair<16>(__float_as_uint(x), a, b);
    x = __uint_as_float(a) + __uint_as_float(b);
    row_pair<32>(__float_as_uint(x), a, b);
    return __uint_as_float(a) + __uint_as_float(b);
}

// ... over all lanes of a wave
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, __uint_as_float(lane_swap<1>(__float_as_uint(x))));
    x = fmaxf(x, __uint_as_float(lane_swap<2>(__float_as_uint(x))));
    x = fmaxf(x, __uint_as_float(lane_swap<4>(__float_as_uint(x))));
    x = fmaxf(x, __uint_as_float(lane_swap<8>(__float_as_uint(x))));
    return column_max(x);
}
__device__ __forceinline__ float wave_sum(float x) {
    x += __uint_as_float(lane_swap<1>(__float_as_uint(x)));
    x += __uint_as_float(lane_swap<2>(__float_as_uint(x)));
    x += __uint_as_float(lane_swap<4>(__float_as_uint(x)));
    x += __uint_as_float(lane_swap<8>(__float_as_uint(x)));
    return column_sum(x);
}

template <bool ONCE, class V>
__device__ __forceinline__ V stream_load(const V *p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}

template <int CW> struct Words;
template <> struct Words<2> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Words<4> { typedef u4 type; };

// fp16 has no numbers below 2^-24, and a long context may have its weight in many slots that get less than that of the largest: weights are
// 2^12 times as large in the loop, which keeps what makes up a millionth of the sum of 2^17 slots.
template <class T> constexpr int ATTEND_LIFT = std::is_same_v<T, F16> ? 12 : 0;

// bf16 and fp32 have values up to the largest of the sums' 32 bits, and weights add up to as much as there are slots before they are divided by their sum: for the product with V they are
// multiplied by this power of two, below 1 / n, and the rows stay so until they are divided.  (fp16: 65504 times 2^12 times 2^31 is far from it.)
template <class T>
__device__ __forceinline__ float attend_scale(int n) {
    return std::is_same_v<T, F16> ? 1.f : __uint_as_float((uint32_t)(127 - (32 - __clz(n))) << 23);
}

// Eight weights as an operand of 16 bits and what that leaves, as another: the product with V then has 16 bits (bf16) or more of
// them.  One part alone would be off by as much as the output's own rounding; the second product costs nothing here.
template <class T>
__device__ __forceinline__ void split_weights(const float (&p)[8], u4 &high, u4 &low);
template <>
__device__ __forceinline__ void split_weights<BF16>(const float (&p)[8], u4 &high, u4 &low) {
    b8 h, l;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        h[i] = (__bf16)p[i];
        l[i] = (__bf16)(p[i] - (float)h[i]);
    }
    high = __builtin_bit_cast(u4, h);
    low = __builtin_bit_cast(u4, l);
}
template <>
__device__ __forceinline__ void split_weights<F16>(const float (&p)[8], u4 &high, u4 &low) {
    h8 h, l;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        h[i] = (_Float16)p[i];
        l[i] = (_Float16)(p[i] - (float)h[i]);
    }
    high = __builtin_bit_cast(u4, h);
    low = __builtin_bit_cast(u4, l);
}

template <class T>
__device__ __forceinline__ f4 scores_step(u4 k, u4 q, f4 c) {
    if constexpr (T::bytes == 2) {
        return mfma16<T>(k, q, c);
    } else {                                              // (which four columns meet in an instruction is all the same)
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[j]), __uint_as_float(q[j]), c, 0, 0, 0);
        return c;
    }
}

__device__ __forceinline__ AttendSpan attend_span(const AttentionArgs &a, int b) {
    return attend_span(a.lengths[b], a.max_length, a.window, a.chunk);
}

// By one wave: largest exponent of head row r and total over its parts.
__device__ __forceinline__ void attend_stats(const AttentionArgs &a, int64_t r, int parts, float &most, float &total) {
    const float *st = a.stats + r * a.splits * 2;
    const int lane = threadIdx.x & (WAVE - 1);
    float m = -INFINITY, t = 0.f;
    for (int s = lane; s < parts; s += WAVE) m = fmaxf(m, st[2 * s]);
    most = wave_max(m);
    for (int s = lane; s < parts; s += WAVE) t += st[2 * s + 1] * (st[2 * s] == -INFINITY ? 1.f : exp2_fast(st[2 * s] - most));
    total = wave_sum(t);
}
__device__ __forceinline__ float attend_lse(float most, float total) {
    return total == 0.f ? -INFINITY : (most == -INFINITY ? 0.f : most) * 0.6931471805599453f + logf(total);
}
// Eight elements of head row r, a sum of its parts; n: the request's slots
template <class T>
__device__ __forceinline__ void attend_write(const AttentionArgs &a, int64_t r, int at, float (&y)[8], float most, float total, int n) {
    const float by = total * attend_scale<T>(n);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = total == 0.f ? 0.f : y[j] / by;
    Eight<T> e;
    e.set(y);
    e.store(static_cast<char *>(a.out) + (r * a.cache.d + at) * T::bytes);
    if (at == 0 && a.lse) a.lse[r] = attend_lse(most, total);
}

// The parts of head row r, joined: by a wave if there are at most ATTEND_FEW of them, which are then all asked for before the request's length says how many
// there are; else by the workgroup.  per_row lanes (at most 32) share a row, and rows lie side by side.  lds: 8 floats for each thread.
template <class T>
__device__ __forceinline__ void attend_join_few(const AttentionArgs &a, int64_t r, float *lds) {
    const int per_row = a.cache.d / 8, lane = threadIdx.x & (WAVE - 1), side = WAVE / per_row, first = lane / per_row;
    const float *from = a.partial + r * a.splits * a.cache.d + (lane % per_row) * 8;
    const float2 own = lane < a.splits ? reinterpret_cast<const float2 *>(a.stats)[r * a.splits + lane] : float2{-INFINITY, 0.f};
    constexpr int AHEAD = 4;
    f4 z[AHEAD][2];
    auto ask = [&](int s0) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int s = s0 + k * side;
            if (first < side && s < a.splits) {
                z[k][0] = reinterpret_cast<const f4 *>(from + (int64_t)s * a.cache.d)[0];
                z[k][1] = reinterpret_cast<const f4 *>(from + (int64_t)s * a.cache.d)[1];
            }
        }
    };
    ask(first);
    const AttendSpan span = attend_span(a, (int)(r / a.q_heads));
    const int parts = max(1, span.parts);
    const float t = lane < parts ? own.x : -INFINITY, most = wave_max(t);
    // (a part without a score has a sum of 0, or NaN, and counts as it is)
    const float f = lane >= parts ? 0.f : t == -INFINITY ? 1.f : exp2_fast(t - most), total = wave_sum(lane < parts ? own.y * f : 0.f);
    float y[8] = {};
    for (int s0 = first; s0 - first < parts; s0 += AHEAD * side) {
        if (s0 != first) ask(s0);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int s = s0 + k * side;
            const float g = __shfl(f, s & (WAVE - 1));
            if (first < side && s < parts) {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = fmaf(z[k][j / 4][j % 4], g, y[j]);
            }
        }
    }
    f4 *mine = reinterpret_cast<f4 *>(lds + threadIdx.x * 8);
    mine[0] = f4{y[0], y[1], y[2], y[3]};
    mine[1] = f4{y[4], y[5], y[6], y[7]};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");                  // (what the wave itself wrote)
    if (lane < per_row) {
        for (int s = 1; s < side && s < parts; ++s) {
            const f4 *o = reinterpret_cast<const f4 *>(lds + (threadIdx.x + s * per_row) * 8);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] += o[j / 4][j % 4];
        }
        attend_write<T>(a, r, 8 * lane, y, most, total, span.n);
    }
}
template <class T>
__device__ __forceinline__ void attend_join(const AttentionArgs &a, int64_t r, float *lds) {
    const AttendSpan span = attend_span(a, (int)(r / a.q_heads));
    const int parts = max(1, span.parts), per_row = a.cache.d / 8, tid = threadIdx.x, side = ATTEND_THREADS / per_row;
    const float *from = a.partial + r * a.splits * a.cache.d + (tid % per_row) * 8;
    const float *st = a.stats + r * a.splits * 2;
    float most, total, y[8] = {};
    attend_stats(a, r, parts, most, total);
    if (tid < side * per_row) {
#pragma unroll 4
        for (int s = tid / per_row; s < parts; s += side) {
            const f4 *z = reinterpret_cast<const f4 *>(from + (int64_t)s * a.cache.d);
            const f4 z0 = z[0], z1 = z[1];
            const float t = st[2 * s], f = t == -INFINITY ? 1.f : exp2_fast(t - most);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                y[j] = fmaf(z0[j], f, y[j]);
                y[4 + j] = fmaf(z1[j], f, y[4 + j]);
            }
        }
    }
    f4 *mine = reinterpret_cast<f4 *>(lds + tid * 8);
    mine[0] = f4{y[0], y[1], y[2], y[3]};
    mine[1] = f4{y[4], y[5], y[6], y[7]};
    __syncthreads();
    if (tid < per_row) {
        for (int s = 1; s < side && s < parts; ++s) {
            const f4 *o = reinterpret_cast<const f4 *>(lds + (tid + s * per_row) * 8);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] += o[j / 4][j % 4];
        }
        attend_write<T>(a, r, 8 * tid, y, most, total, span.n);
    }
}

// Whether `weight` is slot key's: one without a row has 0, but where a head's scores hold a NaN, and is left alone then.
__device__ __forceinline__ bool attend_counts(const AttentionArgs &a, int b, int key, float weight) {
    return weight == weight || (unsigned)a.table[(int64_t)b * a.width + (key >> a.cache.slots_log)] < (unsigned)a.cache.pages;
}

// By a workgroup: the weights of slots start + j0 .. of a cache head, ATTEND_PIECE of them, summed over its query heads in their order and added to mass.
constexpr int ATTEND_PIECE = 4 * ATTEND_THREADS;
__device__ __forceinline__ void attend_add_mass(const AttentionArgs &a, int b, int h, const AttendSpan &span, int j0, float *lds) {
    const int G = a.q_heads / a.cache.heads, tid = threadIdx.x, j = j0 + 4 * tid, from = span.lo - span.start, count = span.n - span.start;
    f4 w = {0.f, 0.f, 0.f, 0.f};
    for (int g0 = 0; g0 < G; g0 += ATTEND_THREADS) {      // (one round as a rule)
        const int heads = min(ATTEND_THREADS, G - g0);
        for (int i = tid / WAVE; i < heads; i += ATTEND_WAVES) {
            float most, total;
            attend_stats(a, (int64_t)b * a.q_heads + h * G + g0 + i, span.parts, most, total);
            lds[2 * i] = most == -INFINITY ? 0.f : most;
            lds[2 * i + 1] = total == 0.f ? 0.f : 1.f / total;
        }
        __syncthreads();
        if (j < count) {
            const float *x = a.scores + ((int64_t)b * a.q_heads + h * G + g0) * a.pad + j;
#pragma unroll 4
            for (int i = 0; i < heads; ++i) {
                const f4 s = *reinterpret_cast<const f4 *>(x + (int64_t)i * a.pad);
                const float most = lds[2 * i], f = lds[2 * i + 1];
#pragma unroll
                for (int c = 0; c < 4; ++c) w[c] += exp2_fast(s[c] - most) * f;
            }
        }
        __syncthreads();
    }
    float *to = a.mass + ((int64_t)b * a.cache.heads + h) * a.mass_slots + span.start + j;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (j + c >= from && j + c < count && attend_counts(a, b, span.start + j + c, w[c])) to[c] += w[c];
}

// FINE: pages of less than 16 slots, looked up for every row and not for a tile.  FULL: d is 16 VE.  ONCE: keys and values are more than the
// last cache holds, and are read past it.  MT: tiles of 16 query heads.
template <class T, int VE, int MT, bool FINE, bool FULL, bool ONCE>
__global__ __launch_bounds__(ATTEND_THREADS, (MT > 1 && (VE == 16 || T::bytes == 4)) || (VE == 16 && T::bytes == 2 && (FINE || !FULL)) ? 1 : 2) void paged_attention_kernel(AttentionArgs a) {
    typedef AttendShape<T, VE> Sh;
    typedef typename Words<Sh::CW>::type VChunk;
    constexpr int NT = Sh::NT, NS = Sh::NS, NU = Sh::NU, CE = Sh::CE, STEP = 16 * NT * ATTEND_WAVES;
    extern __shared__ __align__(16) float lds[];
    const int lane = threadIdx.x & (WAVE - 1), g = lane >> 4, m = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    // First parts of all contexts first.  Workgroups are dealt out in their order, to the 8 XCDs and inside an XCD to its 4 shader engines, whatever
    // they have still to do; from part to part a context moves on by one XCD and by one engine, or the long ones of a batch would all be
    // a few engines' (every second of 64 requests 8 times as long as the others: 542 -> 430 us).  The workgroups that read the same slots for
    // other query heads follow each other on one XCD.
    const int hg = (blockIdx.x >> 3) % a.groups, item = (blockIdx.x >> 3) / a.groups * 8 + (blockIdx.x & 7);
    const int units = a.requests * a.cache.heads, part = item / units, unit = (item % units + 9 * part) % units;
    if (part >= a.splits) return;
    const int h = unit % a.cache.heads, b = unit / a.cache.heads;
    const int G = a.q_heads / a.cache.heads, rows = min(16 * MT, G - 16 * MT * hg);   // query heads of this workgroup
    const AttendSpan span = attend_span(a, b);
    const int n = span.n, lo = span.lo, start = span.start, first = start + part * a.chunk, end = attend_end(n, first, a.chunk);
    if (part >= max(span.parts, 1)) return;               // (the first part of nothing says so)
    const int64_t hq0 = (int64_t)b * a.q_heads + h * G + 16 * MT * hg;
    const float scale = attend_scale<T>(n);

    // (LDS: what the waves' sums are written over afterwards)
    constexpr bool Q_LDS = attend_q_in_lds(VE);
    constexpr int HEADS = 16 * MT, LD = attend_lds_row(VE);
    float *s_top = lds, *s_sum = lds + ATTEND_WAVES * HEADS, *s_o = lds + 2 * ATTEND_WAVES * HEADS;
    float *s_x = s_o + max(ATTEND_WAVES * rows * LD, Q_LDS ? MT * NS * WAVE * 4 : 0);   // scores that stay here
    u4 *s_q = reinterpret_cast<u4 *>(s_o), q[Q_LDS ? 1 : MT][Q_LDS ? 1 : NS];
    auto query = [&](int mt, int s) {                     // this lane's operand of step s
        u4 x = zero_chunk();
        const int at = (4 * s + g) * 16;
        if (16 * mt + m < rows && (FULL || at < a.cache.d * T::bytes))
            x = load_chunk(static_cast<const char *>(a.q) + b * a.q_row + (h * G + 16 * (MT * hg + mt) + m) * a.q_head + at);
        return x;
    };
    if constexpr (Q_LDS) {
        for (int i = wave; i < MT * NS; i += ATTEND_WAVES) s_q[i * WAVE + lane] = query(i / NS, i % NS);
    } else {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int s = 0; s < NS; ++s) q[mt][s] = query(mt, s);
    }
    const int32_t *table = a.table + (int64_t)b * a.width;
    const int slots_log = a.cache.slots_log, mask = (1 << slots_log) - 1;
    const char *k_head = a.cache.k + h * a.cache.k_head, *v_head = a.cache.v + h * a.cache.v_head;
    // where a row is that may be read: its own, or for one that is not there the first of the cache
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
            const int key = k0 + 16 * t + 4 * g;
            out.k[t] = row_page(k0 + 16 * t + m);
            out.v[t][0] = row_page(key);
#pragma unroll
            for (int i = 1; i < (FINE ? 4 : 1); ++i) {
                if (slots_log >= 2) out.v[t][i] = key + i < end ? out.v[t][0] : -1;
                else out.v[t][i] = row_page(key + i);
            }
        }
    };
    auto load_k = [&](int k0, const Pages &pg) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int key = k0 + 16 * t + m, p = pg.k[t];
            const char *row = k_head + (int64_t)max(p, 0) * a.cache.k_page + (FINE && p < 0 ? 0 : key & mask) * a.cache.k_slot;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const int at = (4 * s + g) * 16;
                if (FULL || at < a.cache.d * T::bytes) kr[t][s] = stream_load<ONCE>(reinterpret_cast<const u4 *>(row + at));
                else kr[t][s] = zero_chunk();
            }
        }
    };

    f4 o[MT][VE];
    float top[MT], sum[MT];                               // of head 16 mt + m; the sum of this lane's slots alone
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int c = 0; c < VE; ++c) o[mt][c] = f4{0.f, 0.f, 0.f, 0.f};
        top[mt] = -INFINITY;
        sum[mt] = 0.f;
    }
    int k0 = first + wave * 16 * NT;
    if (k0 < end) {
        pages_of(k0, page);
        load_k(k0, page);
    }
    if constexpr (Q_LDS) __syncthreads();
    for (; k0 < end; k0 += STEP) {
        const bool more = k0 + STEP < end;
        if (more) pages_of(k0 + STEP, page_next);
        VChunk vr[NT][4][NU];
        unsigned there = 0;                               // FINE: which of the lane's slots have a row
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = k0 + 16 * t + 4 * g + i, p = FINE ? page.v[t][FINE ? i : 0] : page.k[t];
                if (FINE && p >= 0 && key >= lo) there |= 1u << (4 * t + i);
                const char *row = v_head + (int64_t)max(p, 0) * a.cache.v_page + (FINE && p < 0 ? 0 : key & mask) * a.cache.v_slot;
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const int at = (u * 16 + m) * CE;
                    if (FULL || at < a.cache.d) vr[t][i][u] = stream_load<ONCE>(reinterpret_cast<const VChunk *>(row + at * T::bytes));
                    else vr[t][i][u] = VChunk(0);
                }
            }
        }
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
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int t = 0; t < NT; ++t) x[mt][t] *= a.scale;
        bool whole = k0 >= lo && k0 + 16 * NT <= end;
#pragma unroll
        for (int t = 0; t < NT; ++t) whole = whole && page.k[t] >= 0;
        if (FINE || !whole) {                             // slots that do not count: no score, and no value that could be NaN
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = k0 + 16 * t + 4 * g + i;
                    const bool use = FINE ? (there >> (4 * t + i)) & 1 : page.k[t] >= 0 && key >= lo && key < end;
                    if (!use) {
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) x[mt][t][i] = -INFINITY;
#pragma unroll
                        for (int u = 0; u < NU; ++u) vr[t][i][u] = VChunk(0);
                    }
                }
            }
        }
        if (a.scores || a.keep) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                if (16 * mt + m < rows) {
                    float *to = a.keep ? s_x + (16 * mt + m) * a.keep : a.scores + (hq0 + 16 * mt + m) * a.pad;
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const int at = k0 - start + 16 * t + 4 * g;
                        if (!a.keep || at < n - start) *reinterpret_cast<f4 *>(to + at) = x[mt][t];
                    }
                }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {                 // x becomes the weights
            float most = x[mt][0][0];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) most = fmaxf(most, x[mt][t][i]);
            const float now = fmaxf(top[mt], column_max(most)), base = now == -INFINITY ? 0.f : now, keep = exp2_fast(top[mt] - base), lifted = base - ATTEND_LIFT<T>;
            top[mt] = now;
            sum[mt] *= keep;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[mt][t][i] = exp2_fast(x[mt][t][i] - lifted);
                    sum[mt] += x[mt][t][i];
                    if (!std::is_same_v<T, F16>) x[mt][t][i] *= scale;
                }
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
                            v[k] = __builtin_amdgcn_perm(vr[t + k / 2][2 * (k & 1) + 1][u][c / 2], vr[t + k / 2][2 * (k & 1)][u][c / 2],
                                                         c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            f4 &acc = o[mt][u * CE + c];
                            acc = mfma16<T>(v, high[mt], acc);
                            acc = mfma16<T>(v, low[mt], acc);
                        }
                    }
            }
        } else {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int u = 0; u < NU; ++u)
#pragma unroll
                        for (int c = 0; c < CE; ++c)
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt)
                                o[mt][u * CE + c] =
                                    __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[t][i][u][c]), x[mt][t][i], o[mt][u * CE + c], 0, 0, 0);
        }
        page = page_next;
    }

    // the waves' sums, joined (of those that had a slot): lane 16 g + m holds elements CE (4 g + i) .. of every 16 CE, head 16 mt + m
    const int used = min(ATTEND_WAVES, (max(end - first, 1) + 16 * NT - 1) / (16 * NT));
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        sum[mt] = column_sum(sum[mt]) * (1.f / (1 << ATTEND_LIFT<T>));
        if (g == 0) {
            s_top[wave * HEADS + 16 * mt + m] = top[mt];
            s_sum[wave * HEADS + 16 * mt + m] = sum[mt];
        }
    }
    __syncthreads();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int head = 16 * mt + m;
        float all = -INFINITY;
#pragma unroll
        for (int w = 0; w < ATTEND_WAVES; ++w) all = fmaxf(all, s_top[w * HEADS + head]);
        const float mine = top[mt] == -INFINITY ? 0.f : exp2_fast(top[mt] - all) * (1.f / (1 << ATTEND_LIFT<T>));
        if (head < rows && wave < used) {
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < CE; c += 4) {
                        const int at = (u * 16 + 4 * g + i) * CE + c, e = u * CE + c;
                        *reinterpret_cast<f4 *>(s_o + (wave * rows + head) * LD + at) = f4{o[mt][e][i], o[mt][e + 1][i], o[mt][e + 2][i], o[mt][e + 3][i]} * mine;
                    }
        }
    }
    __syncthreads();
    const int per_row = a.cache.d / 8;
    for (int i = threadIdx.x; i < rows * per_row; i += ATTEND_THREADS) {
        const int r = i / per_row, at = (i % per_row) * 8;
        float most = -INFINITY, total = 0.f;
#pragma unroll
        for (int w = 0; w < ATTEND_WAVES; ++w) most = fmaxf(most, s_top[w * HEADS + r]);
#pragma unroll
        for (int w = 0; w < ATTEND_WAVES; ++w) {
            const float t = s_top[w * HEADS + r];
            // (a NaN among the scores is in the sum, whatever the maximum says)
            total += s_sum[w * HEADS + r] * (t == -INFINITY ? 1.f : exp2_fast(t - most));
        }
        float y[8] = {};
        for (int w = 0; w < used; ++w) {
            const float *z = s_o + (w * rows + r) * LD + at;
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] += z[j];
        }
        if (at == 0 && a.stats) {
            a.stats[((hq0 + r) * a.splits + part) * 2] = most;
            a.stats[((hq0 + r) * a.splits + part) * 2 + 1] = total;
        }
        if (a.splits > 1) {
            float *to = a.partial + ((hq0 + r) * a.splits + part) * a.cache.d + at;
            reinterpret_cast<f4 *>(to)[0] = f4{y[0], y[1], y[2], y[3]};
            reinterpret_cast<f4 *>(to)[1] = f4{y[4], y[5], y[6], y[7]};
        } else {
            const float f = total == 0.f ? 0.f : 1.f / (total * scale);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = total == 0.f ? 0.f : y[j] * f;
            Eight<T> e;
            e.set(y);
            e.store(static_cast<char *>(a.out) + ((hq0 + r) * a.cache.d + at) * T::bytes);
            if (at == 0 && a.lse) a.lse[hq0 + r] = attend_lse(most, total);
        }
    }
    if (!a.keep) return;

    // the only part: the weights of its slots, summed over the query heads in their order, are added to mass
    __syncthreads();
    for (int r = threadIdx.x; r < rows; r += ATTEND_THREADS) {
        float most = -INFINITY, total = 0.f;
        for (int w = 0; w < ATTEND_WAVES; ++w) most = fmaxf(most, s_top[w * HEADS + r]);
        for (int w = 0; w < ATTEND_WAVES; ++w) {
            const float t = s_top[w * HEADS + r];
            total += s_sum[w * HEADS + r] * (t == -INFINITY ? 1.f : exp2_fast(t - most));
        }
        s_o[2 * r] = most == -INFINITY ? 0.f : most;
        s_o[2 * r + 1] = total == 0.f ? 0.f : 1.f / total;
    }
    __syncthreads();
    float *mass = a.mass + ((int64_t)b * a.cache.heads + h) * a.mass_slots;
    for (int j = lo + threadIdx.x; j < n; j += ATTEND_THREADS) {
        float w = 0.f;
        for (int r = 0; r < rows; ++r) w += exp2_fast(s_x[r * a.keep + j - start] - s_o[2 * r]) * s_o[2 * r + 1];
        if (attend_counts(a, b, j, w)) mass[j] += w;
    }
}

// What the parts of a context left, joined by a launch of its own: the workgroup that is done last was slower at it behind __threadfence, which writes back an XCD's
// whole L2 (one request of 1500 slots: 16.9 us against 10.2); stores and loads at agent scope, which pass the L2 by, were not tried.  The first workgroups take query heads: a wave to a head if there are few parts (FEW), else a
// workgroup to a head; none do where there is one part only.  Those behind them (scores given) take a piece of the slots of a cache head each.
template <class T, bool FEW>
__global__ __launch_bounds__(ATTEND_THREADS) void paged_attention_join_kernel(AttentionArgs a) {
    __shared__ __align__(16) float lds[ATTEND_THREADS * 8];
    const int64_t heads_all = a.splits > 1 ? (int64_t)a.requests * a.q_heads : 0, head_groups = FEW ? (heads_all + ATTEND_WAVES - 1) / ATTEND_WAVES : heads_all;
    if ((int64_t)blockIdx.x < head_groups) {
        const int64_t r = FEW ? (int64_t)blockIdx.x * ATTEND_WAVES + threadIdx.x / WAVE : blockIdx.x;
        if (r < heads_all) {
            if (FEW) attend_join_few<T>(a, r, lds);
            else attend_join<T>(a, r, lds);
        }
        return;
    }
    const int64_t id = blockIdx.x - head_groups;
    const int pieces = (a.pad + ATTEND_PIECE - 1) / ATTEND_PIECE, j0 = (int)(id % pieces) * ATTEND_PIECE;
    const int b = (int)(id / pieces / a.cache.heads), h = (int)(id / pieces % a.cache.heads);
    const AttendSpan span = attend_span(a, b);
    if (j0 < span.n - span.start) attend_add_mass(a, b, h, span, j0, lds);
}

template <class T, int VE, int MT, bool FINE, bool FULL, bool ONCE>
hipError_t attend(const AttentionArgs &a, hipStream_t stream) {
    static size_t granted = 0;
    const size_t bytes = attend_lds_bytes(T::bytes, VE, MT, a.q_heads / a.cache.heads, a.keep);
    const void *kernel = reinterpret_cast<const void *>(paged_attention_kernel<T, VE, MT, FINE, FULL, ONCE>);
    if (hipError_t e = allow_big_lds(kernel, bytes, &granted)) return e;
    const int items = (a.requests * a.cache.heads * a.splits + 7) / 8 * 8;
    hipLaunchKernelGGL((paged_attention_kernel<T, VE, MT, FINE, FULL, ONCE>), dim3(items * a.groups), dim3(ATTEND_THREADS), bytes, stream, a);
    return hipGetLastError();
}

// (variants that few calls would tell apart share the general one: caches of small pages, and of many heads with d < 16 VE, are not read past the last cache)
template <class T, int VE>
hipError_t attend(const AttentionArgs &a, bool once, hipStream_t stream) {
    constexpr int MT = attend_head_tiles(T::bytes, VE, 17);
    const bool full = a.cache.d == 16 * VE, fine = a.cache.slots_log < 4;
    if constexpr (MT > 1) {
        if (a.q_heads / a.cache.heads > 16)
            return fine ? attend<T, VE, MT, true, false, false>(a, stream) : !full ? attend<T, VE, MT, false, false, false>(a, stream)
                   : once ? attend<T, VE, MT, false, true, true>(a, stream) : attend<T, VE, MT, false, true, false>(a, stream);
    }
    if (fine) return full ? attend<T, VE, 1, true, true, false>(a, stream) : attend<T, VE, 1, true, false, false>(a, stream);
    if (once) return full ? attend<T, VE, 1, false, true, true>(a, stream) : attend<T, VE, 1, false, false, true>(a, stream);
    return full ? attend<T, VE, 1, false, true, false>(a, stream) : attend<T, VE, 1, false, false, false>(a, stream);
}

template <class T>
hipError_t launch_attention(const AttentionArgs &a, bool once, hipStream_t stream) {
    const int ve = attend_ve(a.cache.d), B = a.requests;
    if (hipError_t e = ve == 4 ? attend<T, 4>(a, once, stream) : ve == 8 ? attend<T, 8>(a, once, stream) : attend<T, 16>(a, once, stream)) return e;
    if (a.splits == 1 && !a.scores) return hipSuccess;
    const int pieces = a.scores ? (a.pad + ATTEND_PIECE - 1) / ATTEND_PIECE : 0, rows = a.splits > 1 ? B * a.q_heads : 0, mass = B * a.cache.heads * pieces;
    // (64 heads of 64 requests in 5 parts: 10.2 us a workgroup to a head, a wave to a head 5.9)
    if (a.splits <= ATTEND_FEW)
        hipLaunchKernelGGL((paged_attention_join_kernel<T, true>), dim3((rows + ATTEND_WAVES - 1) / ATTEND_WAVES + mass), dim3(ATTEND_THREADS), 0, stream, a);
    else
        hipLaunchKernelGGL((paged_attention_join_kernel<T, false>), dim3(rows + mass), dim3(ATTEND_THREADS), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ann
