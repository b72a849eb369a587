// Attention of many rows: which rows and slots a workgroup takes.
//
// A pass goes through tiles of `rows` rows of sequences of tokens: a request's new ones (CHUNK_NEW), the one of each request of a group (CHUNK_COMMON: the slots in common), or a
// request's one (CHUNK_OWN: its own slots; CHUNK_ALL: those in common too).  A token has a row for each of the G query heads of a cache head.  Long ranges of slots are divided into parts.
// How many tiles and slots there are is known on the
// device alone; up to 64 sequences, a lane each, every workgroup works out for itself how the whole is dealt: parts as long as fill the card, longest sequences first.
#pragma once

#include "launch.hpp"
#include "packed.hpp"
#include "paged_attention_kernel.hpp"

namespace ann {

struct ChunkSpan { int lo, hi; };                         // slots lo .. hi - 1
// Parts begin with multiples of 32 slots, so that 16 rows from a multiple of 16 on are loaded together.
__device__ __forceinline__ int chunk_begin(ChunkSpan range) { return min(range.lo, range.hi) & ~31; }
__device__ __forceinline__ int chunk_slots_of(ChunkSpan range) { return range.hi - chunk_begin(range); }
// Parts of `chunk` slots; the first part of nothing says so.  (There are few: of a quotient below 2^20 a float is off by less than one.)
__device__ __forceinline__ int chunk_parts(int slots, int chunk) {
    if (slots <= chunk) return 1;
    const int guess = (int)((float)(slots - 1) * __builtin_amdgcn_rcpf((float)chunk)), left = (int)((uint32_t)(slots - 1) - (uint32_t)guess * (uint32_t)chunk);
    return guess + 1 + (left >= chunk) - (left < 0);
}

__device__ __forceinline__ int chunk_length(const ChunkArgs &a, int request) { return max(a.lengths[request], 0); }

// The group of request t, or -1, and how many slots it has in common.  By whole waves, whose lanes may ask for different requests.
struct ChunkGroup { int group, common; };
__device__ __forceinline__ int chunk_common(const ChunkArgs &a, int g) { return g < 0 ? 0 : min(max(a.shared[g], 0), a.max_shared); }
__device__ __forceinline__ ChunkGroup chunk_group(const ChunkArgs &a, int t) {
    int n = 0;                                            // starts up to t
    if (a.groups < WAVE) {
        const int lane = threadIdx.x & (WAVE - 1), start = lane <= a.groups ? packed_start(a.group_starts, lane, a.tokens) : INT_MAX, common = lane < a.groups ? chunk_common(a, lane) : 0;
        for (int g = 0; g <= a.groups; ++g) n += __builtin_amdgcn_readlane(start, g) <= t;
        const bool in = n > 0 && n <= a.groups;
        const int mine = __shfl(common, in ? n - 1 : 0);  // (by all lanes: a lane whose request is in no group may hold what others ask for, and a lane that does not take part gives 0)
        return in ? ChunkGroup{n - 1, mine} : ChunkGroup{-1, 0};
    }
    for (int left = a.groups + 1; left > 0;) {            // (halves)
        const int half = left / 2;
        if (packed_start(a.group_starts, n + half, a.tokens) <= t) { n += half + 1; left -= half + 1; }
        else left = half;
    }
    return n > 0 && n <= a.groups ? ChunkGroup{n - 1, chunk_common(a, n - 1)} : ChunkGroup{-1, 0};
}

struct ChunkSequence { int token0, tokens, request; };    // request: whose pages are read
__device__ __forceinline__ int chunk_sequences(const ChunkArgs &a, int mode) { return mode == CHUNK_NEW ? a.requests : mode == CHUNK_COMMON ? a.groups : a.tokens; }
__device__ __forceinline__ ChunkSequence chunk_sequence(const ChunkArgs &a, int mode, int i) {
    if (mode >= CHUNK_OWN) return {i, 1, i};
    const int32_t *starts = mode == CHUNK_NEW ? a.starts : a.group_starts;
    const int s0 = packed_start(starts, i, a.tokens), s1 = packed_start(starts, i + 1, a.tokens);
    return {s0, max(s1 - s0, 0), mode == CHUNK_NEW ? i : min(s0, a.tokens - 1)};
}
// Slots that the token `left` from the end of a request of `length` slots attends to.
__device__ __forceinline__ ChunkSpan chunk_span(const ChunkArgs &a, int length, int left) {
    const int slot = length - left;
    if (slot < 0 || slot >= a.max_length) return {0, 0};
    return {a.window > 0 ? max(slot + 1 - a.window, 0) : 0, slot + 1};
}
// What a wave knows of a sequence: of one, or each lane of another.
struct ChunkKnown {
    ChunkSequence q;
    int length, common;       // slots of q.request, at least 0; of its group in common
    int grouped;              // q.request is in a group
};
__device__ __forceinline__ ChunkKnown chunk_known(const ChunkArgs &a, int mode, int i) {
    ChunkKnown k{chunk_sequence(a, mode, i), 0, 0, 0};
    k.length = chunk_length(a, k.q.request);
    if (mode == CHUNK_COMMON) k.common = chunk_common(a, i);
    if (mode >= CHUNK_OWN) {
        const ChunkGroup g = chunk_group(a, i);
        k.common = g.common;
        k.grouped = g.group >= 0;
    }
    return k;
}
// Slots that tokens t0 to t1 of a sequence attend to, all of them together.
__device__ __forceinline__ ChunkSpan chunk_range(const ChunkArgs &a, int mode, const ChunkKnown &k, int t0, int t1) {
    if (mode == CHUNK_NEW) {
        const int first = k.length - (k.q.tokens - t0), last = k.length - (k.q.tokens - t1);
        return {a.window > 0 ? max(max(first, 0) + 1 - a.window, 0) : 0, min(max(last + 1, 0), a.max_length)};     // (first is below 0 where tokens have no slot, and the window may be the largest number)
    }
    if (mode == CHUNK_COMMON) return {0, k.common};
    const int n = min(k.length, a.max_length), common = min(n, k.common);
    return {mode == CHUNK_ALL ? 0 : common, common + min(n - common, a.max_own)};
}

// Sums and largest over a wave, without LDS
__device__ __forceinline__ int wave_sum_of(int x) {
    x += (int)lane_swap<1>((uint32_t)x);
    x += (int)lane_swap<2>((uint32_t)x);
    x += (int)lane_swap<4>((uint32_t)x);
    x += (int)lane_swap<8>((uint32_t)x);
    uint32_t a, b;
    row_pair<16>((uint32_t)x, a, b);
    x = (int)(a + b);
    row_pair<32>((uint32_t)x, a, b);
    return (int)(a + b);
}
// ... over the lanes below each
__device__ __forceinline__ int wave_sum_before(int x) {
    const int lane = threadIdx.x & (WAVE - 1);
    int all = x, before = 0;                              // of a block of lanes, and of those of it below this one
    auto step = [&](int mask, int other) { before += lane & mask ? other : 0; all += other; };
    step(1, (int)lane_swap<1>((uint32_t)all));
    step(2, (int)lane_swap<2>((uint32_t)all));
    step(4, (int)lane_swap<4>((uint32_t)all));
    step(8, (int)lane_swap<8>((uint32_t)all));
    uint32_t a, b;
    row_pair<16>((uint32_t)all, a, b);
    step(16, (int)(a + b) - all);
    row_pair<32>((uint32_t)all, a, b);
    step(32, (int)(a + b) - all);
    return before;
}
__device__ __forceinline__ int wave_max_of(int x) {
    x = max(x, (int)lane_swap<1>((uint32_t)x));
    x = max(x, (int)lane_swap<2>((uint32_t)x));
    x = max(x, (int)lane_swap<4>((uint32_t)x));
    x = max(x, (int)lane_swap<8>((uint32_t)x));
    uint32_t a, b;
    row_pair<16>((uint32_t)x, a, b);
    x = max((int)a, (int)b);
    row_pair<32>((uint32_t)x, a, b);
    return max((int)a, (int)b);
}

// Slots of a part, up to 64 sequences: lane i has so many tiles and slots of sequence i.  The fewest, in whole tiles of 64, with which no more workgroups have something to do than fill the card,
// once, or twice if tiles of many rows alone make up much of it.
__device__ __forceinline__ int chunk_even(const ChunkPass &p, int tiles, int slots) {
    if (p.most_parts == 1) return INT_MAX;
    const int most = __builtin_amdgcn_readfirstlane(wave_max_of(slots)), all_tiles = __builtin_amdgcn_readfirstlane(wave_sum_of(tiles));
    const int64_t limit = (p.rows == CHUNK_TILE && 4 * (int64_t)all_tiles > p.fill ? 2 : 1) * (int64_t)p.fill;
    if (most <= p.whole && all_tiles >= p.units) return INT_MAX;
    if (limit <= all_tiles) return INT_MAX;
    const float all = wave_sum((float)tiles * (float)slots);
    // in units of 64 slots, of which there are 2^20: `few` are too few or just enough, `enough` are not too few
    const int least = (max(p.least, (most - 1) / p.most_parts + 1) + 63) / 64;
    int few = max((int)min(all / (64.f * (float)limit), 1e7f), least), enough = max((int)min(all / (64.f * (float)(limit - all_tiles)), 1e7f) + 1, least);
    while (few < enough) {
        const int half = (few + enough) / 2;
        if (wave_sum_of(tiles * chunk_parts(slots, 64 * half)) <= limit) enough = half;
        else few = half + 1;
        few = __builtin_amdgcn_readfirstlane(few);
        enough = __builtin_amdgcn_readfirstlane(enough);
    }
    return 64 * enough;
}

// What a workgroup does: slots first .. end - 1 of the tile that begins with row r0 of a sequence, of whose range they are part `part`; count 0: nothing.
struct ChunkDeal {
    ChunkKnown k;
    int r0, count, part, parts;
    int alone;                // nothing is to be joined with it
    ChunkSpan range;          // of the tile's rows, all together
    int first, end;
};
__device__ __forceinline__ ChunkDeal chunk_deal_of(const ChunkArgs &a, const ChunkPass &p, int item, int G) {
    const int n = chunk_sequences(a, p.mode), lane = threadIdx.x & (WAVE - 1), rows_log = __ffs(p.rows) - 1;
    ChunkDeal d{};
    int chunk;
    if (n <= WAVE && !(p.mode >= CHUNK_OWN && p.most_parts == 1)) {         // (own slots that are not divided: all have as many items)
        const ChunkKnown k = chunk_known(a, p.mode, min(lane, n - 1));
        const int tiles = lane < n ? (k.q.tokens * G + p.rows - 1) >> rows_log : 0;
        // (the last tile has most slots, but for what a window leaves it)
        const int t0 = p.mode == CHUNK_NEW ? (int)((uint32_t)max(tiles - 1, 0) * p.rows / (uint32_t)G) : 0;
        const ChunkSpan last = chunk_range(a, p.mode, k, t0, max(k.q.tokens - 1, 0));
        int slots = tiles > 0 ? chunk_slots_of(last) : 0;
        if (tiles > 0 && p.mode == CHUNK_NEW && a.window > 0) slots = (int)max((int64_t)slots, min((int64_t)last.hi, (int64_t)a.window + p.rows + 32));
        chunk = chunk_even(p, tiles, slots);
        const int items = tiles * chunk_parts(slots, chunk);
        int before;
        if (p.items > p.fill) {                           // items of longer sequences go first (of two as long, the first's)
            const uint32_t key = (uint32_t)min(slots, (1 << 26) - 1) << 6 | (WAVE - 1 - lane);
            before = 0;
            for (int i = 0; i < n; ++i) before += (uint32_t)__builtin_amdgcn_readlane((int)key, i) > key ? __builtin_amdgcn_readlane(items, i) : 0;
        } else {                                          // all are on the card at once
            before = wave_sum_before(items);
        }
        const uint64_t mine = __ballot(item >= before && item < before + items);
        if (mine == 0) return d;
        const int i = __ffsll((unsigned long long)mine) - 1;
        auto of = [&](int x) { return __builtin_amdgcn_readlane(x, i); };
        const int local = item - of(before), its = of(tiles);
        d.part = local / its;
        d.r0 = (its - 1 - local % its) * p.rows;
        d.k = ChunkKnown{{of(k.q.token0), of(k.q.tokens), of(k.q.request)}, of(k.length), of(k.common), of(k.grouped)};
    } else {
        // A sequence of m tokens has at most as many tiles as there are numbers from start G / rows + i up to the next one's.
        const int id = p.tiles - 1 - item % p.tiles;
        int i;
        int tile;
        d.part = item / p.tiles;
        chunk = p.chunk;
        if (p.mode >= CHUNK_OWN) {
            const int per = (G + p.rows - 1) >> rows_log;
            i = id / per;
            tile = id % per;
            if (i >= n) return d;
        } else {
            const int32_t *starts = p.mode == CHUNK_NEW ? a.starts : a.group_starts;
            auto first = [&](int k) { return (packed_start(starts, k, a.tokens) * G >> rows_log) + k; };
            i = __builtin_amdgcn_readfirstlane(count_up_to(first, n + 1, id)) - 1;
            if (i < 0 || i >= n) return d;
            tile = id - first(i);
        }
        d.r0 = tile * p.rows;
        d.k = chunk_known(a, p.mode, i);
        d.k.common = __builtin_amdgcn_readfirstlane(d.k.common);             // (the same in all lanes, which the compiler cannot know)
        d.k.grouped = __builtin_amdgcn_readfirstlane(d.k.grouped);
    }
    const int count = max(0, min(p.rows, d.k.q.tokens * G - d.r0));
    if (count == 0) return d;
    d.range = chunk_range(a, p.mode, d.k, d.r0 / G, (d.r0 + count - 1) / G);
    d.parts = chunk_parts(chunk_slots_of(d.range), chunk);
    if (d.part >= d.parts) return d;
    d.count = count;
    d.alone = p.mode == CHUNK_NEW && d.parts == 1;
    d.first = chunk_begin(d.range) + d.part * chunk;
    d.end = d.range.hi - d.first < chunk ? d.range.hi : d.first + chunk;
    return d;
}
// ... worked out by one wave: a SIMD has waves of several workgroups and issues for one at a time (8 requests of 2000 slots, 8 heads of 128: 20.4 us by each wave, 19.2 so; 128 x 125 slots
// 18.4 and 17.4).
__device__ __forceinline__ ChunkDeal chunk_deal(const ChunkArgs &a, const ChunkPass &p, int item, int G) {
    constexpr int WORDS = sizeof(ChunkDeal) / 4;
    struct Words { int w[WORDS]; };
    __shared__ int s_deal[WORDS];
    if (threadIdx.x < WAVE) {
        const Words words = __builtin_bit_cast(Words, chunk_deal_of(a, p, item, G));
        if (threadIdx.x == 0) {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) s_deal[i] = words.w[i];
        }
    }
    __syncthreads();
    Words words;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) words.w[i] = __builtin_amdgcn_readfirstlane(s_deal[i]);
    return __builtin_bit_cast(ChunkDeal, words);
}

}  // namespace ann
