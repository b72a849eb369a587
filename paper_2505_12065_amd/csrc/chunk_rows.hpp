// Attention of many rows: which rows and slots a workgroup takes.
//
// A pass goes through tiles of `rows` rows of sequences of tokens: a request's new ones (CHUNK_NEW), the one of each request of a group (CHUNK_COMMON: the slots in common), or a
// request's one (CHUNK_OWN: its own slots).  A token has a row for each of the G query heads of a cache head.  Long ranges of slots are divided into parts.  How many tiles and slots there are is known on the
// device alone; up to 64 sequences, a lane each, every workgroup works out for itself how the whole is dealt: parts as long as fill the card, longest sequences first.
#pragma once

#include "launch.hpp"
#include "packed.hpp"

namespace ann {

struct ChunkSpan { int lo, hi; };                         // slots lo .. hi - 1
// Parts begin with multiples of 32 slots, so that 16 rows from a multiple of 16 on are loaded together.
__device__ __forceinline__ int chunk_begin(ChunkSpan range) { return min(range.lo, range.hi) & ~31; }
__device__ __forceinline__ int chunk_slots_of(ChunkSpan range) { return range.hi - chunk_begin(range); }
__device__ __forceinline__ int chunk_parts(int slots, int chunk) { return slots > 0 ? (slots - 1) / chunk + 1 : 1; }     // (the first part of nothing says so)

__device__ __forceinline__ int chunk_length(const ChunkArgs &a, int request) { return max(a.lengths[request], 0); }

// The group of request t, or -1.  By whole waves, whose lanes may ask for different requests.
__device__ __forceinline__ int chunk_group(const ChunkArgs &a, int t) {
    int n = 0;                                            // starts up to t
    if (a.groups < WAVE) {
        const int lane = threadIdx.x & (WAVE - 1), start = lane <= a.groups ? packed_start(a.group_starts, lane, a.tokens) : INT_MAX;
        for (int g = 0; g <= a.groups; ++g) n += __builtin_amdgcn_readlane(start, g) <= t;
    } else {
        for (int left = a.groups + 1; left > 0;) {        // (halves)
            const int half = left / 2;
            if (packed_start(a.group_starts, n + half, a.tokens) <= t) { n += half + 1; left -= half + 1; }
            else left = half;
        }
    }
    return n <= a.groups ? n - 1 : -1;
}
__device__ __forceinline__ int chunk_common(const ChunkArgs &a, int g) { return g < 0 ? 0 : min(max(a.shared[g], 0), a.max_shared); }

struct ChunkSequence { int token0, tokens, request; };    // request: whose pages are read
__device__ __forceinline__ int chunk_sequences(const ChunkArgs &a, int mode) { return mode == CHUNK_NEW ? a.requests : mode == CHUNK_COMMON ? a.groups : a.tokens; }
__device__ __forceinline__ ChunkSequence chunk_sequence(const ChunkArgs &a, int mode, int i) {
    if (mode == CHUNK_OWN) return {i, 1, i};
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
// ... that tokens t0 to t1 of sequence i, of a request of `length` slots, attend to, all of them together.  By whole waves.
__device__ __forceinline__ ChunkSpan chunk_range(const ChunkArgs &a, int mode, int i, const ChunkSequence &q, int length, int t0, int t1) {
    if (mode == CHUNK_NEW) {
        const int first = length - (q.tokens - t0), last = length - (q.tokens - t1);
        return {a.window > 0 ? max(first + 1 - a.window, 0) : 0, min(max(last + 1, 0), a.max_length)};
    }
    if (mode == CHUNK_COMMON) return {0, chunk_common(a, i)};
    const int n = min(length, a.max_length), common = min(n, chunk_common(a, chunk_group(a, q.token0)));
    return {common, common + min(n - common, a.max_own)};
}

__device__ __forceinline__ int wave_sum_int(int x) {
#pragma unroll
    for (int i = 1; i < WAVE; i *= 2) x += __shfl_xor(x, i);
    return x;
}

// What lane i knows of sequence i, and slots of a part.
struct ChunkLane { int tiles, slots, chunk; };
__device__ __forceinline__ ChunkLane chunk_lane(const ChunkArgs &a, const ChunkPass &p, int n, int G) {
    const int lane = threadIdx.x & (WAVE - 1);
    ChunkLane l{0, 0, INT_MAX};
    const int i = min(lane, n - 1);
    const ChunkSequence q = chunk_sequence(a, p.mode, i);
    const int64_t rows = (int64_t)q.tokens * G;
    if (lane < n) l.tiles = (int)((rows + p.rows - 1) / p.rows);
    // (the last tile has most, but for what a window leaves it)
    const int t0 = (int)(max(l.tiles - 1, 0) * (int64_t)p.rows / G), t1 = max(q.tokens - 1, 0);
    const ChunkSpan range = chunk_range(a, p.mode, i, q, chunk_length(a, q.request), t0, t1);
    if (l.tiles > 0) l.slots = chunk_slots_of(range);
    if (l.tiles > 0 && p.mode == CHUNK_NEW && a.window > 0) l.slots = (int)max((int64_t)l.slots, min((int64_t)range.hi, (int64_t)a.window + p.rows + 32));
    if (p.most_parts == 1) return l;
    const int tiles = wave_sum_int(l.tiles);
    float slots = (float)l.tiles * (float)l.slots;
    int most = l.slots;
#pragma unroll
    for (int k = 1; k < WAVE; k *= 2) {
        slots += __shfl_xor(slots, k);
        most = max(most, __shfl_xor(most, k));
    }
    // tiles + slots / chunk workgroups at most: once as many as fill the card, twice if tiles alone make up much of it
    const int room = (4 * (int64_t)tiles > p.fill ? 2 : 1) * p.fill - tiles;
    if (room <= 0) return l;
    const int chunk = max(max((int)min(ceilf(slots / room), 1e9f), p.least), (most - 1) / p.most_parts + 1);
    l.chunk = (chunk + 63) & ~63;
    return l;
}

// What a workgroup does: slots first .. end - 1 of the tile that begins with row r0 of a sequence, of whose range they are part `part`; count 0: nothing.
struct ChunkDeal {
    ChunkSequence q;
    int length;               // of q.request, at least 0
    int r0, count, part, parts;
    bool alone;               // nothing is to be joined with it
    int grouped;              // CHUNK_OWN: the request is in a group
    ChunkSpan range;          // of the tile's rows, all together
    int first, end;
};
__device__ __forceinline__ ChunkDeal chunk_deal(const ChunkArgs &a, const ChunkPass &p, int item, int G) {
    const int n = chunk_sequences(a, p.mode), lane = threadIdx.x & (WAVE - 1);
    ChunkDeal d{};
    int i, chunk;
    int64_t tile;
    if (n <= WAVE) {
        const ChunkLane l = chunk_lane(a, p, n, G);
        const int items = l.tiles * chunk_parts(l.slots, l.chunk);
        int before = 0;                                   // items of longer sequences
        for (int k = 0; k < n; ++k) {
            const int other = __builtin_amdgcn_readlane(l.slots, k);
            before += other > l.slots || (other == l.slots && k < lane) ? __builtin_amdgcn_readlane(items, k) : 0;
        }
        const uint64_t mine = __ballot(item >= before && item < before + items);
        if (mine == 0) return d;
        i = __ffsll((unsigned long long)mine) - 1;
        const int local = item - __builtin_amdgcn_readlane(before, i), tiles = __builtin_amdgcn_readlane(l.tiles, i);
        d.part = local / tiles;
        tile = tiles - 1 - local % tiles;
        chunk = l.chunk;
    } else {
        // A sequence of m tokens has at most as many tiles as there are numbers from start G / rows + i up to the next one's.
        const int id = p.tiles - 1 - item % p.tiles;
        d.part = item / p.tiles;
        chunk = p.chunk;
        if (p.mode == CHUNK_OWN) {
            const int per = (G + p.rows - 1) / p.rows;
            i = id / per;
            tile = id % per;
            if (i >= n) return d;
        } else {
            const int32_t *starts = p.mode == CHUNK_NEW ? a.starts : a.group_starts;
            auto first = [&](int k) { return (int)((int64_t)packed_start(starts, k, a.tokens) * G / p.rows) + k; };
            i = count_up_to(first, n + 1, id) - 1;
            if (i < 0 || i >= n) return d;
            tile = id - first(i);
        }
    }
    d.q = chunk_sequence(a, p.mode, i);
    d.length = chunk_length(a, d.q.request);
    d.r0 = (int)(tile * p.rows);
    const int count = (int)max((int64_t)0, min((int64_t)p.rows, (int64_t)d.q.tokens * G - tile * p.rows));
    if (count == 0) return d;
    if (p.mode == CHUNK_OWN) d.grouped = chunk_group(a, i) >= 0;
    d.range = chunk_range(a, p.mode, i, d.q, d.length, d.r0 / G, (d.r0 + count - 1) / G);
    const int slots = chunk_slots_of(d.range);
    d.parts = chunk_parts(slots, chunk);
    if (d.part >= d.parts) return d;
    d.count = count;
    d.alone = p.mode == CHUNK_NEW && d.parts == 1;
    d.first = chunk_begin(d.range) + d.part * chunk;
    d.end = d.range.hi - d.first < chunk ? d.range.hi : d.first + chunk;
    return d;
}

}  // namespace ann
