// Cutting a paged cache to the slots with the most accumulated attention weight: the choice, a workgroup to a cache head, then the copy of the rows.
//
// The copy is bound by its bytes, the choice by one compute unit's instructions and LDS.  32 requests of up to 16000 slots, 4 cache heads of 128, bf16, cut to 4000: 13.6 us for the choice
// and 102 for 0.50 GB of rows (4.9 TB/s, what any copy reaches); 2 requests of 6000, 8 heads, cut to 1500: 9.2 and 5.7.
#include "launch.hpp"
#include "paged.hpp"

namespace ann {

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / WAVE, COPY = 256;
constexpr int DIGIT = 11, BINS = 1 << DIGIT;              // of a rank, from the highest: 11, 11 and 10 bits
constexpr uint32_t KEEP = 0xffffffffu;                    // rank of a slot that is kept whatever its mass

// Unsigned order = order of the numbers; -0 is 0, a NaN comes before everything.
__device__ __forceinline__ uint32_t rank_of(float x) {
    if (x != x) return 0;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// The sum of x over the lanes up to this one.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
    int y = (int)x;
    y += __builtin_amdgcn_update_dpp(0, y, 0x111, 0xf, 0xf, false);          // from 1, 2, 4, 8 lanes before, in rows of 16
    y += __builtin_amdgcn_update_dpp(0, y, 0x112, 0xf, 0xf, false);
    y += __builtin_amdgcn_update_dpp(0, y, 0x114, 0xf, 0xf, false);
    y += __builtin_amdgcn_update_dpp(0, y, 0x118, 0xf, 0xf, false);
    y += __builtin_amdgcn_update_dpp(0, y, 0x142, 0xa, 0xf, false);          // the last of a row to the next one
    y += __builtin_amdgcn_update_dpp(0, y, 0x143, 0xc, 0xf, false);          // lane 31 to the upper half
    return (uint32_t)y;
}

// One workgroup for a cache head of a request.  The rank of the last slot that is kept is found digit by digit by counting in LDS: thread
// t owns the bins BINS / THREADS t on, from the top down.  Then a slot is kept if its rank is higher, or the same and not too many of those
// lie before it; where it goes is the number of kept ones before it, which the slots of a wave (KR times 64 neighbours, THREADS apart) learn from a
// ballot and the waves from a scan over all of their ballots.  HELD: the ranks stay in registers, a thread's KR slots are all that it has;
// else they are read again for every digit, and the last step goes over the row in tiles of KR THREADS.
template <int KR, bool HELD>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(EvictArgs a) {
    constexpr int EACH = BINS / THREADS, PER_LANE = KR * WAVES / WAVE;
    static_assert(PER_LANE >= 1 && 2 * KR * WAVES <= BINS && KR <= WAVE, "ballots of a tile, scanned by a wave");
    // (four counts of a bin, a quarter of the lanes to each: masses that are all the same would have 64 lanes wait for each other)
    __shared__ u4 count[BINS];
    __shared__ uint32_t of_wave[3][WAVES], s_digit[3], s_need[3];
    __shared__ uint2 s_all;
    const int64_t row = blockIdx.x;
    const int b = blockIdx.x / a.cache.heads, h = blockIdx.x % a.cache.heads, tid = threadIdx.x;
    const int lane = tid & (WAVE - 1), wave = tid / WAVE;
    const int n = max(0, min(a.lengths[b], a.most)), left = min(n, a.budget);
    const float *mass = a.mass + row * a.mass_slots;
    int32_t *kept = a.kept + row * a.budget;
    float *new_mass = a.new_mass + row * a.new_mass_slots;
    if (h == 0 && tid == 0) a.new_lengths[b] = left;
    for (int64_t i = left + tid; i < a.new_mass_slots; i += THREADS) new_mass[i] = 0.f;
    for (int i = left + tid; i < a.budget; i += THREADS) kept[i] = -1;
    if (n <= a.budget) {
        for (int i = tid; i < n; i += THREADS) { kept[i] = i; new_mass[i] = mass[i]; }
        return;
    }
    const int lo = a.first, hi = n - a.recent;            // the slots that are chosen from
    constexpr bool VALUES = KR <= 16;                     // (registers: else the kept ones' are read again)
    float value[VALUES ? KR : 1];
    uint32_t rank[KR];
    auto load = [&](int i0) {                             // slots i0, i0 + THREADS, ...
        constexpr int AT_ONCE = KR < 16 ? KR : 16;
#pragma unroll
        for (int k0 = 0; k0 < KR; k0 += AT_ONCE) {
            float x[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) x[k] = i0 + (k0 + k) * THREADS < n ? mass[i0 + (k0 + k) * THREADS] : 0.f;
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int i = i0 + (k0 + k) * THREADS;
                // (one that is not there comes after all that are, like a NaN behind them)
                rank[k0 + k] = i >= n ? 0 : i < lo || i >= hi ? KEEP : rank_of(x[k]);
                if (VALUES) value[VALUES ? k0 + k : 0] = x[k];
            }
        }
    };
    if (HELD) load(tid);
    const int tiles = HELD ? 1 : (n + THREADS * KR - 1) / (THREADS * KR);
#pragma unroll
    for (int j = 0; j < EACH; ++j) count[tid + j * THREADS] = zero_chunk();
    __syncthreads();
    uint32_t prefix = 0, need = a.budget;                 // of the ranks that start with `prefix` so many are kept
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass < 2 ? DIGIT : 32 - 2 * DIGIT, shift = pass < 2 ? 32 - (pass + 1) * DIGIT : 0;
        for (int tile = 0; tile < tiles; ++tile) {
            if (!HELD) load(tile * THREADS * KR + tid);
#pragma unroll
            for (int k = 0; k < KR; ++k) {
                if (pass > 0 && (rank[k] ^ prefix) >> (shift + bits) != 0) continue;
                const uint32_t digit = (rank[k] >> shift) & ((1u << bits) - 1);
                atomicAdd(reinterpret_cast<uint32_t *>(count) + 4 * digit + (lane & 3), 1u);
            }
        }
        __syncthreads();
        uint32_t mine = 0, c[EACH];
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            u4 &bin = count[BINS - 1 - (tid * EACH + j)];
            mine += c[j] = (bin[0] + bin[1]) + (bin[2] + bin[3]);
            bin = zero_chunk();
        }
        const uint32_t up_to = wave_scan(mine);
        if (lane == WAVE - 1) of_wave[pass][wave] = up_to;
        __syncthreads();
        uint32_t above = up_to - mine;                    // slots in the bins above this thread's
#pragma unroll
        for (int w = 0; w < WAVES; ++w) above += w < wave ? of_wave[pass][w] : 0;
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            if (above < need && above + c[j] >= need) {
                s_digit[pass] = BINS - 1 - (tid * EACH + j);
                s_need[pass] = need - above;
            }
            above += c[j];
        }
        __syncthreads();
        prefix |= s_digit[pass] << shift;
        need = s_need[pass];
    }
    // all of a higher rank are kept, and the first `need` of rank `prefix`
    uint32_t *higher = reinterpret_cast<uint32_t *>(count), *equal = higher + KR * WAVES;   // of the ballots: how many; then how many before
    uint32_t more = 0, as_much = 0;                       // such slots in the tiles before
    for (int tile = 0; tile < tiles; ++tile) {
        const int i0 = tile * THREADS * KR + tid;
        if (!HELD) load(i0);
        uint32_t m_of = 0, e_of = 0;                      // kept for sure, and of rank `prefix`; lane k: in ballot k
#pragma unroll
        for (int k = 0; k < KR; ++k) {
            const uint64_t m = __ballot(rank[k] > prefix), e = __ballot(rank[k] == prefix);
            if (lane == k) {
                m_of = __popcll(m);
                e_of = __popcll(e);
            }
        }
        if (lane < KR) {
            higher[lane * WAVES + wave] = m_of;
            equal[lane * WAVES + wave] = e_of;
        }
        __syncthreads();
        if (wave < 2) {                                   // a wave for each of the two
            uint32_t *x = wave == 0 ? higher : equal, v[PER_LANE], sum = 0;
#pragma unroll
            for (int j = 0; j < PER_LANE; ++j) sum += v[j] = x[lane * PER_LANE + j];
            uint32_t up_to = wave_scan(sum), run = up_to - sum;
#pragma unroll
            for (int j = 0; j < PER_LANE; ++j) {
                x[lane * PER_LANE + j] = run;
                run += v[j];
            }
            if (lane == WAVE - 1) (wave == 0 ? s_all.x : s_all.y) = up_to;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < KR; ++k) {
            const uint64_t mb = __ballot(rank[k] > prefix), eb = __ballot(rank[k] == prefix);   // (those among the lanes before)
            const uint32_t m = more + higher[k * WAVES + wave] + __builtin_amdgcn_mbcnt_hi((uint32_t)(mb >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mb, 0));
            const uint32_t e = as_much + equal[k * WAVES + wave] + __builtin_amdgcn_mbcnt_hi((uint32_t)(eb >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)eb, 0));
            if (rank[k] > prefix || (rank[k] == prefix && e < need)) {
                const int i = i0 + k * THREADS;
                kept[m + min(e, need)] = i;
                new_mass[m + min(e, need)] = VALUES ? value[VALUES ? k : 0] : mass[i];
            }
        }
        more += s_all.x;
        as_much += s_all.y;
        if (!HELD) __syncthreads();
    }
}

// LPR lanes for a row of 16-byte chunks.
template <int LPR>
__global__ __launch_bounds__(COPY) void evict_copy_kernel(EvictArgs a, int chunks, int parts) {
    const int lane = threadIdx.x % LPR, i = blockIdx.x % parts * (COPY / LPR) + threadIdx.x / LPR;
    const int64_t row = blockIdx.x / parts;
    const int b = (int)row / a.cache.heads, h = (int)row % a.cache.heads;
    if (i >= a.budget || lane >= chunks) return;
    const int from = a.kept[row * a.budget + i], to = a.new_table[(int64_t)b * a.new_width + (i >> a.cache.slots_log)];
    if (from < 0 || (unsigned)to >= (unsigned)a.cache.pages) return;
    const int source = a.table[(int64_t)b * a.width + (from >> a.cache.slots_log)], mask = (1 << a.cache.slots_log) - 1;
    u4 k = zero_chunk(), v = zero_chunk();
    if ((unsigned)source < (unsigned)a.cache.pages) {
        k = load_chunk(a.cache.k + (int64_t)source * a.cache.k_page + h * a.cache.k_head + (from & mask) * a.cache.k_slot + lane * 16);
        v = load_chunk(a.cache.v + (int64_t)source * a.cache.v_page + h * a.cache.v_head + (from & mask) * a.cache.v_slot + lane * 16);
    }
    *reinterpret_cast<u4 *>(a.cache.k + (int64_t)to * a.cache.k_page + h * a.cache.k_head + (i & mask) * a.cache.k_slot + lane * 16) = k;
    *reinterpret_cast<u4 *>(a.cache.v + (int64_t)to * a.cache.v_page + h * a.cache.v_head + (i & mask) * a.cache.v_slot + lane * 16) = v;
}

template <int LPR>
hipError_t copy(const EvictArgs &a, int rows, int chunks, hipStream_t stream) {
    constexpr int PER = COPY / LPR;
    const int parts = (a.budget + PER - 1) / PER;
    hipLaunchKernelGGL((evict_copy_kernel<LPR>), dim3(rows * parts), dim3(COPY), 0, stream, a, chunks, parts);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_evict(int dtype, const EvictArgs &a, int B, hipStream_t stream) {
    const int rows = B * a.cache.heads, chunks = a.cache.d * elem_bytes(dtype) / 16;
    // A row has at most a.most slots.  As few ranks a thread as hold it (a choice among 6000 with 8: 9.2 us; among 16000 with 16: 13.6; among
    // 32000 with 32: 20.5, or 27 if they are read again for every digit), longer rows are read again (60000: 53; 64 ranks do not fit a thread's registers: 61; 130000: 102).
    if (a.most <= 4 * THREADS) hipLaunchKernelGGL((evict_select_kernel<4, true>), dim3(rows), dim3(THREADS), 0, stream, a);
    else if (a.most <= 8 * THREADS) hipLaunchKernelGGL((evict_select_kernel<8, true>), dim3(rows), dim3(THREADS), 0, stream, a);
    else if (a.most <= 16 * THREADS) hipLaunchKernelGGL((evict_select_kernel<16, true>), dim3(rows), dim3(THREADS), 0, stream, a);
    else if (a.most <= 32 * THREADS) hipLaunchKernelGGL((evict_select_kernel<32, true>), dim3(rows), dim3(THREADS), 0, stream, a);
    else hipLaunchKernelGGL((evict_select_kernel<16, false>), dim3(rows), dim3(THREADS), 0, stream, a);
    if (hipError_t e = hipGetLastError()) return e;
    return chunks <= 8 ? copy<8>(a, rows, chunks, stream) : chunks <= 16 ? copy<16>(a, rows, chunks, stream)
           : chunks <= 32 ? copy<32>(a, rows, chunks, stream) : copy<64>(a, rows, chunks, stream);
}

}  // namespace ann
