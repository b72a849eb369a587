// Cutting a paged cache to the slots with the most accumulated attention weight.
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

// The sum of x over the threads before this one, and over all.
__device__ __forceinline__ uint32_t scan_before(uint32_t x, uint32_t *of_wave, uint32_t &all) {
    const int lane = threadIdx.x & (WAVE - 1), wave = threadIdx.x / WAVE;
    uint32_t y = x;
#pragma unroll
    for (int s = 1; s < WAVE; s *= 2) {
        const uint32_t o = __shfl_up(y, s);
        if (lane >= s) y += o;
    }
    if (lane == WAVE - 1) of_wave[wave] = y;
    __syncthreads();
    uint32_t before = y - x;
    all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const uint32_t o = of_wave[w];
        if (w < wave) before += o;
        all += o;
    }
    __syncthreads();
    return before;
}

typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));

// One workgroup for a cache head of a request.  The rank of the last slot that is kept is found digit by digit by counting in LDS, then every
// thread learns from a scan where the kept ones of its KR neighbouring slots go.  HELD: the ranks stay in registers, a thread's slots are
// all that it has; else they are read again for every digit, and the last step goes over the row in tiles.
template <int KR, bool HELD>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(EvictArgs a) {
    __shared__ uint32_t count[BINS], of_wave[WAVES], s_digit, s_need;
    const int64_t row = blockIdx.x;
    const int b = blockIdx.x / a.cache.heads, h = blockIdx.x % a.cache.heads, tid = threadIdx.x;
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
    float value[KR];
    uint32_t rank[KR];
    auto load = [&](int i0) {
#pragma unroll
        for (int k = 0; k < KR; k += 4) {
            if (i0 + k + 4 <= n) {
                const f4_any x = *reinterpret_cast<const f4_any *>(mass + i0 + k);
#pragma unroll
                for (int j = 0; j < 4; ++j) value[k + j] = x[j];
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) value[k + j] = i0 + k + j < n ? mass[i0 + k + j] : 0.f;
            }
        }
#pragma unroll
        for (int k = 0; k < KR; ++k) rank[k] = i0 + k < lo || i0 + k >= hi ? KEEP : rank_of(value[k]);
    };
    if (HELD) load(tid * KR);
    const int tiles = HELD ? 1 : (n + THREADS * KR - 1) / (THREADS * KR);
    uint32_t prefix = 0, need = a.budget;                 // of the ranks that start with `prefix` so many are kept
    for (int shift = 32 - DIGIT; ; shift = max(0, shift - DIGIT)) {
        const int bits = shift > 0 ? DIGIT : 32 - 2 * DIGIT;
        for (int i = tid; i < BINS; i += THREADS) count[i] = 0;
        __syncthreads();
        for (int tile = 0; tile < tiles; ++tile) {
            const int i0 = (tile * THREADS + tid) * KR;
            if (!HELD) load(i0);
#pragma unroll
            for (int k = 0; k < KR; ++k) {
                const bool in = i0 + k < n && (shift == 32 - DIGIT || rank[k] >> (shift + bits) == prefix >> (shift + bits));
                if (!in) continue;
                const uint32_t digit = (rank[k] >> shift) & ((1u << bits) - 1);
                // (masses that are all the same would have the lanes wait for each other)
                const uint32_t one = __builtin_amdgcn_readfirstlane(digit);
                const uint64_t here = __ballot(true), same = __ballot(digit == one);
                if (here == same) {
                    if ((tid & (WAVE - 1)) == (int)__ffsll((unsigned long long)here) - 1) atomicAdd(&count[digit], (uint32_t)__popcll(here));
                } else {
                    atomicAdd(&count[digit], 1u);
                }
            }
        }
        __syncthreads();
        // thread t takes the bins from the top down: how many lie above its own
        constexpr int EACH = BINS / THREADS;
        uint32_t mine = 0, c[EACH], all;
#pragma unroll
        for (int j = 0; j < EACH; ++j) mine += c[j] = count[BINS - 1 - (tid * EACH + j)];
        uint32_t above = scan_before(mine, of_wave, all);
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            if (above < need && above + c[j] >= need) {
                s_digit = BINS - 1 - (tid * EACH + j);
                s_need = need - above;
            }
            above += c[j];
        }
        __syncthreads();
        prefix |= s_digit << shift;
        need = s_need;
        if (shift == 0) break;
        __syncthreads();
    }
    // all of a higher rank are kept, and the first `need` of rank `prefix`
    uint32_t more = 0, equal = 0;                         // such slots in the tiles before
    for (int tile = 0; tile < tiles; ++tile) {
        const int i0 = (tile * THREADS + tid) * KR;
        if (!HELD) load(i0);
        uint32_t m = 0, e = 0, all_m, all_e;
#pragma unroll
        for (int k = 0; k < KR; ++k) {
            m += i0 + k < n && rank[k] > prefix;
            e += i0 + k < n && rank[k] == prefix;
        }
        const uint32_t m0 = more + scan_before(m, of_wave, all_m);
        uint32_t e0 = equal + scan_before(e, of_wave, all_e), at = m0 + min(e0, need);
#pragma unroll
        for (int k = 0; k < KR; ++k) {
            const bool there = i0 + k < n, same = rank[k] == prefix;
            if (there && (rank[k] > prefix || (same && e0 < need))) {
                kept[at] = i0 + k;
                new_mass[at] = value[k];
                ++at;
            }
            e0 += there && same;
        }
        more += all_m;
        equal += all_e;
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
    // (a row has at most a.most slots)
    if (a.most <= 4 * THREADS) hipLaunchKernelGGL((evict_select_kernel<4, true>), dim3(rows), dim3(THREADS), 0, stream, a);
    else if (a.most <= 8 * THREADS) hipLaunchKernelGGL((evict_select_kernel<8, true>), dim3(rows), dim3(THREADS), 0, stream, a);
    else if (a.most <= 16 * THREADS) hipLaunchKernelGGL((evict_select_kernel<16, true>), dim3(rows), dim3(THREADS), 0, stream, a);
    else hipLaunchKernelGGL((evict_select_kernel<4, false>), dim3(rows), dim3(THREADS), 0, stream, a);
    if (hipError_t e = hipGetLastError()) return e;
    return chunks <= 8 ? copy<8>(a, rows, chunks, stream) : chunks <= 16 ? copy<16>(a, rows, chunks, stream)
           : chunks <= 32 ? copy<32>(a, rows, chunks, stream) : copy<64>(a, rows, chunks, stream);
}

}  // namespace ann
