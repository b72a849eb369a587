// Cutting a paged cache to the slots with the most accumulated attention weight.
#include "launch.hpp"
#include "paged.hpp"

namespace ann {

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / WAVE, COPY = 256;

// Unsigned order = order of the numbers; -0 is 0, a NaN comes before everything.
__device__ __forceinline__ uint32_t rank_of(float x) {
    if (x != x) return 0;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// The sum of x over the threads before this one, and over all.
__device__ __forceinline__ uint64_t scan_before(uint64_t x, uint64_t *of_wave, uint64_t &all) {
    const int lane = threadIdx.x & (WAVE - 1), wave = threadIdx.x / WAVE;
    uint64_t y = x;
#pragma unroll
    for (int s = 1; s < WAVE; s *= 2) {
        const uint64_t o = __shfl_up((unsigned long long)y, s);
        if (lane >= s) y += o;
    }
    if (lane == WAVE - 1) of_wave[wave] = y;
    __syncthreads();
    uint64_t before = y - x;
    all = 0;
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += of_wave[w];
        all += of_wave[w];
    }
    __syncthreads();
    return before;
}

// One workgroup for a cache head of a request.  The rank of the last slot that is kept is found digit by digit, 8 bits at a
// time from the highest, by counting; then every thread takes a run of slots and learns from a scan where its kept ones go.
__global__ __launch_bounds__(THREADS) void evict_select_kernel(EvictArgs a) {
    __shared__ uint32_t count[256];
    __shared__ uint64_t of_wave[WAVES];
    __shared__ uint32_t s_digit, s_need;
    const int64_t row = blockIdx.x;
    const int b = blockIdx.x / a.cache.heads, h = blockIdx.x % a.cache.heads;
    const int n = max(0, min(a.lengths[b], a.most)), left = min(n, a.budget);
    const float *mass = a.mass + row * a.mass_slots;
    int32_t *kept = a.kept + row * a.budget;
    float *new_mass = a.new_mass + row * a.new_mass_slots;
    if (h == 0 && threadIdx.x == 0) a.new_lengths[b] = left;
    for (int64_t i = left + threadIdx.x; i < a.new_mass_slots; i += THREADS) new_mass[i] = 0.f;
    for (int i = left + threadIdx.x; i < a.budget; i += THREADS) kept[i] = -1;
    if (n <= a.budget) {
        for (int i = threadIdx.x; i < n; i += THREADS) { kept[i] = i; new_mass[i] = mass[i]; }
        return;
    }
    const int lo = a.first, hi = n - a.recent;            // the slots that have to be chosen from
    uint32_t prefix = 0, need = a.budget - a.first - a.recent;
    if (need > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (threadIdx.x < 256) count[threadIdx.x] = 0;
            __syncthreads();
            for (int i = lo + threadIdx.x; i < hi; i += THREADS) {
                const uint32_t r = rank_of(mass[i]);
                if (shift == 24 || (r >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&count[(r >> shift) & 255], 1u);
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                int digit = 255;
                while (digit > 0 && count[digit] < need) need -= count[digit--];
                s_digit = digit;
                s_need = need;
            }
            __syncthreads();
            prefix |= s_digit << shift;
            need = s_need;
            __syncthreads();
        }
    }
    // need = slots of rank `prefix` that are kept, the lowest ones (none at all if nothing was to be chosen)
    const bool some = a.budget - a.first - a.recent > 0;
    const int each = (n + THREADS - 1) / THREADS, i0 = threadIdx.x * each, i1 = min(n, i0 + each);
    uint64_t mine = 0, all;                               // kept for sure, and of rank `prefix` (upper half)
    for (int i = i0; i < i1; ++i) {
        if (i < lo || i >= hi) { mine += 1; continue; }
        const uint32_t r = rank_of(mass[i]);
        mine += some && r > prefix ? 1 : some && r == prefix ? (1ull << 32) : 0;
    }
    const uint64_t before = scan_before(mine, of_wave, all);
    uint32_t equal = (uint32_t)(before >> 32), at = (uint32_t)before + min(equal, need);
    for (int i = i0; i < i1; ++i) {
        bool keep = i < lo || i >= hi;
        if (!keep && some) {
            const uint32_t r = rank_of(mass[i]);
            keep = r > prefix || (r == prefix && equal < need);
            equal += r == prefix;
        }
        if (keep) { kept[at] = i; new_mass[at] = mass[i]; ++at; }
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
    hipLaunchKernelGGL(evict_select_kernel, dim3(rows), dim3(THREADS), 0, stream, a);
    if (hipError_t e = hipGetLastError()) return e;
    return chunks <= 8 ? copy<8>(a, rows, chunks, stream) : chunks <= 16 ? copy<16>(a, rows, chunks, stream)
           : chunks <= 32 ? copy<32>(a, rows, chunks, stream) : copy<64>(a, rows, chunks, stream);
}

}  // namespace ann
