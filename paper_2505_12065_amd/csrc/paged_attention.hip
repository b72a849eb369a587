// Attention of one new token per request over a paged cache.
#include "launch.hpp"
#include "paged.hpp"

namespace ann {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / WAVE;

// One workgroup for a query head: a wave takes every fourth slot, its lanes share the row in pieces of eight elements, and
// keeps the running maximum, the sum and the weighted row.  The waves' are joined at the end.
template <class T>
__global__ __launch_bounds__(THREADS) void paged_attention_kernel(AttentionArgs a) {
    __shared__ float s_m[WAVES], s_l[WAVES], s_o[WAVES][ANN_HEAD_MAX];
    const int lane = threadIdx.x & (WAVE - 1), wave = threadIdx.x / WAVE;
    const int b = blockIdx.x / a.q_heads, hq = blockIdx.x % a.q_heads, h = hq / (a.q_heads / a.cache.heads);
    const int n = min(a.lengths[b], a.max_length), lo = a.window > 0 ? max(0, n - a.window) : 0;
    const int32_t *table = a.table + (int64_t)b * a.width;
    const int mask = (1 << a.cache.slots_log) - 1, d = a.cache.d;
    const bool mine = 8 * lane < d;
    float q[8] = {}, o[8] = {}, m = -INFINITY, l = 0.f;
    if (mine) {
        Eight<T> x;
        x.load(static_cast<const char *>(a.q) + b * a.q_row + hq * a.q_head + lane * 8 * T::bytes);
        x.get(q);
    }
    auto score = [&](int j, int64_t page) {
        float s = 0.f;
        if (mine) {
            Eight<T> x;
            float k[8];
            x.load(a.cache.k + page * a.cache.k_page + h * a.cache.k_head + (j & mask) * a.cache.k_slot + lane * 8 * T::bytes);
            x.get(k);
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(q[i], k[i], s);
        }
#pragma unroll
        for (int w = 1; w < WAVE; w *= 2) s += __shfl_xor(s, w);
        return s * a.scale;
    };
    for (int j = lo + wave; j < n; j += WAVES) {
        const int page = table[j >> a.cache.slots_log];
        if ((unsigned)page >= (unsigned)a.cache.pages) continue;
        const float s = score(j, page), top = fmaxf(m, s), base = top == -INFINITY ? 0.f : top;
        const float keep = expf(m - base), p = expf(s - base);
        m = top;
        l = l * keep + p;
        if (mine) {
            Eight<T> x;
            float v[8];
            x.load(a.cache.v + (int64_t)page * a.cache.v_page + h * a.cache.v_head + (j & mask) * a.cache.v_slot + lane * 8 * T::bytes);
            x.get(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = fmaf(p, v[i], o[i] * keep);
        }
    }
    if (lane == 0) { s_m[wave] = m; s_l[wave] = l; }
    if (mine) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s_o[wave][8 * lane + i] = o[i];
    }
    __syncthreads();
    float top = -INFINITY, total = 0.f;
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, s_m[w]);
    const float base = top == -INFINITY ? 0.f : top;
    for (int w = 0; w < WAVES; ++w) total += s_l[w] * expf(s_m[w] - base);
    const float lse = total == 0.f ? -INFINITY : base + logf(total);
    if (a.lse && threadIdx.x == 0) a.lse[(int64_t)b * a.q_heads + hq] = lse;
    if (wave == 0 && mine) {
        float r[8] = {};
        for (int w = 0; w < WAVES; ++w) {
            const float f = total == 0.f ? 0.f : expf(s_m[w] - base) / total;
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = fmaf(s_o[w][8 * lane + i], f, r[i]);
        }
        Eight<T> x;
        x.set(r);
        x.store(static_cast<char *>(a.out) + ((int64_t)b * a.q_heads + hq) * d * T::bytes + lane * 8 * T::bytes);
    }
}

// The weight of every slot, summed over the query heads of a cache head in their order: a wave takes a slot.
template <class T>
__global__ __launch_bounds__(THREADS) void paged_mass_kernel(AttentionArgs a) {
    const int lane = threadIdx.x & (WAVE - 1), wave = threadIdx.x / WAVE, G = a.q_heads / a.cache.heads;
    const int parts = (a.max_length + WAVES - 1) / WAVES, row = blockIdx.x / parts, b = row / a.cache.heads, h = row % a.cache.heads;
    const int n = min(a.lengths[b], a.max_length), lo = a.window > 0 ? max(0, n - a.window) : 0;
    const int j = blockIdx.x % parts * WAVES + wave;
    if (j < lo || j >= n) return;
    const int page = a.table[(int64_t)b * a.width + (j >> a.cache.slots_log)], d = a.cache.d;
    if ((unsigned)page >= (unsigned)a.cache.pages) return;
    const bool mine = 8 * lane < d;
    float k[8] = {}, sum = 0.f;
    Eight<T> x;
    if (mine) {
        x.load(a.cache.k + (int64_t)page * a.cache.k_page + h * a.cache.k_head +
               (j & ((1 << a.cache.slots_log) - 1)) * a.cache.k_slot + lane * 8 * T::bytes);
        x.get(k);
    }
    for (int g = 0; g < G; ++g) {
        float s = 0.f, q[8];
        if (mine) {
            x.load(static_cast<const char *>(a.q) + b * a.q_row + (h * G + g) * a.q_head + lane * 8 * T::bytes);
            x.get(q);
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(q[i], k[i], s);
        }
#pragma unroll
        for (int w = 1; w < WAVE; w *= 2) s += __shfl_xor(s, w);
        const float lse = a.lse[(int64_t)b * a.q_heads + h * G + g];
        sum += lse == -INFINITY ? 0.f : expf(s * a.scale - lse);
    }
    if (lane == 0) a.mass[((int64_t)b * a.cache.heads + h) * a.mass_slots + j] += sum;
}

template <class T>
hipError_t launch(const AttentionArgs &a, int B, hipStream_t stream) {
    hipLaunchKernelGGL((paged_attention_kernel<T>), dim3(B * a.q_heads), dim3(THREADS), 0, stream, a);
    if (a.mass)
        hipLaunchKernelGGL((paged_mass_kernel<T>), dim3((a.max_length + WAVES - 1) / WAVES * B * a.cache.heads), dim3(THREADS), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attention(int dtype, const AttentionArgs &a, int B, hipStream_t stream) {
    return dtype == ANN_F16 ? launch<F16>(a, B, stream) : dtype == ANN_BF16 ? launch<BF16>(a, B, stream) : launch<F32>(a, B, stream);
}

}  // namespace ann
