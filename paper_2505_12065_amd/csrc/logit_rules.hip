// Penalties for repeated tokens, biases and grammar masks on logits.
#include "launch.hpp"
#include "paged.hpp"

namespace ann {

namespace {

constexpr int THREADS = 256, CHUNK = 4096;
constexpr uint32_t SEEN = 1u << 31;                       // beside the count

template <class T> struct Scalar;
template <> struct Scalar<F16> { typedef _Float16 type; };
template <> struct Scalar<BF16> { typedef __bf16 type; };
template <> struct Scalar<F32> { typedef float type; };

// A workgroup takes CHUNK tokens of the vocabulary of one request: it counts them in the request's history, finds the last
// bias of each, and goes through its logits once.
template <class T>
__global__ __launch_bounds__(THREADS) void logit_rules_kernel(RulesArgs a) {
    typedef typename Scalar<T>::type E;
    __shared__ uint32_t count[CHUNK];
    __shared__ int bias[CHUNK];
    const int parts = (a.V + CHUNK - 1) / CHUNK, b = blockIdx.x / parts, v0 = blockIdx.x % parts * CHUNK, m = min(CHUNK, a.V - v0);
    for (int i = threadIdx.x; i < m; i += THREADS) { count[i] = 0; bias[i] = -1; }
    __syncthreads();
    const int n = max(0, min(a.lengths[b], a.T)), prompt = max(0, a.prompt[b]);
    const int32_t *tokens = a.tokens + (int64_t)b * a.T;
    for (int t = threadIdx.x; t < n; t += THREADS) {
        const uint32_t at = (uint32_t)(tokens[t] - v0);
        if (tokens[t] < 0 || at >= (uint32_t)m) continue;
        if (t < prompt) atomicOr(&count[at], SEEN);
        else atomicAdd(&count[at], 1u);
    }
    for (int i = threadIdx.x; i < a.K; i += THREADS) {
        const int token = a.bias_tokens[(int64_t)b * a.K + i];
        if (token >= v0 && token - v0 < m) atomicMax(&bias[token - v0], i);
    }
    __syncthreads();
    const float repetition = a.repetition[b], presence = a.presence[b], frequency = a.frequency[b];
    const int mask_row = a.masks ? a.mask_rows[b] : -1;
    const uint32_t *mask = (unsigned)mask_row < (unsigned)a.n_masks ? a.masks + (int64_t)mask_row * ((a.V + 31) / 32) : nullptr;
    const E *in = static_cast<const E *>(a.logits) + b * a.row + v0;
    E *out = static_cast<E *>(a.out) + b * a.out_row + v0;
    for (int i = threadIdx.x; i < m; i += THREADS) {
        float x = (float)in[i];
        if (const uint32_t c = count[i]) {
            x = x > 0.f ? x / repetition : x * repetition;
            if (c & ~SEEN) x = x - frequency * (float)(c & ~SEEN) - presence;
        }
        if (bias[i] >= 0) x += a.bias_values[(int64_t)b * a.K + bias[i]];
        if (mask && !((mask[(v0 + i) / 32] >> ((v0 + i) & 31)) & 1)) x = -INFINITY;
        out[i] = (E)x;
    }
}

template <class T>
hipError_t launch(const RulesArgs &a, int B, hipStream_t stream) {
    hipLaunchKernelGGL((logit_rules_kernel<T>), dim3((a.V + CHUNK - 1) / CHUNK * B), dim3(THREADS), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_logit_rules(int dtype, const RulesArgs &a, int B, hipStream_t stream) {
    return dtype == ANN_F16 ? launch<F16>(a, B, stream) : dtype == ANN_BF16 ? launch<BF16>(a, B, stream) : launch<F32>(a, B, stream);
}

}  // namespace ann
