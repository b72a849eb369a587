// Attention of one new token per request over a paged cache of F32 elements.
#include "paged_attention_kernel.hpp"

namespace ann {

hipError_t launch_paged_attention_f32(const AttentionArgs &a, bool once, hipStream_t stream) { return launch_attention<F32>(a, once, stream); }

}  // namespace ann
