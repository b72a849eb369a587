// Attention of one new token per request over a paged cache of BF16 elements.
#include "paged_attention_kernel.hpp"

namespace ann {

hipError_t launch_paged_attention_bf16(const AttentionArgs &a, bool once, hipStream_t stream) { return launch_attention<BF16>(a, once, stream); }

}  // namespace ann
