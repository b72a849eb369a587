// Attention of many rows over paged caches of BF16 elements.
#include "chunk_attention_kernel.hpp"

namespace ann {

hipError_t launch_chunk_attention_bf16(const ChunkArgs &a, const ChunkPlan &pl, hipStream_t stream) { return launch_chunk<BF16>(a, pl, stream); }

}  // namespace ann
