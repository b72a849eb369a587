// Attention of many rows over paged caches of F16 elements.
#include "chunk_attention_kernel.hpp"

namespace ann {

hipError_t launch_chunk_attention_f16(const ChunkArgs &a, const ChunkPlan &pl, hipStream_t stream) { return launch_chunk<F16>(a, pl, stream); }

}  // namespace ann
