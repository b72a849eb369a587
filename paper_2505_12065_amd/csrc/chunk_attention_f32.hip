// Attention of many rows over paged caches of F32 elements.
#include "chunk_attention_kernel.hpp"

namespace ann {

hipError_t launch_chunk_attention_f32(const ChunkArgs &a, const ChunkPlan &pl, hipStream_t stream) { return launch_chunk<F32>(a, pl, stream); }

}  // namespace ann
