// The chunk attention kernel for 2-bit codes.
#include "iq_chunk_kernel.cuh"

namespace iq {
cudaError_t launch_chunk_b2(const ChunkParams& p, int head_dim, cudaStream_t stream) { return chunk_launch<2>(p, head_dim, stream); }
}  // namespace iq
