// The tree attention kernel for 2-bit codes.
#include "iq_tree_kernel.cuh"

namespace iq {
cudaError_t launch_tree_b2(const TreeParams& p, int head_dim, cudaStream_t stream) { return tree_launch<2>(p, head_dim, stream); }
}  // namespace iq
