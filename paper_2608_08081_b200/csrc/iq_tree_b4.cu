// The tree attention kernel for 4-bit codes.
#include "iq_tree_kernel.cuh"

namespace iq {
cudaError_t launch_tree_b4(const TreeParams& p, int head_dim, cudaStream_t stream) { return tree_launch<4>(p, head_dim, stream); }
}  // namespace iq
