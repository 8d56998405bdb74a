// The tree attention kernel for 3-bit codes.
#include "iq_tree_kernel.cuh"

namespace iq {
cudaError_t launch_tree_b3(const TreeParams& p, int head_dim, cudaStream_t stream) { return tree_launch<3>(p, head_dim, stream); }
}  // namespace iq
