// Kernels around a block: float32 branch, float32 residual stream.
#define FLARE_BLOCK_INSTANTIATE
#include "flare_block_launch.cuh"

namespace flare {
template int block_forward<float, float>(const BlockArgs &, bool, int, cudaStream_t);
template int block_backward<float, float>(const BlockArgs &, bool, bool, const BlockPlan &, cudaStream_t);
template int block_sums<float>(const BlockSums &, cudaStream_t);
}  // namespace flare
