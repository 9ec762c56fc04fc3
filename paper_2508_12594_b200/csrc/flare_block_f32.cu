// Kernels around a block, float32 branch.
#define FLARE_BLOCK_INSTANTIATE
#include "flare_block_launch.cuh"

namespace flare {
template int block_forward<float, float>(BlockArgs, bool, bool, const BlockPlan &, cudaStream_t);
template int block_backward<float, float>(BlockArgs, bool, bool, bool, const BlockPlan &, cudaStream_t);
template int block_sums<float>(const BlockSums &, cudaStream_t);
}  // namespace flare
