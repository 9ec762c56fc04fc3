// Kernels around a block, float16 branch.
#define FLARE_BLOCK_INSTANTIATE
#include "flare_block_launch.cuh"

namespace flare {
template int block_forward<__half, __half>(BlockArgs, bool, bool, const BlockPlan &, cudaStream_t);
template int block_backward<__half, __half>(BlockArgs, bool, bool, bool, const BlockPlan &, cudaStream_t);
template int block_forward<__half, float>(BlockArgs, bool, bool, const BlockPlan &, cudaStream_t);
template int block_backward<__half, float>(BlockArgs, bool, bool, bool, const BlockPlan &, cudaStream_t);
template int block_sums<__half>(const BlockSums &, cudaStream_t);
}  // namespace flare
