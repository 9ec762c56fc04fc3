// Kernels around a block: float16 branch, float16 residual stream.
#define FLARE_BLOCK_INSTANTIATE
#include "flare_block_launch.cuh"

namespace flare {
template int block_forward<__half, __half>(const BlockArgs &, bool, int, cudaStream_t);
template int block_backward<__half, __half>(const BlockArgs &, bool, bool, const BlockPlan &, cudaStream_t);
template int block_sums<__half>(const BlockSums &, cudaStream_t);
}  // namespace flare
