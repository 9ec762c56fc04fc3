// Kernels around a block: bfloat16 branch, float32 residual stream.
#define FLARE_BLOCK_INSTANTIATE
#include "flare_block_launch.cuh"

namespace flare {
template int block_forward<__nv_bfloat16, float>(const BlockArgs &, bool, int, cudaStream_t);
template int block_backward<__nv_bfloat16, float>(const BlockArgs &, bool, bool, const BlockPlan &, cudaStream_t);
}  // namespace flare
