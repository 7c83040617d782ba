// Backward pass of the norms around a block, row kernels: bf16 gradients of the residual stream, f32 ones of the block.
#include "block_norm_bwd.cuh"

namespace turnopd {
template cudaError_t launch_block_rows_bwd<__nv_bfloat16, float>(const BlockGradCall &, int *, bool *, cudaStream_t);
}  // namespace turnopd
