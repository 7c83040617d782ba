// Backward pass of the norms around a block, row kernels: f32 gradients of the residual stream, bf16 ones of the block.
#include "block_norm_bwd.cuh"

namespace turnopd {
template cudaError_t launch_block_rows_bwd<float, __nv_bfloat16>(const BlockGradCall &, int *, bool *, cudaStream_t);
}  // namespace turnopd
