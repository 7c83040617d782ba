// Forward pass of the norms around a block, row kernels: f32 residual stream, bf16 block output.
#include "block_norm_fwd.cuh"

namespace turnopd {
template cudaError_t launch_block_rows_fwd<float, __nv_bfloat16>(const BlockCall &, const Phases &, cudaStream_t);
}  // namespace turnopd
