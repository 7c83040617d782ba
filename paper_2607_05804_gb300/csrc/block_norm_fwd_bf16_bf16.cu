// Forward pass of the norms around a block, row kernels: bf16 residual stream, bf16 block output.
#include "block_norm_fwd.cuh"

namespace turnopd {
template cudaError_t launch_block_rows_fwd<__nv_bfloat16, __nv_bfloat16>(const BlockCall &, const Phases &, cudaStream_t);
}  // namespace turnopd
