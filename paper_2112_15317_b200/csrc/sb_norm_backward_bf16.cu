// Backward pass of the norms around a block, bfloat16 activations.
#include "sb_norm_backward.cuh"

namespace sb {

cudaError_t launch_norm_backward_bf16(const NormParams& p, bool layer, int64_t ctas, cudaStream_t st) { return backward_pieces<__nv_bfloat16>(p, layer, ctas, st); }

}  // namespace sb
