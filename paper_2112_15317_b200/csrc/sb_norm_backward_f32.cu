// Backward pass of the norms around a block, float activations.
#include "sb_norm_backward.cuh"

namespace sb {

cudaError_t launch_norm_backward_f32(const NormParams& p, bool layer, int64_t ctas, cudaStream_t st) { return backward_pieces<float>(p, layer, ctas, st); }

}  // namespace sb
