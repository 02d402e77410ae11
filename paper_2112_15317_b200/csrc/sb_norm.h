// Internal form of the norms around a block (sb_norm.cu): the model's layer below may be a ReLU layer.
#pragma once

#include "../../include/splitbrain.h"
#include <cuda_runtime.h>

namespace sb {

// sb_norm_backward; relu_x: dx is zero where x <= 0
sb_status norm_backward(const sb_norm_config* c, const void* dy, const void* dn, const float* stats, const void* x, const float* w_pre, const void* f,
                        const float* w_post, const float* gate, const float* scale, void* dx, void* df, float* dw_pre, float* dw_post, float* dgate,
                        float* dscale, void* ws, size_t ws_bytes, bool relu_x, cudaStream_t st);

}  // namespace sb
