// The gated feed-forward block's tensor-core form (sb_ffn_umma.cu): bf16, d and f multiples of eight.
#pragma once

#include "sb_internal.h"

namespace sb {

bool ffn_umma_ok(const sb_ffn_config* c);
size_t ffn_umma_bytes(const sb_ffn_config* c, bool backward);
sb_status ffn_umma_forward(const sb_ffn_config* c, const void* x, const void* w_gu, const void* w_down, void* gu, void* y, void* ws, cudaStream_t st);
sb_status ffn_umma_backward(const sb_ffn_config* c, const void* dy, const void* x, const void* gu, const void* w_gu, const void* w_down, void* dx, void* dw_gu,
                            void* dw_down, void* ws, cudaStream_t st);

}  // namespace sb
