// The gated feed-forward block's tensor-core forms: bf16, d and f multiples of eight.
#pragma once

#include "sb_internal.h"

namespace sb {

// f_real: columns of H (and of dG and dU) from there on are the filling of an odd width, c->f where there is none.  They are left as they are or written as zeros:
// the caller has put zeros there, and what an infinite operand times the filling's zeros gives must not replace them.
bool ffn_umma_ok(const sb_ffn_config* c);
// Where H [rows, f] and the backward pass's [dG dU] [rows, 2f] lie in the workspace
__nv_bfloat16* ffn_umma_h(const sb_ffn_config* c, void* ws);
__nv_bfloat16* ffn_umma_dgu(const sb_ffn_config* c, void* ws);
size_t ffn_umma_bytes(const sb_ffn_config* c, bool backward);
sb_status ffn_umma_forward(const sb_ffn_config* c, const void* x, const void* w_gu, const void* w_down, void* gu, void* y, void* ws, int f_real,
                           cudaStream_t st);
sb_status ffn_umma_backward(const sb_ffn_config* c, const void* dy, const void* x, const void* gu, const void* w_gu, const void* w_down, void* dx, void* dw_gu,
                            void* dw_down, void* ws, int f_real, cudaStream_t st);

// Estimated time of one product there, us: tiles of 128 weight columns (64 pairs), chunks of 64 reduction steps; mn: these run down the weights' columns.
double ffn_rows_us(int64_t rows, int tiles, int chunks, int mn);

// Few rows (sb_ffn_rows.cu).  down and dx fetch weights before they wait for the kernel in front of them: it must be the first product of the same pass,
// which triggers its dependents only after its own wait.
sb_status ffn_rows_glu(const sb_ffn_config* c, const void* x, const void* w_gu, void* gu, __nv_bfloat16* h, int f_real, cudaStream_t st);
sb_status ffn_rows_down(const sb_ffn_config* c, const __nv_bfloat16* h, const void* w_down, void* y, cudaStream_t st);
sb_status ffn_rows_glu_back(const sb_ffn_config* c, const void* dy, const void* gu, const void* w_down, __nv_bfloat16* dgu, __nv_bfloat16* h, int f_real, cudaStream_t st);
sb_status ffn_rows_dx(const sb_ffn_config* c, const __nv_bfloat16* dgu, const void* w_gu, void* dx, cudaStream_t st);

}  // namespace sb
