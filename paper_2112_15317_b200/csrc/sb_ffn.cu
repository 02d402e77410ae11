// Gated feed-forward block, forward and backward: host side, the form that takes any width, and the elementwise kernels.
//
//   GU = X Wgu^T,  H = a(G) * U,  Y = H Wd^T                      X [R, D], Wgu [2F, D] (gate rows first), Wd [D, F]
//   dH = dY Wd,  dG = dH * U * a'(G),  dU = dH * a(G),  dX = [dG dU] Wgu,  dWgu = [dG dU]^T X,  dWd = dY^T H
//
// a is SiLU, GELU (with erf) or ReLU.  The form here runs the products on the library's contraction kernels (float operands as three bf16
// terms on tensor cores, or CUDA cores; any width) with GU and dH in float between them.  Roundings in bf16: H, and dG and dU, where they become
// operands of a product; everything else is rounded once, at the end.
#include "sb_ffn.h"
#include "sb_ffn_umma.h"

#include <algorithm>

namespace sb {

namespace {

constexpr size_t MAX_PART_FLOATS = (size_t)16 << 20;

template <typename T> __device__ __forceinline__ float value(T v);
template <> __device__ __forceinline__ float value<float>(float v) { return v; }
template <> __device__ __forceinline__ float value<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// H = a(G) * U from the float products; GU itself where the backward pass will want it.
template <typename T>
__global__ void __launch_bounds__(256) ffn_act_kernel(const float* gu32, T* gu, T* h, int64_t rows, int f, int act)
{
    pdl_prologue();
    const int64_t n = rows * f, step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
        const int64_t r = i / f, at = r * 2 * f + (i - r * f);
        const float g = gu32[at], u = gu32[at + f];
        if (gu) { gu[at] = rounded<T>(g); gu[at + f] = rounded<T>(u); }
        h[i] = rounded<T>(ffn_act<true>(g, act) * u);
    }
}
// dG, dU and H from GU and the float dH.
template <typename T>
__global__ void __launch_bounds__(256) ffn_act_backward_kernel(const float* dh32, const T* gu, T* dgu, T* h, int64_t rows, int f, int act)
{
    pdl_prologue();
    const int64_t n = rows * f, step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
        const int64_t r = i / f, at = r * 2 * f + (i - r * f);
        const float u = value<T>(gu[at + f]), dh = dh32[i];
        float da;
        const float a = ffn_act_grad<true>(value<T>(gu[at]), act, da);
        dgu[at] = rounded<T>(dh * u * da);
        dgu[at + f] = rounded<T>(dh * a);
        h[i] = rounded<T>(a * u);
    }
}

__global__ void __launch_bounds__(256) ffn_round_kernel(const float* in, __nv_bfloat16* out, int64_t n)
{
    pdl_prologue();
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) out[i] = __float2bfloat16_rn(in[i]);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

sb_status check_config(const sb_ffn_config* c)
{
    if (!c) return set_error(SB_ERR_INVALID_ARG, "null config");
    if (c->precision != SB_FP32 && c->precision != SB_BF16) return set_error(SB_ERR_INVALID_ARG, "precision must be SB_FP32 or SB_BF16");
    if (c->act < SB_ACT_SILU || c->act > SB_ACT_RELU) return set_error(SB_ERR_INVALID_ARG, "unknown activation %d", c->act);
    if (c->rows < 0 || c->d < 1 || c->f < 1) return set_error(SB_ERR_SHAPE, "rows must not be negative, d and f must be positive");
    if (c->rows >= (int64_t)1 << 31 || c->f > (1 << 20) || c->d > (1 << 20)) return set_error(SB_ERR_UNSUPPORTED, "rows below 2^31, d and f up to 2^20");
    if (c->grad_dtype != SB_DT_F32 && !(c->grad_dtype == SB_DT_BF16 && c->precision == SB_BF16))
        return set_error(SB_ERR_INVALID_ARG, "weight gradients are SB_DT_F32, or SB_DT_BF16 with SB_BF16");
    return SB_OK;
}

// Consecutive 256-byte aligned pieces of the workspace.
struct Carve {
    char* base;
    size_t off = 0;
    template <typename T> T* take(size_t n) { T* p = base ? (T*)(base + off) : nullptr; off += (n * sizeof(T) + 255) / 256 * 256; return p; }
};
struct AnyForward { float *gu32, *zero, *part; void* h; };
struct AnyBackward { float *dh32, *part, *dw32; void *dgu, *h; };

ContractPlan product(int mode, const sb_ffn_config* c, int cin, int cout)
{
    return contract_plan(mode, (int)c->rows, 1, 1, 1, cin, cout, MAX_PART_FLOATS, c->precision == SB_FP32);
}
size_t part_of(const ContractPlan& p, size_t result) { return p.splits > 1 ? p.splits * result : 0; }

AnyForward carve_forward(Carve& k, const sb_ffn_config* c)
{
    AnyForward w{};
    const size_t R = c->rows, e = c->precision == SB_BF16 ? 2 : 4;
    w.gu32 = k.take<float>(R * 2 * c->f);
    w.h = k.take<char>(R * c->f * e);
    w.zero = k.take<float>(std::max(2 * c->f, c->d));
    w.part = k.take<float>(std::max(part_of(product(CMODE_FWD, c, c->d, 2 * c->f), R * 2 * c->f), part_of(product(CMODE_FWD, c, c->f, c->d), R * c->d)));
    return w;
}
AnyBackward carve_backward(Carve& k, const sb_ffn_config* c)
{
    AnyBackward w{};
    const size_t R = c->rows, D = c->d, F = c->f, e = c->precision == SB_BF16 ? 2 : 4;
    w.dh32 = k.take<float>(R * F);
    w.dgu = k.take<char>(R * 2 * F * e);
    w.h = k.take<char>(R * F * e);
    w.dw32 = k.take<float>((c->grad_dtype == SB_DT_BF16 ? 2 * F * D : 0) + std::max(2 * F, D));       // (the column sums of dY, which nobody wants, go behind it)
    size_t part = std::max(part_of(product(CMODE_DGRAD, c, c->f, c->d), R * F), part_of(product(CMODE_DGRAD, c, c->d, 2 * c->f), R * D));
    part = std::max(part, part_of(product(CMODE_WGRAD, c, c->d, 2 * c->f), 2 * F * D + 2 * F));
    part = std::max(part, part_of(product(CMODE_WGRAD, c, c->f, c->d), F * D + D));
    w.part = k.take<float>(part);
    return w;
}

#define F_TRY(expr)                                                                                    \
    do {                                                                                               \
        const cudaError_t e_ = (expr);                                                                 \
        if (e_ != cudaSuccess) return set_error(SB_ERR_CUDA, "ffn: %s: %s", #expr, cudaGetErrorString(e_)); \
    } while (0)

ContractArgs contract_of(int mode, const sb_ffn_config* c, int cin, int cout, float* part)
{
    ContractArgs a{};
    a.mode = mode; a.taps = 1; a.B = (int)c->rows; a.H = a.W = 1; a.Cin = cin; a.Cout = cout;
    a.plan = product(mode, c, cin, cout);
    a.part = part;
    a.split_stride = (long)c->rows * (mode == CMODE_FWD ? cout : cin);
    a.status = ops_status();
    return a;
}
int blocks_of(int64_t n) { return (int)std::min<int64_t>((n + 255) / 256, 148 * 16); }

sb_status any_forward(const sb_ffn_config* c, const void* x, const void* w_gu, const void* w_down, void* gu, void* y, void* ws, cudaStream_t st)
{
    Carve k{(char*)ws};
    const AnyForward w = carve_forward(k, c);
    const bool bf = c->precision == SB_BF16;
    F_TRY(cudaMemsetAsync(w.zero, 0, std::max(2 * c->f, c->d) * sizeof(float), st));
    ContractArgs a = contract_of(CMODE_FWD, c, c->d, 2 * c->f, w.part);
    a.act = x; a.wt = w_gu; a.bias = w.zero; a.out32 = w.gu32;
    F_TRY(launch_contract(a, bf, st));
    const int64_t n = c->rows * c->f;
    if (bf) F_TRY(pdl_launch(ffn_act_kernel<__nv_bfloat16>, dim3(blocks_of(n)), dim3(256), 0, st, w.gu32, (__nv_bfloat16*)gu, (__nv_bfloat16*)w.h, c->rows, c->f, c->act));
    else F_TRY(pdl_launch(ffn_act_kernel<float>, dim3(blocks_of(n)), dim3(256), 0, st, w.gu32, (float*)gu, (float*)w.h, c->rows, c->f, c->act));
    ContractArgs b = contract_of(CMODE_FWD, c, c->f, c->d, w.part);
    b.act = w.h; b.wt = w_down; b.bias = w.zero; b.out = y;
    F_TRY(launch_contract(b, bf, st));
    return SB_OK;
}

// dW [cout, cin] = dy^T act
sb_status weight_gradient(const sb_ffn_config* c, const void* act, const void* dy, int cin, int cout, void* dw, const AnyBackward& w, cudaStream_t st)
{
    const size_t n = (size_t)cin * cout;
    const bool bf = c->precision == SB_BF16, round = c->grad_dtype == SB_DT_BF16;
    float* out = round ? w.dw32 : (float*)dw;
    float* sums = round ? w.dw32 + n : w.dw32;
    ContractArgs a = contract_of(CMODE_WGRAD, c, cin, cout, w.part);
    a.act = act; a.dy = dy;
    const int S = a.plan.splits;
    a.part = S > 1 ? w.part : out;
    a.split_stride = (long)(n + cout);
    a.bias_off = S > 1 ? (long)n : (long)(sums - out);
    F_TRY(launch_contract(a, bf, st));
    if (S > 1) F_TRY(launch_reduce_partials(w.part, n + cout, out, n, S, st));
    if (round) F_TRY(pdl_launch(ffn_round_kernel, dim3(blocks_of((int64_t)n)), dim3(256), 0, st, out, (__nv_bfloat16*)dw, (int64_t)n));
    return SB_OK;
}

sb_status any_backward(const sb_ffn_config* c, const void* dy, const void* x, const void* gu, const void* w_gu, const void* w_down, void* dx, void* dw_gu,
                       void* dw_down, void* ws, cudaStream_t st)
{
    Carve k{(char*)ws};
    const AnyBackward w = carve_backward(k, c);
    const bool bf = c->precision == SB_BF16;
    ContractArgs a = contract_of(CMODE_DGRAD, c, c->f, c->d, w.part);
    a.wt = w_down; a.dy = dy; a.out32 = w.dh32;
    F_TRY(launch_contract(a, bf, st));
    const int64_t n = c->rows * c->f;
    if (bf) F_TRY(pdl_launch(ffn_act_backward_kernel<__nv_bfloat16>, dim3(blocks_of(n)), dim3(256), 0, st, w.dh32, (const __nv_bfloat16*)gu, (__nv_bfloat16*)w.dgu, (__nv_bfloat16*)w.h, c->rows, c->f, c->act));
    else F_TRY(pdl_launch(ffn_act_backward_kernel<float>, dim3(blocks_of(n)), dim3(256), 0, st, w.dh32, (const float*)gu, (float*)w.dgu, (float*)w.h, c->rows, c->f, c->act));
    if (dx) {
        ContractArgs b = contract_of(CMODE_DGRAD, c, c->d, 2 * c->f, w.part);
        b.wt = w_gu; b.dy = w.dgu; b.out = dx;
        F_TRY(launch_contract(b, bf, st));
    }
    if (dw_gu) { const sb_status s = weight_gradient(c, x, w.dgu, c->d, 2 * c->f, dw_gu, w, st); if (s != SB_OK) return s; }
    if (dw_down) { const sb_status s = weight_gradient(c, w.h, dy, c->f, c->d, dw_down, w, st); if (s != SB_OK) return s; }
    return SB_OK;
}

}  // namespace

static __device__ uint32_t g_ops_status;

// (the address is looked up once per device)
uint32_t* ops_status()
{
    if (ops_status_of_model()) return ops_status_of_model();
    static uint32_t* at[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    if (!at[dev]) {
        void* p = nullptr;
        if (cudaGetSymbolAddress(&p, g_ops_status) != cudaSuccess) return nullptr;
        at[dev] = (uint32_t*)p;
    }
    return at[dev];
}

size_t ffn_any_bytes(const sb_ffn_config* c, bool backward)
{
    Carve k{nullptr};
    if (backward) carve_backward(k, c); else carve_forward(k, c);
    return k.off;
}

}  // namespace sb

using namespace sb;

extern "C" {

sb_status sb_ffn_bytes(const sb_ffn_config* c, int32_t backward, size_t* bytes)
{
    const sb_status s = check_config(c);
    if (s != SB_OK) return s;
    if (!bytes) return set_error(SB_ERR_INVALID_ARG, "bytes is null");
    *bytes = c->rows == 0 ? 0 : ffn_umma_ok(c) ? ffn_umma_bytes(c, backward != 0) : ffn_any_bytes(c, backward != 0);
    return SB_OK;
}

sb_status sb_ops_check(void* stream)
{
    uint32_t* word = ops_status();
    if (!word) return set_error(SB_ERR_CUDA, "the status word has no address on this device");
    uint32_t code = 0;
    F_TRY(cudaMemcpyAsync(&code, word, sizeof(code), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
    F_TRY(cudaStreamSynchronize((cudaStream_t)stream));
    if (code == DEV_OK) return SB_OK;
    F_TRY(cudaMemsetAsync(word, 0, sizeof(code), (cudaStream_t)stream));
    return set_error(SB_ERR_TIMEOUT, "a bounded wait ran out in an operator's kernel (code %u)", code);
}

static sb_status check_workspace(const sb_ffn_config* c, bool backward, const void* ws, size_t ws_bytes)
{
    size_t need = 0;
    const sb_status s = sb_ffn_bytes(c, backward, &need);
    if (s != SB_OK) return s;
    if (need > 0 && (!ws || ((uintptr_t)ws & 255))) return set_error(SB_ERR_INVALID_ARG, "the workspace is null or not 256-byte aligned");
    if (ws_bytes < need) return set_error(SB_ERR_ARENA_TOO_SMALL, "the workspace has %zu bytes, the call needs %zu", ws_bytes, need);
    return SB_OK;
}

sb_status sb_ffn_forward(const sb_ffn_config* c, const void* x, const void* w_gate_up, const void* w_down, void* gu, void* y, void* ws, size_t ws_bytes, void* stream)
{
    const sb_status s = check_workspace(c, false, ws, ws_bytes);
    if (s != SB_OK) return s;
    if (c->rows == 0) return SB_OK;
    if (!x || !w_gate_up || !w_down || !y) return set_error(SB_ERR_INVALID_ARG, "null matrix");
    if (!aligned16(x) || !aligned16(w_gate_up) || !aligned16(w_down) || !aligned16(gu) || !aligned16(y)) return set_error(SB_ERR_INVALID_ARG, "every matrix must be 16-byte aligned");
    if (!ops_status()) return set_error(SB_ERR_CUDA, "the status word has no address on this device");
    if (ffn_umma_ok(c)) return ffn_umma_forward(c, x, w_gate_up, w_down, gu, y, ws, (cudaStream_t)stream);
    return any_forward(c, x, w_gate_up, w_down, gu, y, ws, (cudaStream_t)stream);
}

sb_status sb_ffn_backward(const sb_ffn_config* c, const void* dy, const void* x, const void* gu, const void* w_gate_up, const void* w_down, void* dx,
                          void* dw_gate_up, void* dw_down, void* ws, size_t ws_bytes, void* stream)
{
    const sb_status s = check_workspace(c, true, ws, ws_bytes);
    if (s != SB_OK) return s;
    const size_t ge = c->grad_dtype == SB_DT_BF16 ? 2 : 4, n = (size_t)c->d * c->f;
    if (!aligned16(dy) || !aligned16(x) || !aligned16(gu) || !aligned16(w_gate_up) || !aligned16(w_down) || !aligned16(dx) || !aligned16(dw_gate_up) || !aligned16(dw_down))
        return set_error(SB_ERR_INVALID_ARG, "every matrix must be 16-byte aligned");
    if (c->rows == 0) {           // empty sums
        if (dw_gate_up) F_TRY(cudaMemsetAsync(dw_gate_up, 0, 2 * n * ge, (cudaStream_t)stream));
        if (dw_down) F_TRY(cudaMemsetAsync(dw_down, 0, n * ge, (cudaStream_t)stream));
        return SB_OK;
    }
    if (!dy || !x || !gu || !w_gate_up || !w_down) return set_error(SB_ERR_INVALID_ARG, "null matrix");
    if (!ops_status()) return set_error(SB_ERR_CUDA, "the status word has no address on this device");
    if (ffn_umma_ok(c)) return ffn_umma_backward(c, dy, x, gu, w_gate_up, w_down, dx, dw_gate_up, dw_down, ws, (cudaStream_t)stream);
    return any_backward(c, dy, x, gu, w_gate_up, w_down, dx, dw_gate_up, dw_down, ws, (cudaStream_t)stream);
}

}  // extern "C"
