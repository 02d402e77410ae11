// Gated feed-forward block, forward and backward: host side, the form that takes any width, and the elementwise kernels.
//
//   GU = X Wgu^T,  H = a(G) * U,  Y = H Wd^T                      X [R, D], Wgu [2F, D] (gate rows first), Wd [D, F]
//   dH = dY Wd,  dG = dH * U * a'(G),  dU = dH * a(G),  dX = [dG dU] Wgu,  dWgu = [dG dU]^T X,  dWd = dY^T H
//
// a is SiLU, GELU (with erf) or ReLU.  bf16 runs on the kernels of sb_ffn_umma.cu and sb_ffn_rows.cu.  Float runs the products on the library's contraction
// kernels (every operand as three bf16 terms on tensor cores, or on CUDA cores where that is faster) with an elementwise kernel between them.
// Widths that are not multiples of eight: the operands are copied into rows of the next multiple, filled up with zeros, which add nothing to any product, and
// the results cut out again.  (250 rows, 1023 x 2731, float, backward: 350 us on the CUDA-core kernel for odd widths, 131 so.)
// (H, dG and dU are zero in the filled-up columns whatever comes out there: an infinite operand times their zeros is NaN, which the next product would spread over the row.)
// Roundings in bf16: H, and dG and dU, where they become operands of a product; everything else is rounded once, at the end.
#include "sb_ffn.h"
#include "sb_ffn_umma.h"

#include <algorithm>

namespace sb {

namespace {

constexpr size_t MAX_PART_FLOATS = (size_t)16 << 20;

// Four columns, those from `live` on as zeros
__device__ __forceinline__ float4 live_columns(float4 v, int live) { return make_float4(live > 0 ? v.x : 0.f, live > 1 ? v.y : 0.f, live > 2 ? v.z : 0.f, live > 3 ? v.w : 0.f); }
// H = a(G) * U; widths that are multiples of four, four columns a thread; columns from f_real on are zero
__global__ void __launch_bounds__(256) ffn_act_kernel(const float4* gu, float4* h, int64_t rows, int f4, int f_real, int act)
{
    pdl_prologue();
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int c = blockIdx.y * 256 + threadIdx.x; c < f4; c += gridDim.y * 256) {
            const float4 g = gu[r * 2 * f4 + c], u = gu[r * 2 * f4 + f4 + c];
            h[r * f4 + c] = live_columns(make_float4(ffn_act<true>(g.x, act) * u.x, ffn_act<true>(g.y, act) * u.y, ffn_act<true>(g.z, act) * u.z, ffn_act<true>(g.w, act) * u.w),
                                         f_real - 4 * c);
        }
}
// dG, dU and H from GU and dH
__global__ void __launch_bounds__(256) ffn_act_backward_kernel(const float4* dh, const float4* gu, float4* dgu, float4* h, int64_t rows, int f4, int f_real, int act)
{
    pdl_prologue();
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int c = blockIdx.y * 256 + threadIdx.x; c < f4; c += gridDim.y * 256) {
            const int64_t at = r * 2 * f4 + c;
            const float4 g = gu[at], u = gu[at + f4], d = dh[r * f4 + c];
            float4 da, a;
            a.x = ffn_act_grad<true>(g.x, act, da.x); a.y = ffn_act_grad<true>(g.y, act, da.y);
            a.z = ffn_act_grad<true>(g.z, act, da.z); a.w = ffn_act_grad<true>(g.w, act, da.w);
            const int live = f_real - 4 * c;
            dgu[at] = live_columns(make_float4(d.x * u.x * da.x, d.y * u.y * da.y, d.z * u.z * da.z, d.w * u.w * da.w), live);
            dgu[at + f4] = live_columns(make_float4(d.x * a.x, d.y * a.y, d.z * a.z, d.w * a.w), live);
            h[r * f4 + c] = live_columns(make_float4(a.x * u.x, a.y * u.y, a.z * u.z, a.w * u.w), live);
        }
}

// Matrices of one element size copied into others with rows of another length; what the source does not have is zero.  A block takes pieces of eight
// rows x 256 columns of any of them, a thread one column: eight loads under way, whatever the shapes.
struct CopyOne { const void* src; void* dst; int64_t src_rows, src_cols; int src_ld; int64_t rows, cols; int ld; int64_t first; int across; };      // pieces before it, pieces across
struct CopyArgs { CopyOne m[10]; int count; int64_t pieces; };
template <typename T>
__global__ void __launch_bounds__(256) ffn_copy_kernel(const __grid_constant__ CopyArgs a)
{
    pdl_prologue();
    for (int64_t q = blockIdx.x; q < a.pieces; q += gridDim.x) {
        int k = 0;
        while (k + 1 < a.count && q >= a.m[k + 1].first) ++k;
        const CopyOne& m = a.m[k];
        const uint32_t at = (uint32_t)(q - m.first), down = at / (uint32_t)m.across;
        const int64_t r = (int64_t)down * 8, c = (int64_t)(at - down * (uint32_t)m.across) * 256 + threadIdx.x;
        if (c >= m.cols) continue;
        const int have = c < m.src_cols ? (int)min((int64_t)8, m.src_rows - r) : 0, rows = (int)min((int64_t)8, m.rows - r);
        const T* src = (const T*)m.src + r * m.src_ld + c;
        T* dst = (T*)m.dst + r * m.ld + c;
        T v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < have ? __ldg(src + i * m.src_ld) : T(0);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < rows) dst[i * m.ld] = v[i];
    }
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

#define F_TRY(expr)                                                                                    \
    do {                                                                                               \
        const cudaError_t e_ = (expr);                                                                 \
        if (e_ != cudaSuccess) return set_error(SB_ERR_CUDA, "ffn: %s: %s", #expr, cudaGetErrorString(e_)); \
    } while (0)
#define S_TRY(expr)                     \
    do {                                \
        const sb_status s_ = (expr);    \
        if (s_ != SB_OK) return s_;     \
    } while (0)

// ---- float, widths that are multiples of eight ----
struct FloatForward { float *gu, *h, *zero, *part; };
struct FloatBackward { float *dh, *dgu, *h, *sums, *part; };

ContractPlan product(int mode, const sb_ffn_config* c, int cin, int cout) { return contract_plan(mode, (int)c->rows, 1, 1, 1, cin, cout, MAX_PART_FLOATS, true); }
size_t part_of(const ContractPlan& p, size_t result) { return p.splits > 1 ? p.splits * result : 0; }

FloatForward carve_forward(Carve& k, const sb_ffn_config* c)
{
    FloatForward w{};
    const size_t R = c->rows;
    w.gu = k.take<float>(R * 2 * c->f);
    w.h = k.take<float>(R * c->f);
    w.zero = k.take<float>(std::max(2 * c->f, c->d));
    w.part = k.take<float>(std::max(part_of(product(CMODE_FWD, c, c->d, 2 * c->f), R * 2 * c->f), part_of(product(CMODE_FWD, c, c->f, c->d), R * c->d)));
    return w;
}
FloatBackward carve_backward(Carve& k, const sb_ffn_config* c)
{
    FloatBackward w{};
    const size_t R = c->rows, D = c->d, F = c->f;
    w.dh = k.take<float>(R * F);
    w.dgu = k.take<float>(R * 2 * F);
    w.h = k.take<float>(R * F);
    w.sums = k.take<float>(std::max(2 * F, D));       // (column sums that the weight-gradient kernel also makes and nobody wants)
    size_t part = std::max(part_of(product(CMODE_DGRAD, c, c->f, c->d), R * F), part_of(product(CMODE_DGRAD, c, c->d, 2 * c->f), R * D));
    part = std::max(part, part_of(product(CMODE_WGRAD, c, c->d, 2 * c->f), 2 * F * D + 2 * F));
    part = std::max(part, part_of(product(CMODE_WGRAD, c, c->f, c->d), F * D + D));
    w.part = k.take<float>(part);
    return w;
}
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
dim3 act_grid(const sb_ffn_config* c)
{
    const int cols = (c->f / 4 + 255) / 256;
    return dim3((unsigned)std::min<int64_t>(c->rows, 148 * 8), (unsigned)std::min(cols, 16));
}

sb_status float_forward(const sb_ffn_config* c, const float* x, const float* w_gu, const float* w_down, float* gu, float* y, void* ws, int f_real, cudaStream_t st)
{
    Carve k{(char*)ws};
    const FloatForward w = carve_forward(k, c);
    float* g = gu ? gu : w.gu;
    F_TRY(cudaMemsetAsync(w.zero, 0, std::max(2 * c->f, c->d) * sizeof(float), st));      // (the contraction adds a bias)
    ContractArgs a = contract_of(CMODE_FWD, c, c->d, 2 * c->f, w.part);
    a.act = x; a.wt = w_gu; a.bias = w.zero; a.out = g;
    F_TRY(launch_contract(a, false, st));
    F_TRY(pdl_launch(ffn_act_kernel, act_grid(c), dim3(256), 0, st, (const float4*)g, (float4*)w.h, c->rows, c->f / 4, f_real, c->act));
    ContractArgs b = contract_of(CMODE_FWD, c, c->f, c->d, w.part);
    b.act = w.h; b.wt = w_down; b.bias = w.zero; b.out = y;
    F_TRY(launch_contract(b, false, st));
    return SB_OK;
}

// dW [cout, cin] = dy^T act
sb_status weight_gradient(const sb_ffn_config* c, const float* act, const float* dy, int cin, int cout, float* dw, const FloatBackward& w, cudaStream_t st)
{
    const size_t n = (size_t)cin * cout;
    ContractArgs a = contract_of(CMODE_WGRAD, c, cin, cout, w.part);
    a.act = act; a.dy = dy;
    const int S = a.plan.splits;
    a.part = S > 1 ? w.part : dw;
    a.split_stride = (long)(n + cout);
    a.bias_off = S > 1 ? (long)n : (long)(w.sums - dw);
    F_TRY(launch_contract(a, false, st));
    if (S > 1) F_TRY(launch_reduce_partials(w.part, n + cout, dw, n, S, st));
    return SB_OK;
}

sb_status float_backward(const sb_ffn_config* c, const float* dy, const float* x, const float* gu, const float* w_gu, const float* w_down, float* dx, float* dw_gu,
                         float* dw_down, void* ws, int f_real, cudaStream_t st)
{
    Carve k{(char*)ws};
    const FloatBackward w = carve_backward(k, c);
    ContractArgs a = contract_of(CMODE_DGRAD, c, c->f, c->d, w.part);
    a.wt = w_down; a.dy = dy; a.out = w.dh;
    F_TRY(launch_contract(a, false, st));
    F_TRY(pdl_launch(ffn_act_backward_kernel, act_grid(c), dim3(256), 0, st, (const float4*)w.dh, (const float4*)gu, (float4*)w.dgu, (float4*)w.h, c->rows, c->f / 4, f_real, c->act));
    if (dx) {
        ContractArgs b = contract_of(CMODE_DGRAD, c, c->d, 2 * c->f, w.part);
        b.wt = w_gu; b.dy = w.dgu; b.out = dx;
        F_TRY(launch_contract(b, false, st));
    }
    if (dw_gu) S_TRY(weight_gradient(c, x, w.dgu, c->d, 2 * c->f, dw_gu, w, st));
    if (dw_down) S_TRY(weight_gradient(c, w.h, dy, c->f, c->d, dw_down, w, st));
    return SB_OK;
}

// ---- any precision, widths that are multiples of eight ----
size_t even_bytes(const sb_ffn_config* c, bool backward)
{
    if (ffn_umma_ok(c)) return ffn_umma_bytes(c, backward);
    Carve k{nullptr};
    if (backward) carve_backward(k, c); else carve_forward(k, c);
    return k.off;
}
sb_status even_forward(const sb_ffn_config* c, const void* x, const void* w_gu, const void* w_down, void* gu, void* y, void* ws, int f_real, cudaStream_t st)
{
    if (ffn_umma_ok(c)) return ffn_umma_forward(c, x, w_gu, w_down, gu, y, ws, f_real, st);
    return float_forward(c, (const float*)x, (const float*)w_gu, (const float*)w_down, (float*)gu, (float*)y, ws, f_real, st);
}
sb_status even_backward(const sb_ffn_config* c, const void* dy, const void* x, const void* gu, const void* w_gu, const void* w_down, void* dx, void* dw_gu,
                        void* dw_down, void* ws, int f_real, cudaStream_t st)
{
    if (ffn_umma_ok(c)) return ffn_umma_backward(c, dy, x, gu, w_gu, w_down, dx, dw_gu, dw_down, ws, f_real, st);
    return float_backward(c, (const float*)dy, (const float*)x, (const float*)gu, (const float*)w_gu, (const float*)w_down, (float*)dx, (float*)dw_gu, (float*)dw_down, ws, f_real, st);
}

// ---- any width ----
bool even(const sb_ffn_config* c) { return c->d % 8 == 0 && c->f % 8 == 0; }
sb_ffn_config padded(const sb_ffn_config* c)
{
    sb_ffn_config p = *c;
    p.d = (c->d + 7) / 8 * 8;
    p.f = (c->f + 7) / 8 * 8;
    return p;
}
struct Padded { char *x, *dy, *gu, *w_gu, *w_down, *y, *dw_gu, *dw_down; void* inner; };      // y: y, or dx
Padded carve_padded(Carve& k, const sb_ffn_config* p, bool backward)
{
    Padded w{};
    const size_t e = p->precision == SB_BF16 ? 2 : 4, ge = p->grad_dtype == SB_DT_BF16 ? 2 : 4, R = p->rows, D = p->d, F = p->f;
    w.x = k.take<char>(R * D * e);
    if (backward) w.dy = k.take<char>(R * D * e);
    w.gu = k.take<char>(R * 2 * F * e);
    w.w_gu = k.take<char>(2 * F * D * e);
    w.w_down = k.take<char>(F * D * e);
    w.y = k.take<char>(R * D * e);
    if (backward) { w.dw_gu = k.take<char>(2 * F * D * ge); w.dw_down = k.take<char>(F * D * ge); }
    w.inner = k.take<char>(even_bytes(p, backward));
    return w;
}
// [rows, cols] of src, cols apart, into [to_rows, to_cols] of dst, ld apart
void copy_of(CopyArgs& a, const void* src, int64_t rows, int64_t cols, int64_t src_ld, void* dst, int64_t to_rows, int64_t to_cols, int64_t ld)
{
    const int across = (int)((to_cols + 255) / 256);
    a.m[a.count++] = CopyOne{src, dst, rows, cols, (int)src_ld, to_rows, to_cols, (int)ld, a.pieces, across};
    a.pieces += (to_rows + 7) / 8 * across;
}
// zeros into what is H's filling in bf16, [dG dU]'s too in the backward pass (float: the activation kernels write them)
void clear_filling(CopyArgs& a, const sb_ffn_config* c, const sb_ffn_config* p, void* inner, bool backward)
{
    if (c->precision != SB_BF16 || c->f == p->f) return;
    const int64_t fill = p->f - c->f;
    copy_of(a, nullptr, 0, 0, 0, ffn_umma_h(p, inner) + c->f, c->rows, fill, p->f);
    if (!backward) return;
    copy_of(a, nullptr, 0, 0, 0, ffn_umma_dgu(p, inner) + c->f, c->rows, fill, 2 * p->f);
    copy_of(a, nullptr, 0, 0, 0, ffn_umma_dgu(p, inner) + p->f + c->f, c->rows, fill, 2 * p->f);
}
cudaError_t launch_copies(const CopyArgs& a, size_t e, cudaStream_t st)
{
    const dim3 grid((unsigned)std::min<int64_t>(a.pieces, 148 * 32));
    return e == 2 ? pdl_launch(ffn_copy_kernel<uint16_t>, grid, dim3(256), 0, st, a) : pdl_launch(ffn_copy_kernel<uint32_t>, grid, dim3(256), 0, st, a);
}
const void* behind(const void* p, size_t elements, size_t e) { return (const char*)p + elements * e; }
void* behind(void* p, size_t elements, size_t e) { return (char*)p + elements * e; }

sb_status odd_forward(const sb_ffn_config* c, const void* x, const void* w_gu, const void* w_down, void* gu, void* y, void* ws, cudaStream_t st)
{
    const sb_ffn_config p = padded(c);
    Carve k{(char*)ws};
    const Padded w = carve_padded(k, &p, false);
    const size_t e = c->precision == SB_BF16 ? 2 : 4;
    const int64_t R = c->rows, D = c->d, F = c->f, D2 = p.d, F2 = p.f;
    CopyArgs in{}, out{};
    copy_of(in, x, R, D, D, w.x, R, D2, D2);
    copy_of(in, w_gu, F, D, D, w.w_gu, F2, D2, D2);
    copy_of(in, behind(w_gu, F * D, e), F, D, D, behind((void*)w.w_gu, F2 * D2, e), F2, D2, D2);
    copy_of(in, w_down, D, F, F, w.w_down, D2, F2, F2);
    clear_filling(in, c, &p, w.inner, false);
    F_TRY(launch_copies(in, e, st));
    S_TRY(even_forward(&p, w.x, w.w_gu, w.w_down, gu ? w.gu : nullptr, w.y, w.inner, c->f, st));
    copy_of(out, w.y, R, D, D2, y, R, D, D);
    if (gu) {
        copy_of(out, w.gu, R, F, 2 * F2, gu, R, F, 2 * F);
        copy_of(out, behind((const void*)w.gu, F2, e), R, F, 2 * F2, behind(gu, F, e), R, F, 2 * F);
    }
    F_TRY(launch_copies(out, e, st));
    return SB_OK;
}
sb_status odd_backward(const sb_ffn_config* c, const void* dy, const void* x, const void* gu, const void* w_gu, const void* w_down, void* dx, void* dw_gu,
                       void* dw_down, void* ws, cudaStream_t st)
{
    const sb_ffn_config p = padded(c);
    Carve k{(char*)ws};
    const Padded w = carve_padded(k, &p, true);
    const size_t e = c->precision == SB_BF16 ? 2 : 4, ge = c->grad_dtype == SB_DT_BF16 ? 2 : 4;
    const int64_t R = c->rows, D = c->d, F = c->f, D2 = p.d, F2 = p.f;
    CopyArgs in{}, out{}, grads{};
    copy_of(in, x, R, D, D, w.x, R, D2, D2);
    copy_of(in, dy, R, D, D, w.dy, R, D2, D2);
    copy_of(in, gu, R, F, 2 * F, w.gu, R, F2, 2 * F2);
    copy_of(in, behind(gu, F, e), R, F, 2 * F, behind((void*)w.gu, F2, e), R, F2, 2 * F2);
    copy_of(in, w_gu, F, D, D, w.w_gu, F2, D2, D2);
    copy_of(in, behind(w_gu, F * D, e), F, D, D, behind((void*)w.w_gu, F2 * D2, e), F2, D2, D2);
    copy_of(in, w_down, D, F, F, w.w_down, D2, F2, F2);
    clear_filling(in, c, &p, w.inner, true);
    F_TRY(launch_copies(in, e, st));
    S_TRY(even_backward(&p, w.dy, w.x, w.gu, w.w_gu, w.w_down, dx ? w.y : nullptr, dw_gu ? w.dw_gu : nullptr, dw_down ? w.dw_down : nullptr, w.inner, c->f, st));
    CopyArgs& g = ge == e ? out : grads;
    if (dx) copy_of(out, w.y, R, D, D2, dx, R, D, D);
    if (dw_gu) {
        copy_of(g, w.dw_gu, F, D, D2, dw_gu, F, D, D);
        copy_of(g, behind((const void*)w.dw_gu, F2 * D2, ge), F, D, D2, behind(dw_gu, F * D, ge), F, D, D);
    }
    if (dw_down) copy_of(g, w.dw_down, D, F, F2, dw_down, D, F, F);
    if (out.count) F_TRY(launch_copies(out, e, st));
    if (grads.count) F_TRY(launch_copies(grads, ge, st));
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

}  // namespace sb

using namespace sb;

extern "C" {

sb_status sb_ffn_bytes(const sb_ffn_config* c, int32_t backward, size_t* bytes)
{
    const sb_status s = check_config(c);
    if (s != SB_OK) return s;
    if (!bytes) return set_error(SB_ERR_INVALID_ARG, "bytes is null");
    *bytes = 0;
    if (c->rows == 0) return SB_OK;
    if (even(c)) *bytes = even_bytes(c, backward != 0);
    else {
        const sb_ffn_config p = padded(c);
        Carve k{nullptr};
        carve_padded(k, &p, backward != 0);
        *bytes = k.off;
    }
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
    return even(c) ? even_forward(c, x, w_gate_up, w_down, gu, y, ws, c->f, (cudaStream_t)stream) : odd_forward(c, x, w_gate_up, w_down, gu, y, ws, (cudaStream_t)stream);
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
    return even(c) ? even_backward(c, dy, x, gu, w_gate_up, w_down, dx, dw_gate_up, dw_down, ws, c->f, (cudaStream_t)stream)
                   : odd_backward(c, dy, x, gu, w_gate_up, w_down, dx, dw_gate_up, dw_down, ws, (cudaStream_t)stream);
}

}  // extern "C"
