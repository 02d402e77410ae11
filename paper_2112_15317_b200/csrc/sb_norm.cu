// Norms before and after a residual block, fused with the block's gate and the residual scale, forward and backward.
//
//   y = s * x + g * (wpost * N(f)),   n = wpre * N(y)          N(v) = (v - mean) * inv,  inv = 1 / sqrt(mean((v - mean)^2) + eps)
//
// (rms: mean = 0).  x is the residual, f the block's output, n the input of the next block; without f, y is x and only n is computed;
// without wpre there is no n; s and g default to one.  g has one row for rows / groups consecutive rows.
//
// Backward, with hats for the normalised vectors, dz = wpre * dn and q = g * wpost:
//   d  = dy + inv_y (dz - mean(dz) - yhat mean(dz yhat))                   gradient of y
//   dx = s * d,   df = inv_f (q d - mean(q d) - fhat mean(q d fhat))
//   dwpre = sum dn yhat,  dwpost = sum g d fhat,  dg = sum over the group of d wpost fhat,  ds = sum d x
// y is computed again from x and f (nothing but four floats a row is kept from the forward pass).  mean(q d) and mean(q d fhat) are linear in
// the two means in d, so that all sums of a row are taken in one round: with e = dy + inv_y dz,
//   sum q d fhat = sum q e fhat - inv_y (mean(dz) sum q fhat + mean(dz yhat) sum q yhat fhat), and the same without fhat.
//
// What bounds it: HBM, each activation read or written once.  A CTA takes consecutive rows, a thread the same columns of each, so that the
// vectors stay in registers and the gradients of the vectors are summed in registers; a CTA's sums go to scratch and a second kernel
// adds them in order (no atomics: the same bits every time).  Row chunks are whole groups, or whole parts of one group.
#include "../../include/splitbrain.h"
#include "sb_internal.h"
#include "sb_norm.h"

#include <cmath>

namespace sb {

namespace {

constexpr int MAX_D = 16384, MAX_THREADS = 512;

struct NormParams {
    const void *x, *f, *dy, *dn;
    const float *w_pre, *w_post, *gate, *scale;
    void *y, *n, *dx, *df;
    float* stats;                 // [rows][4]: mean and inv of f, mean and inv of y
    float *part, *gate_out;       // backward: [chunk][3][d] sums of dwpre, dwpost, ds; [groups or chunks][d] of dg
    int64_t rows, per_group, chunk;      // rows of a gate; rows of a CTA's turn
    int chunks_per_group;         // > 1: a group's rows fall to that many turns (chunk of them each, the last one fewer)
    int64_t turns;
    int d, relu_x;                // relu_x: dx is zero where x <= 0 (x is the output of a ReLU layer)
    float eps, rd;                // rd = 1 / d
};

template <typename T> __device__ __forceinline__ float one(T v);
template <> __device__ __forceinline__ float one<float>(float v) { return v; }
template <> __device__ __forceinline__ float one<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T to(float v);
template <> __device__ __forceinline__ float to<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 to<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Eight columns of thread t's piece c.  VEC: consecutive ones, 16-byte accesses; otherwise blockDim.x apart.
template <bool VEC> __device__ __forceinline__ int column(int c, int j)
{
    return VEC ? (c * (int)blockDim.x + (int)threadIdx.x) * 8 + j : (c * 8 + j) * (int)blockDim.x + (int)threadIdx.x;
}
template <bool VEC> __device__ __forceinline__ void get(const float* p, int c, int d, float (&o)[8])
{
    if (VEC) {
        const int i = column<true>(c, 0);
        if (i < d) {
            const float4 a = *(const float4*)(p + i), b = *(const float4*)(p + i + 4);
            o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w; o[4] = b.x; o[5] = b.y; o[6] = b.z; o[7] = b.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = 0.f;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) { const int i = column<false>(c, j); o[j] = i < d ? p[i] : 0.f; }
}
template <bool VEC> __device__ __forceinline__ void get(const __nv_bfloat16* p, int c, int d, float (&o)[8])
{
    if (VEC) {
        const int i = column<true>(c, 0);
        uint4 a = make_uint4(0u, 0u, 0u, 0u);
        if (i < d) a = *(const uint4*)(p + i);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { o[2 * j] = __uint_as_float(w[j] << 16); o[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) { const int i = column<false>(c, j); o[j] = i < d ? __bfloat162float(p[i]) : 0.f; }
}
template <bool VEC> __device__ __forceinline__ void put(float* p, int c, int d, const float (&v)[8])
{
    if (VEC) {
        const int i = column<true>(c, 0);
        if (i < d) { *(float4*)(p + i) = make_float4(v[0], v[1], v[2], v[3]); *(float4*)(p + i + 4) = make_float4(v[4], v[5], v[6], v[7]); }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) { const int i = column<false>(c, j); if (i < d) p[i] = v[j]; }
}
template <bool VEC> __device__ __forceinline__ void put(__nv_bfloat16* p, int c, int d, const float (&v)[8])
{
    if (VEC) {
        const int i = column<true>(c, 0);
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) { const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]); w[j] = *(const uint32_t*)&b; }
        if (i < d) *(uint4*)(p + i) = make_uint4(w[0], w[1], w[2], w[3]);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) { const int i = column<false>(c, j); if (i < d) p[i] = __float2bfloat16_rn(v[j]); }
}
template <bool VEC> __device__ __forceinline__ void get_or_one(const float* p, int c, int d, float (&o)[8])
{
    if (p) get<VEC>(p, c, d, o);
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = 1.f;
    }
}

// Sums of K values over the block; every thread gets them.  The two halves of `buf` ([2][K][16]) are used in turn, so that one barrier a
// call is enough.
template <int K>
__device__ __forceinline__ void block_sum(float (&v)[K], float* buf, int& turn)
{
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
    float* b = buf + turn * (K * 16);
    turn ^= 1;
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    }
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) b[k * 16 + warp] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float s = lane < warps ? b[k * 16 + lane] : 0.f;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        v[k] = __shfl_sync(0xffffffffu, s, 0);
    }
}

// mean and inv of a row held in registers (columns at or beyond d are zero)
template <int V, bool VEC, bool LAYER>
__device__ __forceinline__ void row_stats(const float (&v)[V][8], const NormParams& p, float* buf, int& turn, float& mean, float& inv)
{
    mean = 0.f;
    if (LAYER) {
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < V; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] += v[c][j];
        block_sum<1>(s, buf, turn);
        mean = s[0] * p.rd;
    }
    float s[1] = {0.f};
#pragma unroll
    for (int c = 0; c < V; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float t = LAYER ? (column<VEC>(c, j) < p.d ? v[c][j] - mean : 0.f) : v[c][j];
            s[0] += t * t;
        }
    block_sum<1>(s, buf, turn);
    inv = 1.0f / sqrtf(s[0] * p.rd + p.eps);
}

template <typename T, int V, bool VEC, bool LAYER>
__global__ void __launch_bounds__(MAX_THREADS)
norm_forward_kernel(const NormParams p)
{
    pdl_prologue();
    __shared__ float buf[32];
    int turn = 0;
    const int d = p.d;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        float y[V][8];
#pragma unroll
        for (int c = 0; c < V; ++c) get<VEC>((const T*)p.x + row * d, c, d, y[c]);
        float st[4] = {0.f, 0.f, 0.f, 0.f};
        if (p.f) {
            float f[V][8];
#pragma unroll
            for (int c = 0; c < V; ++c) get<VEC>((const T*)p.f + row * d, c, d, f[c]);
            if (p.w_post) row_stats<V, VEC, LAYER>(f, p, buf, turn, st[0], st[1]);
            const float* gate = p.gate ? p.gate + row / p.per_group * d : nullptr;
#pragma unroll
            for (int c = 0; c < V; ++c) {
                float s[8], w[8], g[8];
                get_or_one<VEC>(p.scale, c, d, s);
                get_or_one<VEC>(p.w_post, c, d, w);
                get_or_one<VEC>(gate, c, d, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float h = p.w_post ? (f[c][j] - st[0]) * st[1] : f[c][j];
                    y[c][j] = s[j] * y[c][j] + g[j] * (w[j] * h);
                    if (column<VEC>(c, j) >= d) y[c][j] = 0.f;
                }
                if (p.y) put<VEC>((T*)p.y + row * d, c, d, y[c]);
            }
        }
        if (p.w_pre) {
            row_stats<V, VEC, LAYER>(y, p, buf, turn, st[2], st[3]);
#pragma unroll
            for (int c = 0; c < V; ++c) {
                float w[8], o[8];
                get<VEC>(p.w_pre, c, d, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = w[j] * ((y[c][j] - st[2]) * st[3]);
                put<VEC>((T*)p.n + row * d, c, d, o);
            }
        }
        if (p.stats && threadIdx.x == 0) *(float4*)(p.stats + row * 4) = make_float4(st[0], st[1], st[2], st[3]);
    }
}

// Rows of turn t: [lo, hi); the group they begin in.
__device__ __forceinline__ void turn_rows(const NormParams& p, int64_t t, int64_t& lo, int64_t& hi)
{
    if (p.chunks_per_group > 1) {
        const int64_t g = t / p.chunks_per_group, k = t - g * p.chunks_per_group, end = (g + 1) * p.per_group;
        lo = g * p.per_group + k * p.chunk;
        hi = lo + p.chunk < end ? lo + p.chunk : end;
        if (lo > end) lo = end;
    } else {
        lo = t * p.chunk;
        hi = lo + p.chunk < p.rows ? lo + p.chunk : p.rows;
    }
}

template <typename T, int V, bool VEC, bool LAYER>
__global__ void __launch_bounds__(MAX_THREADS)
norm_backward_kernel(const NormParams p)
{
    pdl_prologue();
    constexpr int K = LAYER ? 8 : 3;
    __shared__ float buf[2 * K * 16];
    int turn = 0;
    const int d = p.d;
    float a_pre[V][8], a_post[V][8], a_scale[V][8], a_gate[V][8];
    auto clear = [&](float (&a)[V][8]) {
#pragma unroll
        for (int c = 0; c < V; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) a[c][j] = 0.f;
    };
    clear(a_pre); clear(a_post); clear(a_scale); clear(a_gate);
    for (int64_t t = blockIdx.x; t < p.turns; t += gridDim.x) {
        int64_t lo, hi;
        turn_rows(p, t, lo, hi);
        for (int64_t row = lo; row < hi; ++row) {
            const float4 st = *(const float4*)(p.stats + row * 4);
            const float* gate = p.gate ? p.gate + row / p.per_group * d : nullptr;
            float x[V][8], fh[V][8], yh[V][8], dz[V][8], e[V][8];
            float s[K];
#pragma unroll
            for (int k = 0; k < K; ++k) s[k] = 0.f;
#pragma unroll
            for (int c = 0; c < V; ++c) {
                float sc[8], wp[8], g[8], w[8];
                get<VEC>((const T*)p.x + row * d, c, d, x[c]);
                get_or_one<VEC>(p.scale, c, d, sc);
                if (p.dy) get<VEC>((const T*)p.dy + row * d, c, d, e[c]);
                else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) e[c][j] = 0.f;
                }
                if (p.f) {
                    get<VEC>((const T*)p.f + row * d, c, d, fh[c]);
                    get_or_one<VEC>(p.w_post, c, d, wp);
                    get_or_one<VEC>(gate, c, d, g);
                }
                if (p.dn) { get<VEC>((const T*)p.dn + row * d, c, d, dz[c]); get<VEC>(p.w_pre, c, d, w); }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool in = column<VEC>(c, j) < d;
                    float y = p.f ? sc[j] * x[c][j] : x[c][j], q = 0.f;
                    if (p.f) {
                        if (p.w_post) fh[c][j] = (fh[c][j] - st.x) * st.y;
                        q = g[j] * wp[j];
                        y += g[j] * (wp[j] * fh[c][j]);
                    } else fh[c][j] = 0.f;
                    yh[c][j] = 0.f;
                    if (p.dn) {
                        yh[c][j] = (y - st.z) * st.w;
                        const float z = w[j] * dz[c][j];
                        if (in) a_pre[c][j] += dz[c][j] * yh[c][j];
                        dz[c][j] = z;
                        e[c][j] += st.w * z;
                        if (in) { s[0] += z * yh[c][j]; if (LAYER) s[3] += z; }
                    }
                    if (p.w_post && in) {
                        const float qf = q * fh[c][j];
                        s[1] += qf * e[c][j];
                        s[2] += qf * yh[c][j];
                        if (LAYER) { s[4] += qf; s[5] += q * e[c][j]; s[6] += q * yh[c][j]; s[7] += q; }
                    }
                }
            }
            if (p.dn || p.w_post) block_sum<K>(s, buf, turn);
            // the means in d, then those in df
            const float c1 = p.dn ? s[0] * p.rd : 0.f, c0 = LAYER && p.dn ? s[LAYER ? 3 : 0] * p.rd : 0.f, iy = p.dn ? st.w : 0.f;
            const float f1 = (s[1] - iy * (c0 * (LAYER ? s[LAYER ? 4 : 0] : 0.f) + c1 * s[2])) * p.rd;
            const float f0 = LAYER ? (s[LAYER ? 5 : 0] - iy * (c0 * s[LAYER ? 7 : 0] + c1 * s[LAYER ? 6 : 0])) * p.rd : 0.f;
#pragma unroll
            for (int c = 0; c < V; ++c) {
                float sc[8], wp[8], g[8], o[8];
                get_or_one<VEC>(p.f ? p.scale : nullptr, c, d, sc);
                if (p.f) { get_or_one<VEC>(p.w_post, c, d, wp); get_or_one<VEC>(gate, c, d, g); }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float D = e[c][j] - iy * (c0 + yh[c][j] * c1);
                    e[c][j] = D;
                    a_scale[c][j] += D * x[c][j];
                    o[j] = p.relu_x && !(x[c][j] > 0.f) ? 0.f : sc[j] * D;
                }
                if (p.dx) put<VEC>((T*)p.dx + row * d, c, d, o);
                if (p.f) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float D = e[c][j], h = fh[c][j];
                        a_post[c][j] += g[j] * D * h;
                        a_gate[c][j] += D * (wp[j] * h);
                        o[j] = p.w_post ? st.y * (g[j] * wp[j] * D - f0 - h * f1) : g[j] * D;
                    }
                    if (p.df) put<VEC>((T*)p.df + row * d, c, d, o);
                }
            }
            if (p.gate_out && p.chunks_per_group == 1 && (row + 1) % p.per_group == 0) {
#pragma unroll
                for (int c = 0; c < V; ++c) put<VEC>(p.gate_out + row / p.per_group * d, c, d, a_gate[c]);
                clear(a_gate);
            }
        }
        if (p.gate_out && p.chunks_per_group > 1) {
#pragma unroll
            for (int c = 0; c < V; ++c) put<VEC>(p.gate_out + t * d, c, d, a_gate[c]);
            clear(a_gate);
        }
    }
    if (p.part) {
        float* out = p.part + (int64_t)blockIdx.x * 3 * d;
#pragma unroll
        for (int c = 0; c < V; ++c) {
            put<VEC>(out, c, d, a_pre[c]);
            put<VEC>(out + d, c, d, a_post[c]);
            put<VEC>(out + 2 * (int64_t)d, c, d, a_scale[c]);
        }
    }
}

// out[b][col] = sum over k < n, in order within eighths and then over those, of part[(b * n + k) * stride + col]
struct SumArgs { const float* part; float* out[3]; int64_t n, stride, batch; int d; };
__global__ void __launch_bounds__(256) norm_sum_kernel(const SumArgs a)
{
    pdl_prologue();
    __shared__ float s[8][32];
    const int lane = threadIdx.x % 32, w = threadIdx.x / 32, which = blockIdx.y;
    float* out = a.out[which];
    if (!out) return;
    const int col = blockIdx.x * 32 + lane;
    const int64_t per = (a.n + 7) / 8, k0 = w * per, k1 = k0 + per < a.n ? k0 + per : a.n;
    for (int64_t b = blockIdx.z; b < a.batch; b += gridDim.z) {
        const float* p = a.part + b * a.n * a.stride + (int64_t)which * a.d + col;
        float v = 0.f;
        if (col < a.d) {
#pragma unroll 4
            for (int64_t k = k0; k < k1; ++k) v += p[k * a.stride];
        }
        s[w][lane] = v;
        __syncthreads();
        if (w == 0 && col < a.d) {
            for (int i = 1; i < 8; ++i) v += s[i][lane];
            out[b * a.d + col] = v;
        }
        __syncthreads();
    }
}

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

int threads_of(int d)
{
    const int t = (d + 255) / 256 * 32;
    return t < MAX_THREADS ? t : MAX_THREADS;
}
int pieces_of(int d) { return d <= MAX_THREADS * 8 ? 1 : d <= MAX_THREADS * 16 ? 2 : 4; }

// How the rows fall to CTAs in the backward pass: about `want` turns, each of whole groups or a part of one.
struct Turns { int64_t chunk, turns; int per_group; };
Turns turns_of(int64_t rows, int64_t groups, int want)
{
    Turns t{};
    const int64_t per = groups > 0 ? rows / groups : rows;
    const int64_t rows_each = (rows + want - 1) / want;
    t.per_group = 1;
    if (groups > 0 && per > rows_each) {          // parts of a group
        const int64_t parts = (per + rows_each - 1) / rows_each;
        t.chunk = (per + parts - 1) / parts;
        t.per_group = (int)((per + t.chunk - 1) / t.chunk);
        t.turns = groups * t.per_group;
    } else {
        const int64_t unit = groups > 0 ? per : 1, units = rows / unit;
        t.chunk = (units + want - 1) / want * unit;
        t.turns = (rows + t.chunk - 1) / t.chunk;
    }
    return t;
}
// CTAs of the backward kernel: as many as are resident at once
int backward_ctas(int d) { return 148 * (threads_of(d) <= 128 ? 4 : threads_of(d) <= 256 ? 2 : 1); }
size_t part_floats(const sb_norm_config* c)
{
    const Turns t = turns_of(c->rows, c->groups, backward_ctas(c->d));
    const int64_t ctas = t.turns < backward_ctas(c->d) ? t.turns : backward_ctas(c->d);
    return (size_t)ctas * 3 * c->d + (t.per_group > 1 ? (size_t)t.turns * c->d : 0) + 64;
}

template <template <typename, int, bool, bool> class Run, typename T, int V, bool VEC, typename... A>
cudaError_t pick_kind(bool layer, A&&... a) { return layer ? Run<T, V, VEC, true>::go(a...) : Run<T, V, VEC, false>::go(a...); }
template <template <typename, int, bool, bool> class Run, typename T, int V, typename... A>
cudaError_t pick_vec(bool vec, bool layer, A&&... a) { return vec ? pick_kind<Run, T, V, true>(layer, a...) : pick_kind<Run, T, V, false>(layer, a...); }
template <template <typename, int, bool, bool> class Run, typename T, typename... A>
cudaError_t pick_pieces(int v, bool vec, bool layer, A&&... a)
{
    return v == 1 ? pick_vec<Run, T, 1>(vec, layer, a...) : v == 2 ? pick_vec<Run, T, 2>(vec, layer, a...) : pick_vec<Run, T, 4>(vec, layer, a...);
}
template <template <typename, int, bool, bool> class Run, typename... A>
cudaError_t pick(bool bf16, int v, bool vec, bool layer, A&&... a)
{
    return bf16 ? pick_pieces<Run, __nv_bfloat16>(v, vec, layer, a...) : pick_pieces<Run, float>(v, vec, layer, a...);
}
template <typename T, int V, bool VEC, bool LAYER> struct Forward {
    static cudaError_t go(const NormParams& p, int64_t ctas, cudaStream_t st)
    {
        return pdl_launch(norm_forward_kernel<T, V, VEC, LAYER>, dim3((unsigned)ctas), dim3(threads_of(p.d)), 0, st, p);
    }
};
template <typename T, int V, bool VEC, bool LAYER> struct Backward {
    static cudaError_t go(const NormParams& p, int64_t ctas, cudaStream_t st)
    {
        return pdl_launch(norm_backward_kernel<T, V, VEC, LAYER>, dim3((unsigned)ctas), dim3(threads_of(p.d)), 0, st, p);
    }
};

sb_status check_config(const sb_norm_config* c)
{
    if (!c) return set_error(SB_ERR_INVALID_ARG, "null config");
    if (c->precision != SB_FP32 && c->precision != SB_BF16) return set_error(SB_ERR_INVALID_ARG, "precision must be SB_FP32 or SB_BF16");
    if (c->kind != SB_NORM_RMS && c->kind != SB_NORM_LAYER) return set_error(SB_ERR_INVALID_ARG, "unknown norm kind %d", c->kind);
    if (c->rows < 0 || c->d < 1) return set_error(SB_ERR_SHAPE, "rows must not be negative and d must be positive");
    if (c->d > MAX_D) return set_error(SB_ERR_UNSUPPORTED, "d = %d: rows of at most %d columns", c->d, MAX_D);
    if (c->groups < 0 || (c->groups > 0 && c->rows % c->groups != 0)) return set_error(SB_ERR_SHAPE, "%lld rows are not %lld groups of the same size", (long long)c->rows, (long long)c->groups);
    if (!(c->eps >= 0.f) || std::isinf(c->eps)) return set_error(SB_ERR_INVALID_ARG, "eps must be finite and not negative");
    return SB_OK;
}
NormParams params_of(const sb_norm_config* c, const void* x, const float* w_pre, const void* f, const float* w_post, const float* gate, const float* scale)
{
    NormParams p{};
    p.x = x; p.f = f; p.w_pre = w_pre; p.w_post = w_post; p.gate = gate; p.scale = scale;
    p.rows = c->rows; p.d = c->d; p.eps = c->eps; p.rd = (float)(1.0 / c->d);
    p.per_group = c->groups > 0 ? c->rows / c->groups : (c->rows > 0 ? c->rows : 1);
    p.chunks_per_group = 1;
    return p;
}
sb_status check_vectors(const sb_norm_config* c, const void* f, const float* w_post, const float* gate, const float* scale)
{
    if (!f && (w_post || gate || scale)) return set_error(SB_ERR_INVALID_ARG, "w_post, gate and scale belong to f, which is null");
    if ((gate != nullptr) != (c->groups > 0)) return set_error(SB_ERR_INVALID_ARG, "a gate needs groups > 0, and groups a gate");
    return SB_OK;
}
// 16-byte accesses: rows of whole pieces, every pointer aligned
template <typename... P> bool vec_ok(int d, P... p) { return d % 8 == 0 && (aligned(p, 16) && ...); }

}  // namespace

sb_status norm_backward(const sb_norm_config* c, const void* dy, const void* dn, const float* stats, const void* x, const float* w_pre, const void* f,
                        const float* w_post, const float* gate, const float* scale, void* dx, void* df, float* dw_pre, float* dw_post, float* dgate,
                        float* dscale, void* ws, size_t ws_bytes, bool relu_x, cudaStream_t st)
{
    sb_status s = check_config(c);
    if (s != SB_OK) return s;
    float* sums[3] = {dw_pre, dw_post, dscale};
    const bool want = dw_pre || dw_post || dscale;
    if (c->rows == 0) {           // empty sums
        for (float* o : sums)
            if (o) { const cudaError_t r = cudaMemsetAsync(o, 0, (size_t)c->d * 4, st); if (r != cudaSuccess) return set_error(SB_ERR_CUDA, "%s", cudaGetErrorString(r)); }
        if (dgate) { const cudaError_t r = cudaMemsetAsync(dgate, 0, (size_t)c->groups * c->d * 4, st); if (r != cudaSuccess) return set_error(SB_ERR_CUDA, "%s", cudaGetErrorString(r)); }
        return SB_OK;
    }
    if ((s = check_vectors(c, f, w_post, gate, scale)) != SB_OK) return s;
    if (!dy && !dn) return set_error(SB_ERR_INVALID_ARG, "dy and dn are both null");
    if (dn && !w_pre) return set_error(SB_ERR_INVALID_ARG, "dn needs w_pre");
    if (dw_pre && !dn) return set_error(SB_ERR_INVALID_ARG, "dw_pre needs dn");
    if (df && !f) return set_error(SB_ERR_INVALID_ARG, "df needs f");
    if ((dw_post && !w_post) || (dgate && !gate) || (dscale && !scale)) return set_error(SB_ERR_INVALID_ARG, "a gradient of a vector that is null");
    const size_t e = c->precision == SB_BF16 ? 2 : 4;
    if (!aligned(x, e) || !aligned(dy, e) || !aligned(dn, e) || !aligned(f, e) || !aligned(dx, e) || !aligned(df, e)) return set_error(SB_ERR_INVALID_ARG, "a matrix is misaligned");
    if (!x || !stats || !aligned(stats, 16)) return set_error(SB_ERR_INVALID_ARG, "x or stats is null, or stats not 16-byte aligned");
    const size_t floats = part_floats(c);
    if (!ws || !aligned(ws, 16) || ws_bytes < floats * 4) return set_error(SB_ERR_ARENA_TOO_SMALL, "the workspace must be 16-byte aligned and hold %zu bytes (got %zu)", floats * 4, ws_bytes);
    NormParams p = params_of(c, x, w_pre, f, w_post, gate, scale);
    const Turns t = turns_of(c->rows, c->groups, backward_ctas(c->d));
    const int64_t ctas = t.turns < backward_ctas(c->d) ? t.turns : backward_ctas(c->d);
    p.dy = dy; p.dn = dn; p.dx = dx; p.df = df; p.stats = (float*)stats; p.relu_x = relu_x;
    p.chunk = t.chunk; p.turns = t.turns; p.chunks_per_group = t.per_group;
    float* part = (float*)ws;
    float* gate_part = part + ((size_t)ctas * 3 * c->d + 15) / 16 * 16;
    p.part = want ? part : nullptr;
    p.gate_out = !dgate ? nullptr : t.per_group > 1 ? gate_part : dgate;
    const bool vec = vec_ok(c->d, x, f, dy, dn, dx, df, w_pre, w_post, gate, scale, dgate);
    cudaError_t r = pick<Backward>(c->precision == SB_BF16, pieces_of(c->d), vec, c->kind == SB_NORM_LAYER, p, ctas, st);
    const unsigned cols = (unsigned)((c->d + 31) / 32);
    if (r == cudaSuccess && want) {
        SumArgs a{part, {dw_pre, dw_post, dscale}, ctas, (int64_t)3 * c->d, 1, c->d};
        r = pdl_launch(norm_sum_kernel, dim3(cols, 3, 1), dim3(256), 0, st, a);
    }
    if (r == cudaSuccess && dgate && t.per_group > 1) {
        SumArgs a{gate_part, {dgate, nullptr, nullptr}, t.per_group, (int64_t)c->d, c->groups, c->d};
        r = pdl_launch(norm_sum_kernel, dim3(cols, 1, (unsigned)(c->groups < 64 ? c->groups : 64)), dim3(256), 0, st, a);
    }
    return r == cudaSuccess ? SB_OK : set_error(SB_ERR_CUDA, "norm backward: %s", cudaGetErrorString(r));
}

}  // namespace sb

using namespace sb;

extern "C" {

sb_status sb_norm_forward(const sb_norm_config* c, const void* x, const float* w_pre, const void* f, const float* w_post, const float* gate,
                          const float* scale, void* y, void* n, float* stats, void* stream)
{
    sb_status s = check_config(c);
    if (s != SB_OK || c->rows == 0) return s;
    if ((s = check_vectors(c, f, w_post, gate, scale)) != SB_OK) return s;
    if (!f && !w_pre) return set_error(SB_ERR_INVALID_ARG, "neither f nor w_pre: there is nothing to compute");
    if ((n != nullptr) != (w_pre != nullptr)) return set_error(SB_ERR_INVALID_ARG, "n and w_pre go together");
    if (y && !f) return set_error(SB_ERR_INVALID_ARG, "y is x where f is null");
    const size_t e = c->precision == SB_BF16 ? 2 : 4;
    if (!aligned(x, e) || !aligned(f, e) || !aligned(y, e) || !aligned(n, e) || !aligned(stats, 16)) return set_error(SB_ERR_INVALID_ARG, "a matrix or stats is misaligned");
    if (!x) return set_error(SB_ERR_INVALID_ARG, "x is null");
    NormParams p = params_of(c, x, w_pre, f, w_post, gate, scale);
    p.y = y; p.n = n; p.stats = stats;
    const bool vec = vec_ok(c->d, x, f, y, n, w_pre, w_post, gate, scale);
    const int64_t most = 148 * (2048 / threads_of(c->d)), ctas = c->rows < most ? c->rows : most;
    const cudaError_t r = pick<Forward>(c->precision == SB_BF16, pieces_of(c->d), vec, c->kind == SB_NORM_LAYER, p, ctas, (cudaStream_t)stream);
    return r == cudaSuccess ? SB_OK : set_error(SB_ERR_CUDA, "norm forward: %s", cudaGetErrorString(r));
}

sb_status sb_norm_bytes(const sb_norm_config* c, size_t* bytes)
{
    const sb_status s = check_config(c);
    if (s != SB_OK) return s;
    if (!bytes) return set_error(SB_ERR_INVALID_ARG, "bytes is null");
    *bytes = c->rows > 0 ? part_floats(c) * 4 : 0;
    return SB_OK;
}

sb_status sb_norm_backward(const sb_norm_config* c, const void* dy, const void* dn, const float* stats, const void* x, const float* w_pre, const void* f,
                           const float* w_post, const float* gate, const float* scale, void* dx, void* df, float* dw_pre, float* dw_post, float* dgate,
                           float* dscale, void* ws, size_t ws_bytes, void* stream)
{
    return norm_backward(c, dy, dn, stats, x, w_pre, f, w_post, gate, scale, dx, df, dw_pre, dw_post, dgate, dscale, ws, ws_bytes, false, (cudaStream_t)stream);
}

}  // extern "C"
