// AdamW over a list of tensors in one kernel, moments in 32 or in 8 bits.
//
//   m <- b1 m + (1 - b1) g       v <- b2 v + (1 - b2) g^2
//   p <- (1 - lr wd) p - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps)          (and, where wanted, p's bf16 copy)
//
// What bounds it: HBM.  A parameter moves 28 bytes with float moments and gradients, 14 with 8-bit moments and bf16 gradients (plus 2 for
// the bf16 copy).  138 M parameters (VGG-16, 32 tensors) with their copy take 656 us (6.3 TB/s) and 429 us (5.2): the second moves half as much for some 60
// instructions an element, so that a warp fetches its next block before it works on one (446 us without).  A warp walks blocks of 256 elements, eight consecutive ones a lane, which is also the block that shares a scale of the
// 8-bit states: its largest magnitudes are one redux instruction, and nothing crosses the warp otherwise.  The tensors' pointers
// travel as kernel parameters, so that a call needs no table in device memory and can be captured into a graph as it is.
//
// 8-bit moments.  The scale of a block is a power of two, so that scaling rounds nothing and the codes depend on the moments alone.
//   m: e4m3 of m / (scale = 2^(floor(log2 max) - 7)), to nearest even.  A step moves m by a tenth, more than half a code.
//   v: five bits of exponent and three of mantissa, no sign, of v / (scale = 2^floor(log2 max)).  A step moves v by a thousandth, which
//      rounding to nearest would never show: it is rounded up or down by chance, with 16 random bits for each element from
//      Philox-4x32-10 (counter = {element / 8, tensor, step}, key = seed), so that its expectation is the unrounded value.
//      Held in the bits of a float: value * 2^-97 has the code in its bits 20 .. 27, subnormal numbers included.
// A moment that is not finite becomes a code of its own (0x7F, 255) and leaves its block's scale alone.
// The moments are rounded in the order the formulas above are written in, without fused multiply-adds: with the codes' coarse
// grids one m in a hundred lies exactly between two codes, and falls to the same side in every implementation that keeps the order.
#include "../../include/splitbrain.h"
#include "sb_f32x2.cuh"
#include "sb_internal.h"

#include <cuda_fp8.h>

#include <cmath>
#include <type_traits>

namespace sb {

namespace {

constexpr int ADAMW_THREADS = 256, QBLOCK = 256;

struct Entry {
    float* p;
    const void* g;
    void *m, *v;
    float *ms, *vs;
    __nv_bfloat16* shadow;
    int64_t n, first;        // elements; blocks of all tensors before this one
    int vec, index;          // every pointer suits wide accesses (see load8); place in the caller's list
};
template <int N> struct AdamwArgs {
    Entry e[N];
    int count;
    int64_t blocks;
    float b1, c1, b2, c2, decay, rate, rs2, eps;
    double beta1, beta2, lr, wd;
    const int64_t* dev_step;
    const float* dev_lr;
    uint32_t key0, key1, step;
};

__device__ __forceinline__ uint4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint32_t h0 = __umulhi(0xD2511F53u, c0), l0 = 0xD2511F53u * c0, h1 = __umulhi(0xCD9E8D57u, c2), l1 = 0xCD9E8D57u * c2;
        c0 = h1 ^ c1 ^ k0; c1 = l1; c2 = h0 ^ c3 ^ k1; c3 = l0;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// Eight consecutive elements from i on, n of the tensor in all: one access where the whole run is there and aligned (floats: 32 bytes; two of 16 bytes for
// each take 672 us where this takes 656, 138 M parameters with a bf16 copy).
__device__ __forceinline__ void load8(const float* p, int64_t i, int64_t n, bool vec, float (&o)[8])
{
    if (vec && i + 8 <= n) {
        asm volatile("ld.global.L1::no_allocate.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(o[0]), "=f"(o[1]), "=f"(o[2]), "=f"(o[3]), "=f"(o[4]), "=f"(o[5]), "=f"(o[6]), "=f"(o[7]) : "l"(p + i) : "memory");
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = i + j < n ? p[i + j] : 0.f;
}
// Gradients as they lie in memory, and as floats.
template <typename G> struct RawRun;
template <> struct RawRun<float> {
    float v[8];
    __device__ __forceinline__ void load(const float* p, int64_t i, int64_t n, bool vec) { load8(p, i, n, vec, v); }
    __device__ __forceinline__ float at(int j) const { return v[j]; }
};
template <> struct RawRun<__nv_bfloat16> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int64_t i, int64_t n, bool vec)
    {
        if (vec && i + 8 <= n) {
            const uint4 a = __ldcs((const uint4*)(p + i));
            w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
            return;
        }
        const uint16_t* u = (const uint16_t*)p;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = (i + 2 * j < n ? (uint32_t)u[i + 2 * j] : 0u) | (i + 2 * j + 1 < n ? (uint32_t)u[i + 2 * j + 1] << 16 : 0u);
    }
    __device__ __forceinline__ float at(int j) const { return __uint_as_float(j % 2 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16); }
};
__device__ __forceinline__ void store8(float* p, int64_t i, int64_t n, bool vec, const float (&v)[8])
{
    if (vec && i + 8 <= n) {
        asm volatile("st.global.L1::no_allocate.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(p + i), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (i + j < n) p[i + j] = v[j];
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, int64_t i, int64_t n, bool vec, const float (&v)[8])
{
    if (vec && i + 8 <= n) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) { const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]); w[j] = *(const uint32_t*)&b; }
        __stcs((uint4*)(p + i), make_uint4(w[0], w[1], w[2], w[3]));
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (i + j < n) p[i + j] = __float2bfloat16_rn(v[j]);
}
__device__ __forceinline__ void load_codes(const uint8_t* p, int64_t i, int64_t n, bool vec, uint32_t (&o)[2])
{
    if (vec && i + 8 <= n) {
        const uint2 a = __ldcs((const uint2*)(p + i));
        o[0] = a.x; o[1] = a.y;
        return;
    }
    o[0] = o[1] = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (i + j < n) o[j / 4] |= (uint32_t)p[i + j] << (8 * (j % 4));
}
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t i, int64_t n, bool vec, const uint32_t (&v)[2])
{
    if (vec && i + 8 <= n) {
        __stcs((uint2*)(p + i), make_uint2(v[0], v[1]));
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (i + j < n) p[i + j] = (uint8_t)(v[j / 4] >> (8 * (j % 4)));
}

__device__ __forceinline__ void decode_m(const uint32_t (&c)[2], float scale, float (&o)[8])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(c[j / 2] >> (16 * (j % 2))), __NV_E4M3);
        const float2 f = __half22float2(*(const __half2*)&h);
        o[2 * j] = f.x * scale;
        o[2 * j + 1] = f.y * scale;
    }
}
__device__ __forceinline__ void decode_v(const uint32_t (&c)[2], float scale, float (&o)[8])
{
    // (a code of 255: a byte whose low seven bits carry into a high bit that is set)
    const bool odd = ((((c[0] & 0x7f7f7f7fu) + 0x01010101u) & c[0]) | (((c[1] & 0x7f7f7f7fu) + 0x01010101u) & c[1])) & 0x80808080u;
    const F2 up = f2(0x1p97f), by = f2(scale);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t w = c[j / 2] >> (16 * (j % 2));
        const F2 v = f2(__uint_as_float((w << 20) & 0x0ff00000u), __uint_as_float((w << 12) & 0x0ff00000u)) * up * by;
        o[2 * j] = lo(v);
        o[2 * j + 1] = hi(v);
    }
    if (odd) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (((c[j / 4] >> (8 * (j % 4))) & 255u) == 255u) o[j] = __int_as_float(0x7fffffff);
    }
}
// The power of two at or below the largest finite magnitude of a warp's block, 2^-100 at least.
__device__ __forceinline__ float block_power(const float (&a)[8])
{
    uint32_t top = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t b = __float_as_uint(a[j]) & 0x7fffffffu;
        if (b < 0x7f800000u && b > top) top = b;
    }
    top = __reduce_max_sync(0xffffffffu, top) & 0x7f800000u;
    return __uint_as_float(top > 0x0d800000u ? top : 0x0d800000u);
}
__device__ __forceinline__ void encode_m(const float (&a)[8], float inv, uint32_t (&c)[2])
{
    c[0] = c[1] = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t two = __nv_cvt_float2_to_fp8x2(make_float2(a[2 * j] * inv, a[2 * j + 1] * inv), __NV_SATFINITE, __NV_E4M3);
        if (isinf(a[2 * j])) two |= 0x7fu;           // (the conversion keeps NaN, but takes infinities for the largest number)
        if (isinf(a[2 * j + 1])) two |= 0x7f00u;
        c[j / 2] |= two << (16 * (j % 2));
    }
}
__device__ __forceinline__ void encode_v(const float (&a)[8], float inv, uint4 r, uint32_t (&c)[2])
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
    c[0] = c[1] = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t half = j % 2 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu;
        uint32_t code = (__float_as_uint(a[j] * inv * 0x1p-97f) + (half << 4)) >> 20;
        code = !isfinite(a[j]) ? 255u : code < 254u ? code : 254u;
        c[j / 4] |= code << (8 * (j % 4));
    }
}

__device__ __forceinline__ float root(float x)
{
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// The bits of the largest magnitude of a warp's block (those of an infinity or more: something in it is not finite)
__device__ __forceinline__ uint32_t block_top(const float (&a)[8])
{
    uint32_t top = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(a[j]) & 0x7fffffffu);
    return __reduce_max_sync(0xffffffffu, top);
}
__device__ __forceinline__ float power_of(uint32_t top) { return __uint_as_float(max(top & 0x7f800000u, 0x0d800000u)); }
// encode_m and encode_v for blocks that are finite throughout (no code can reach 254 then: the largest number's exponent is 30)
__device__ __forceinline__ void encode_finite(const float (&m)[8], const float (&v)[8], float inv_m, float inv_v, uint4 r, uint32_t (&cm)[2], uint32_t (&cv)[2])
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
    const F2 im = f2(inv_m), iv = f2(inv_v), down = f2(0x1p-97f);
    uint32_t two[4], z[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const F2 a = f2(m[2 * j], m[2 * j + 1]) * im, b = f2(v[2 * j], v[2 * j + 1]) * iv * down;
        two[j] = __nv_cvt_float2_to_fp8x2(make_float2(lo(a), hi(a)), __NV_SATFINITE, __NV_E4M3);
        z[2 * j] = __float_as_uint(lo(b)) + ((w[j] << 4) & 0xffff0u);
        z[2 * j + 1] = __float_as_uint(hi(b)) + ((w[j] >> 12) & 0xffff0u);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        cm[h] = two[2 * h] | two[2 * h + 1] << 16;
        cv[h] = z[4 * h] >> 20 | (z[4 * h + 1] >> 20) << 8 | (z[4 * h + 2] >> 20) << 16 | (z[4 * h + 3] >> 20) << 24;
    }
}

// Warp w's block: the tensor it lies in (binary search over the tensors' first blocks), and its first element there.
template <int N>
__device__ __forceinline__ int find_entry(const AdamwArgs<N>& a, int64_t block)
{
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.e[mid].first <= block) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// What a lane reads of a block.
template <int BITS, typename G> struct Block {
    int entry;
    float p[8];
    RawRun<G> g;
    typename std::conditional<BITS == 32, float[8], uint32_t[2]>::type m, v;
    float ms, vs;
    template <int N> __device__ __forceinline__ void load(const AdamwArgs<N>& a, int64_t b, int lane)
    {
        entry = find_entry(a, b);
        const Entry& e = a.e[entry];
        const int64_t q = b - e.first, i = q * QBLOCK + lane * 8, n = e.n;
        const bool vec = e.vec != 0;
        load8(e.p, i, n, vec, p);
        g.load((const G*)e.g, i, n, vec);
        if constexpr (BITS == 32) {
            load8((const float*)e.m, i, n, vec, m);
            load8((const float*)e.v, i, n, vec, v);
        } else {
            load_codes((const uint8_t*)e.m, i, n, vec, m);
            load_codes((const uint8_t*)e.v, i, n, vec, v);
            ms = e.ms[q];
            vs = e.vs[q];
        }
    }
};

template <int N, int BITS, typename G>
__global__ void __launch_bounds__(ADAMW_THREADS)
adamw_kernel(const __grid_constant__ AdamwArgs<N> a)
{
    pdl_prologue();
    const int lane = threadIdx.x % 32;
    float decay = a.decay, rate = a.rate, rs2 = a.rs2;
    uint32_t step = a.step;
    if (a.dev_step != nullptr || a.dev_lr != nullptr) {      // (a replayed step: what changes from replay to replay lies in device memory)
        __shared__ float s_words[3];
        __shared__ uint32_t s_step;
        if (threadIdx.x == 0) {
            const double lr = a.dev_lr ? (double)*a.dev_lr : a.lr;
            const int64_t t = a.dev_step ? *a.dev_step : (int64_t)a.step;
            s_words[0] = (float)(1.0 - lr * a.wd);
            s_words[1] = (float)(lr / (1.0 - pow(a.beta1, (double)t)));
            s_words[2] = (float)(1.0 / sqrt(1.0 - pow(a.beta2, (double)t)));
            s_step = (uint32_t)t;
        }
        __syncthreads();
        decay = s_words[0]; rate = s_words[1]; rs2 = s_words[2]; step = s_step;
    }
    const int64_t warps = (int64_t)gridDim.x * (ADAMW_THREADS / 32);
    int64_t b = (int64_t)blockIdx.x * (ADAMW_THREADS / 32) + threadIdx.x / 32;
    Block<BITS, G> next;
    if (BITS == 8 && b < a.blocks) next.load(a, b, lane);
    for (; b < a.blocks; b += warps) {
        Block<BITS, G> at;
        if (BITS == 8) {
            at = next;
            if (b + warps < a.blocks) next.load(a, b + warps, lane);
        } else at.load(a, b, lane);
        const Entry& e = a.e[at.entry];
        const int64_t q = b - e.first, i = q * QBLOCK + lane * 8, n = e.n;
        const bool vec = e.vec != 0;
        float (&p)[8] = at.p;
        float m[8], v[8];
        if constexpr (BITS == 32) {
#pragma unroll
            for (int j = 0; j < 8; ++j) { m[j] = at.m[j]; v[j] = at.v[j]; }
        } else {
            decode_m(at.m, at.ms, m);
            decode_v(at.v, at.vs, v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // (not in pairs: a product and a sum of two floats at a time come out fused, rounded once)
            const float g = at.g.at(j);
            m[j] = __fadd_rn(__fmul_rn(a.b1, m[j]), __fmul_rn(a.c1, g));
            v[j] = __fadd_rn(__fmul_rn(a.b2, v[j]), __fmul_rn(__fmul_rn(a.c2, g), g));
            // (8 bits: the step by the approximations of root and quotient, 2^-21 of it, where the moments' codes leave 2^-5.  138 M parameters without a copy,
            // float gradients: 395 us, 423 with the exact ones.  Float moments: exact, 599 us, 596 with the approximations.)
            p[j] = p[j] * decay - rate * (BITS == 32 ? __fdiv_rn(m[j], __fsqrt_rn(v[j]) * rs2 + a.eps) : __fdividef(m[j], root(v[j]) * rs2 + a.eps));
        }
        store8(e.p, i, n, vec, p);
        if (e.shadow) store8(e.shadow, i, n, vec, p);
        if (BITS == 32) {
            store8((float*)e.m, i, n, vec, m);
            store8((float*)e.v, i, n, vec, v);
        } else {
            // (elements behind the tensor's end are zero)
            const uint64_t eight = (uint64_t)(i / 8);
            const uint4 r = philox((uint32_t)eight, (uint32_t)(eight >> 32), (uint32_t)e.index, step, a.key0, a.key1);
            const uint32_t top_m = block_top(m), top_v = block_top(v);
            uint32_t cm[2], cv[2];
            float ms, vs;
            if (top_m < 0x7f800000u && top_v < 0x7f800000u) {
                ms = power_of(top_m) * 0x1p-7f; vs = power_of(top_v);
                encode_finite(m, v, 1.0f / ms, 1.0f / vs, r, cm, cv);
            } else {
                ms = block_power(m) * 0x1p-7f; vs = block_power(v);
                encode_m(m, 1.0f / ms, cm);
                encode_v(v, 1.0f / vs, r, cv);
            }
            store_codes((uint8_t*)e.m, i, n, vec, cm);
            store_codes((uint8_t*)e.v, i, n, vec, cv);
            __syncwarp();                                    // every lane has read the old scales
            if (lane == 0) { e.ms[q] = ms; e.vs[q] = vs; }
        }
    }
}

// What the 8-bit moments stand for, as bf16 (a code of four significant bits times a power of two fits).
template <int N>
__global__ void __launch_bounds__(ADAMW_THREADS)
adamw_moments_kernel(const __grid_constant__ AdamwArgs<N> a)
{
    pdl_prologue();
    const int lane = threadIdx.x % 32;
    const int64_t warps = (int64_t)gridDim.x * (ADAMW_THREADS / 32);
    for (int64_t b = (int64_t)blockIdx.x * (ADAMW_THREADS / 32) + threadIdx.x / 32; b < a.blocks; b += warps) {
        const Entry& e = a.e[find_entry(a, b)];
        const int64_t q = b - e.first, i = q * QBLOCK + lane * 8, n = e.n;
        const bool vec = e.vec != 0;
        uint32_t c[2];
        float f[8];
        load_codes((const uint8_t*)e.m, i, n, vec, c);
        decode_m(c, e.ms[q], f);
        store8((__nv_bfloat16*)e.p, i, n, vec, f);           // (the outputs travel in the places of parameter and copy)
        load_codes((const uint8_t*)e.v, i, n, vec, c);
        decode_v(c, e.vs[q], f);
        store8(e.shadow, i, n, vec, f);
    }
}

bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

template <int N>
cudaError_t launch_list(AdamwArgs<N>& a, int bits, bool bf16_grad, bool moments, cudaStream_t st)
{
    const int64_t want = (a.blocks + ADAMW_THREADS / 32 - 1) / (ADAMW_THREADS / 32);
    // (138 M parameters with a bf16 copy, CTAs an SM: 8-bit moments, of which three fit at a time, 8: 444 us, 12: 429, 16: 427; float ones 678, 674, 656)
    const int64_t most = 148 * (bits == 8 && !moments ? 12 : 16);
    const dim3 grid((unsigned)(want < most ? want : most)), block(ADAMW_THREADS);
    if (moments) return pdl_launch(adamw_moments_kernel<N>, grid, block, 0, st, a);
    if (bits == 32) return bf16_grad ? pdl_launch(adamw_kernel<N, 32, __nv_bfloat16>, grid, block, 0, st, a) : pdl_launch(adamw_kernel<N, 32, float>, grid, block, 0, st, a);
    return bf16_grad ? pdl_launch(adamw_kernel<N, 8, __nv_bfloat16>, grid, block, 0, st, a) : pdl_launch(adamw_kernel<N, 8, float>, grid, block, 0, st, a);
}

// The list in as many launches as it takes: up to 32 tensors as 2.4 KB of parameters, more as up to 28 KB (350 at a time).
template <int N, typename Fill>
sb_status run_list(const sb_adamw_tensor* list, int from, int to, int bits, bool bf16_grad, bool moments, cudaStream_t st, Fill fill)
{
    static thread_local AdamwArgs<N> a;
    a = AdamwArgs<N>{};
    fill(a);
    for (int i = from; i < to; ++i) {
        if (list[i].n == 0) continue;
        const sb_adamw_tensor& t = list[i];
        Entry& e = a.e[a.count++];
        e.p = t.param; e.g = t.grad; e.m = t.m; e.v = t.v; e.ms = t.m_scale; e.vs = t.v_scale; e.shadow = (__nv_bfloat16*)t.shadow;
        e.n = t.n; e.first = a.blocks; e.index = i;
        e.vec = aligned(t.param, moments ? 16 : 32) && aligned(t.grad, bf16_grad ? 16 : 32) && aligned(t.m, bits == 32 ? 32 : 8) && aligned(t.v, bits == 32 ? 32 : 8) && aligned(t.shadow, 16);
        a.blocks += (t.n + QBLOCK - 1) / QBLOCK;
    }
    if (a.count == 0) return SB_OK;
    const cudaError_t e = launch_list(a, bits, bf16_grad, moments, st);
    return e == cudaSuccess ? SB_OK : set_error(SB_ERR_CUDA, "adamw: %s", cudaGetErrorString(e));
}
template <typename F>
sb_status in_pieces(int n, F piece)
{
    for (int from = 0; from < n;) {
        const int to = n - from <= 32 ? n : n - from < 350 ? n : from + 350;
        const sb_status s = piece(from, to, to - from <= 32);
        if (s != SB_OK) return s;
        from = to;
    }
    return SB_OK;
}

sb_status check_list(const sb_adamw_tensor* list, int32_t n, const sb_adamw_config* cfg)
{
    if (n < 0 || (n > 0 && !list) || !cfg) return set_error(SB_ERR_INVALID_ARG, "null list or config, or a negative count");
    if (cfg->state_bits != 32 && cfg->state_bits != 8) return set_error(SB_ERR_INVALID_ARG, "state_bits must be 32 or 8 (got %d)", cfg->state_bits);
    if (cfg->grad_dtype != SB_DT_F32 && cfg->grad_dtype != SB_DT_BF16) return set_error(SB_ERR_INVALID_ARG, "gradients are SB_DT_F32 or SB_DT_BF16");
    const size_t ga = cfg->grad_dtype == SB_DT_F32 ? 4 : 2, sa = cfg->state_bits == 32 ? 4 : 1;
    for (int32_t i = 0; i < n; ++i) {
        const sb_adamw_tensor& t = list[i];
        if (t.n < 0) return set_error(SB_ERR_SHAPE, "tensor %d: negative size", i);
        if (t.n == 0) continue;
        if (!t.m || !t.v || !aligned(t.m, sa) || !aligned(t.v, sa)) return set_error(SB_ERR_INVALID_ARG, "tensor %d: a moment is null or misaligned", i);
        if (cfg->state_bits == 8 && (!t.m_scale || !t.v_scale || !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4)))
            return set_error(SB_ERR_INVALID_ARG, "tensor %d: 8-bit moments need their scales", i);
        if (!t.param || !aligned(t.param, 4)) return set_error(SB_ERR_INVALID_ARG, "tensor %d: the parameter is null or misaligned", i);
        if (!t.grad || !aligned(t.grad, ga)) return set_error(SB_ERR_INVALID_ARG, "tensor %d: the gradient is null or misaligned", i);
        if (!aligned(t.shadow, 2)) return set_error(SB_ERR_INVALID_ARG, "tensor %d: the bf16 copy is misaligned", i);
    }
    return SB_OK;
}

}  // namespace
}  // namespace sb

using namespace sb;

extern "C" {

sb_status sb_adamw_tensors(const sb_adamw_tensor* list, int32_t n, const sb_adamw_config* cfg, const sb_adamw_hyper* h, int64_t step, void* stream)
{
    const sb_status c = check_list(list, n, cfg);
    if (c != SB_OK) return c;
    if (!h) return set_error(SB_ERR_INVALID_ARG, "null hyper-parameters");
    if (!(h->beta1 >= 0.0 && h->beta1 < 1.0) || !(h->beta2 >= 0.0 && h->beta2 < 1.0)) return set_error(SB_ERR_INVALID_ARG, "beta1 and beta2 must be in [0, 1)");
    if (!(h->eps >= 0.0) || !std::isfinite(h->lr) || !std::isfinite(h->weight_decay) || !std::isfinite(h->eps)) return set_error(SB_ERR_INVALID_ARG, "lr, eps and weight_decay must be finite, eps not negative");
    if (!h->dev_step && step < 1) return set_error(SB_ERR_INVALID_ARG, "the step number starts at 1 (got %lld)", (long long)step);
    if (!aligned(h->dev_step, 8) || !aligned(h->dev_lr, 4)) return set_error(SB_ERR_INVALID_ARG, "dev_step or dev_lr is misaligned");
    auto fill = [&](auto& a) {
        const double t = h->dev_step ? 1.0 : (double)step;
        a.beta1 = h->beta1; a.beta2 = h->beta2; a.lr = h->lr; a.wd = h->weight_decay;
        a.b1 = (float)h->beta1; a.c1 = (float)(1.0 - h->beta1); a.b2 = (float)h->beta2; a.c2 = (float)(1.0 - h->beta2); a.eps = (float)h->eps;
        a.decay = (float)(1.0 - h->lr * h->weight_decay);
        a.rate = (float)(h->lr / (1.0 - std::pow(h->beta1, t)));
        a.rs2 = (float)(1.0 / std::sqrt(1.0 - std::pow(h->beta2, t)));
        a.dev_step = h->dev_step; a.dev_lr = h->dev_lr;
        a.key0 = (uint32_t)cfg->seed; a.key1 = (uint32_t)(cfg->seed >> 32); a.step = (uint32_t)step;
    };
    const bool bf = cfg->grad_dtype == SB_DT_BF16;
    return in_pieces(n, [&](int from, int to, bool few) {
        return few ? run_list<32>(list, from, to, cfg->state_bits, bf, false, (cudaStream_t)stream, fill)
                   : run_list<350>(list, from, to, cfg->state_bits, bf, false, (cudaStream_t)stream, fill);
    });
}

sb_status sb_adamw_moments(const sb_adamw_tensor* list, int32_t n, const sb_adamw_config* cfg, void* const* m_out, void* const* v_out, void* stream)
{
    const sb_status c = check_list(list, n, cfg);
    if (c != SB_OK) return c;
    if (cfg->state_bits != 8) return set_error(SB_ERR_INVALID_ARG, "float moments are what they stand for: read them where they are");
    if (n > 0 && (!m_out || !v_out)) return set_error(SB_ERR_INVALID_ARG, "null outputs");
    for (int32_t i = 0; i < n; ++i)
        if (list[i].n > 0 && (!m_out[i] || !v_out[i] || !aligned(m_out[i], 2) || !aligned(v_out[i], 2)))
            return set_error(SB_ERR_INVALID_ARG, "tensor %d: an output is null or misaligned", i);
    auto piece = [&](int from, int to, bool few) {
        // the outputs in the places of parameter and copy
        sb_adamw_tensor out[350];
        for (int i = from; i < to; ++i) { out[i - from] = list[i]; out[i - from].param = (float*)m_out[i]; out[i - from].shadow = v_out[i]; out[i - from].grad = nullptr; }
        auto fill = [](auto&) {};
        return few ? run_list<32>(out, 0, to - from, 8, false, true, (cudaStream_t)stream, fill)
                   : run_list<350>(out, 0, to - from, 8, false, true, (cudaStream_t)stream, fill);
    };
    return in_pieces(n, piece);
}

}  // extern "C"
