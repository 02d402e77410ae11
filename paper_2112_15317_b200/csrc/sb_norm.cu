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
// What bounds it: HBM, each activation read or written once: 16384 x 4096 in bf16 with both norms, a gate and both scales, forward 96 us (5.6 TB/s; 85 at the
// measured copy rate), backward 166 (4.9 TB/s; 128): there the latency of a row's sums, with 8 warps an SM, whose registers hold the row.  A row belongs to a team of warps, 16 columns a thread (eight in rows of up to 256), so that
// a CTA works on 1 to 16 rows at a time; a team takes consecutive rows, which come through a ring of bulk copies in shared memory, two
// stages ahead.  A thread has the same columns of each row: the vectors stay in its registers and the vectors' gradients are summed there.  A
// CTA's sums go to scratch and a second kernel adds them in order (no atomics: the same bits every time).  Row chunks are whole groups, or whole parts
// of one group.  Rows that are not a multiple of 16 bytes, or too long for the ring, are read straight from global memory.
#include "sb_norm.cuh"

#include <cmath>

namespace sb {

namespace {

template <typename T, int V, int BY, bool LAYER, int PARTS>
__global__ void __launch_bounds__(THREADS, V == 1 ? 2 : 1)
norm_forward_kernel(const NormParams p)
{
    SB_NORM_BEGIN(1, THREADS);
    const bool has_f = PARTS == ALL_PARTS || (PARTS == ANY_PARTS && p.f), has_post = PARTS == ALL_PARTS || (PARTS == ANY_PARTS && p.w_post), has_pre = PARTS != ANY_PARTS || p.w_pre;
    if (team_id >= p.teams) return;
    // the vectors, once: w_pre, scale, and q = gate * w_post (for each gate row)
    F2 w_pre[V][4], scale[V][4], q[V][4];
#pragma unroll
    for (int c = 0; c < V; ++c) {
        get_vector<T, BY>(p.w_pre, w, c, d, 1.f, w_pre[c]);
        get_vector<T, BY>(p.scale, w, c, d, 1.f, scale[c]);
        get_vector<T, BY>(p.w_post, w, c, d, 1.f, q[c]);
    }
    auto use_gate = [&](const float* g) {
#pragma unroll
        for (int c = 0; c < V; ++c) {
            F2 a[4], b[4];
            get_vector<T, BY>(g, w, c, d, 1.f, a);
            get_vector<T, BY>(p.w_post, w, c, d, 1.f, b);
#pragma unroll
            for (int j = 0; j < 4; ++j) q[c][j] = a[j] * b[j];
        }
    };
    for (int64_t t = first_turn(p, team_id); t < p.turns; t += (int64_t)gridDim.x * p.teams) {
        int64_t first, end;
        turn_rows(p, t, first, end);
        const int rows = (int)(end - first), per = BY == BY_RING ? p.stage_rows : 1;
        if (BY == BY_RING && mine)
            for (int s = 0, r = 0; s < p.stages && r < rows; ++s, r += per) ring.fill(p, (ring.slot + s) % p.stages, first + r, min(per, rows - r), (int)sizeof(T));
        int64_t gate_end = 0;         // the row behind the last one of the gate row held
        for (int r0 = 0; r0 < rows; r0 += per) {
            uint32_t stage = 0u;
            if (BY == BY_RING) {
                if (r0 > 0) {
                    const int old = ring.slot, next = r0 + (p.stages - 1) * per;
                    ring.move();
                    if (mine && next < rows) ring.fill(p, old, first + next, min(per, rows - next), (int)sizeof(T));
                }
                stage = ring.wait(p);
            }
            const uint32_t one = (uint32_t)(per * d) * (uint32_t)sizeof(T);
            for (int k = 0; k < per && r0 + k < rows; ++k) {
                const int64_t row = first + r0 + k;
                const uint32_t at = stage + (uint32_t)(k * d) * (uint32_t)sizeof(T);
                float st[4] = {0.f, 0.f, 0.f, 0.f};
                F2 y[V][4];
#pragma unroll
                for (int c = 0; c < V; ++c) {
                    if (BY == BY_RING) get_ring<T>(at, w, c, d, y[c]);
                    else get_row<BY>((const T*)p.x + row * d, w, c, d, y[c]);
                }
                if (has_f) {
                    F2 h[V][4];
#pragma unroll
                    for (int c = 0; c < V; ++c) {
                        if (BY == BY_RING) get_ring<T>(at + one, w, c, d, h[c]);
                        else get_row<BY>((const T*)p.f + row * d, w, c, d, h[c]);
                    }
                    if (p.gate) {
                        if (p.gate_ring) {
                            const float* g = (const float*)(smem + (stage - smem_u32(smem)) + 2 * one) + (size_t)k * d;
                            use_gate(g);
                        } else if (row >= gate_end) {
                            const int64_t g = row / p.per_group;
                            gate_end = (g + 1) * p.per_group;
                            use_gate(p.gate + g * d);
                        }
                    }
                    if (has_post) {
                        row_stats<T, V, BY, LAYER>(h, p, w, team, st[0], st[1]);
                        if (LAYER) SB_PAIRS(c, j) h[c][j] = (h[c][j] + f2(-st[0])) * f2(st[1]);
                        else SB_PAIRS(c, j) h[c][j] = h[c][j] * f2(st[1]);
                    }
                    SB_PAIRS(c, j) y[c][j] = fma2(scale[c][j], y[c][j], q[c][j] * h[c][j]);
                    if (LAYER && has_post) {          // (the mean has moved the columns beyond d off zero)
                        SB_PAIRS(c, j) {
                            if (BY == BY_ELEMENT) y[c][j] = f2(column<T, BY>(w, c, 2 * j) < d ? lo(y[c][j]) : 0.f, column<T, BY>(w, c, 2 * j + 1) < d ? hi(y[c][j]) : 0.f);
                            else if (column<T, BY>(w, c, j / 2 * 4) >= d) y[c][j] = f2(0.f);
                        }
                    }
                    if (p.y) {
#pragma unroll
                        for (int c = 0; c < V; ++c) put_row<BY>((T*)p.y + row * d, w, c, d, y[c]);
                    }
                }
                if (has_pre) {
                    row_stats<T, V, BY, LAYER>(y, p, w, team, st[2], st[3]);
                    if (LAYER) SB_PAIRS(c, j) y[c][j] = w_pre[c][j] * ((y[c][j] + f2(-st[2])) * f2(st[3]));
                    else SB_PAIRS(c, j) y[c][j] = w_pre[c][j] * (y[c][j] * f2(st[3]));
#pragma unroll
                    for (int c = 0; c < V; ++c) put_row<BY>((T*)p.n + row * d, w, c, d, y[c]);
                }
                if (BY == BY_RING && ((!has_pre && !has_post) || team.warps == 1)) team.barrier();       // (behind the row's last read)
                if (p.stats && mine) *(float4*)(p.stats + row * 4) = make_float4(st[0], st[1], st[2], st[3]);
            }
        }
        if (BY == BY_RING) ring.move();
    }
}

// out[b][col] = sum over k < n, in order within parts of n and then over these, of part[(b * n + k) * stride + col].  One launch for the vectors
// (blockIdx.y 0 .. 2) and the gate's groups (from 3 on).
struct SumArgs { const float *part, *gate_part; float *out[3], *gate; int64_t n, gate_n, groups; int d; };
constexpr int SUM_WARPS = 16;
__global__ void __launch_bounds__(SUM_WARPS * 32) norm_sum_kernel(const SumArgs a)
{
    pdl_prologue();
    __shared__ float s[SUM_WARPS][32];
    const int lane = threadIdx.x % 32, w = threadIdx.x / 32, col = blockIdx.x * 32 + lane;
    const bool gate = blockIdx.y >= 3;
    const int64_t n = gate ? a.gate_n : a.n, stride = gate ? a.d : (int64_t)3 * a.d;
    const int64_t per = (n + SUM_WARPS - 1) / SUM_WARPS, k0 = w * per, k1 = k0 + per < n ? k0 + per : n;
    for (int64_t b = gate ? blockIdx.y - 3 : 0; b < (gate ? a.groups : 1); b += gate ? gridDim.y - 3 : 1) {
        float* out = gate ? a.gate + b * a.d : a.out[blockIdx.y];
        if (!out) return;
        const float* p = gate ? a.gate_part + b * n * stride + col : a.part + (int64_t)blockIdx.y * a.d + col;
        float v = 0.f;
        if (col < a.d) {
#pragma unroll 8
            for (int64_t k = k0; k < k1; ++k) v += p[k * stride];
        }
        s[w][lane] = v;
        __syncthreads();
        if (w == 0 && col < a.d) {
            for (int i = 1; i < SUM_WARPS; ++i) v += s[i][lane];
            out[col] = v;
        }
        __syncthreads();
    }
}

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

template <typename T, int V, int BY, bool LAYER, int PARTS>
cudaError_t run_forward(const NormParams& p, int64_t ctas, cudaStream_t st)
{
    const cudaError_t e = raise_smem_limit<norm_forward_kernel<T, V, BY, LAYER, PARTS>>(RING_LIMIT);
    return e != cudaSuccess ? e : pdl_launch(norm_forward_kernel<T, V, BY, LAYER, PARTS>, dim3((unsigned)ctas), dim3(THREADS), ring_bytes(p), st, p);
}
template <typename T, int V, int BY, bool LAYER>
cudaError_t forward_parts(const NormParams& p, int64_t ctas, cudaStream_t st)
{
    if constexpr (BY == BY_RING && V <= 2) {
        if (p.f && p.w_post && p.w_pre) return run_forward<T, V, BY, LAYER, ALL_PARTS>(p, ctas, st);
        if (!p.f) return run_forward<T, V, BY, LAYER, PRE_ONLY>(p, ctas, st);
    }
    return run_forward<T, V, BY, LAYER, ANY_PARTS>(p, ctas, st);
}
template <typename T, int V, int BY>
cudaError_t forward_kind(const NormParams& p, bool layer, int64_t ctas, cudaStream_t st) { return layer ? forward_parts<T, V, BY, true>(p, ctas, st) : forward_parts<T, V, BY, false>(p, ctas, st); }
template <typename T, int V>
cudaError_t forward_by(const NormParams& p, bool layer, int64_t ctas, cudaStream_t st)
{
    const int by = by_of(p);
    if (by == BY_RING) return forward_kind<T, V, BY_RING>(p, layer, ctas, st);
    if constexpr (V == 4)                    // (up to 8192 columns a ring always fits)
        if (by == BY_PIECES) return forward_kind<T, V, BY_PIECES>(p, layer, ctas, st);
    return forward_kind<T, V, BY_ELEMENT>(p, layer, ctas, st);
}
template <typename T>
cudaError_t forward_pieces(const NormParams& p, bool layer, int64_t ctas, cudaStream_t st)
{
    const int v = pieces_of(p.d, p.vec);
    return v == 1 ? forward_by<T, 1>(p, layer, ctas, st) : v == 2 ? forward_by<T, 2>(p, layer, ctas, st) : forward_by<T, 4>(p, layer, ctas, st);
}

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
sb_status check_vectors(const sb_norm_config* c, const void* f, const float* w_pre, const float* w_post, const float* gate, const float* scale)
{
    if (!aligned(w_pre, 4) || !aligned(w_post, 4) || !aligned(gate, 4) || !aligned(scale, 4)) return set_error(SB_ERR_INVALID_ARG, "a vector is misaligned");
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
    if ((s = check_vectors(c, f, w_pre, w_post, gate, scale)) != SB_OK) return s;
    if (!dy && !dn) return set_error(SB_ERR_INVALID_ARG, "dy and dn are both null");
    if (dn && !w_pre) return set_error(SB_ERR_INVALID_ARG, "dn needs w_pre");
    if (dw_pre && !dn) return set_error(SB_ERR_INVALID_ARG, "dw_pre needs dn");
    if (df && !f) return set_error(SB_ERR_INVALID_ARG, "df needs f");
    if ((dw_post && !w_post) || (dgate && !gate) || (dscale && !scale)) return set_error(SB_ERR_INVALID_ARG, "a gradient of a vector that is null");
    if (!aligned(dw_pre, 4) || !aligned(dw_post, 4) || !aligned(dgate, 4) || !aligned(dscale, 4)) return set_error(SB_ERR_INVALID_ARG, "a vector's gradient is misaligned");
    const size_t e = c->precision == SB_BF16 ? 2 : 4;
    if (!aligned(x, e) || !aligned(dy, e) || !aligned(dn, e) || !aligned(f, e) || !aligned(dx, e) || !aligned(df, e)) return set_error(SB_ERR_INVALID_ARG, "a matrix is misaligned");
    if (!x || !stats || !aligned(stats, 16)) return set_error(SB_ERR_INVALID_ARG, "x or stats is null, or stats not 16-byte aligned");
    const size_t floats = part_floats(c);
    if (!ws || !aligned(ws, 16) || ws_bytes < floats * 4) return set_error(SB_ERR_ARENA_TOO_SMALL, "the workspace must be 16-byte aligned and hold %zu bytes (got %zu)", floats * 4, ws_bytes);
    NormParams p = params_of(c, x, w_pre, f, w_post, gate, scale);
    const bool vec = vec_ok(c->d, x, f, dy, dn, dx, df, w_pre, w_post, gate, scale, dgate);
    const Grid g = grid_of(c, true, vec);
    const Turns& t = g.turns;
    p.vec = vec;
    p.dy = dy; p.dn = dn; p.dx = dx; p.df = df; p.stats = (float*)stats; p.relu_x = relu_x;
    spread(p, g);
    p.chunks_per_group = t.per_group;
    float* part = (float*)ws;
    float* gate_part = part + ((size_t)g.ctas * 3 * c->d + 15) / 16 * 16;
    p.part = want ? part : nullptr;
    p.gate_out = !dgate ? nullptr : t.per_group > 1 ? gate_part : dgate;
    p.status = ops_status();
    if (!p.status) return set_error(SB_ERR_CUDA, "the status word has no address on this device");
    if (vec) { p.gate_ring = gate && p.per_group == 1; plan_ring(p, g, (int)e, pieces_of(c->d, vec) == 1 ? RING_LIMIT / 2 : RING_LIMIT); }
    cudaError_t r = c->precision == SB_BF16 ? launch_norm_backward_bf16(p, c->kind == SB_NORM_LAYER, g.ctas, st)
                                             : launch_norm_backward_f32(p, c->kind == SB_NORM_LAYER, g.ctas, st);
    const bool gate_sum = dgate && t.per_group > 1;
    if (r == cudaSuccess && (want || gate_sum)) {
        const SumArgs a{part, gate_part, {dw_pre, dw_post, dscale}, dgate, g.ctas, t.per_group, c->groups, c->d};
        const unsigned extra = !gate_sum ? 0u : (unsigned)(c->groups < 256 ? c->groups : 256);
        r = pdl_launch(norm_sum_kernel, dim3((unsigned)((c->d + 31) / 32), 3 + extra), dim3(SUM_WARPS * 32), 0, st, a);
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
    if ((s = check_vectors(c, f, w_pre, w_post, gate, scale)) != SB_OK) return s;
    if (!f && !w_pre) return set_error(SB_ERR_INVALID_ARG, "neither f nor w_pre: there is nothing to compute");
    if ((n != nullptr) != (w_pre != nullptr)) return set_error(SB_ERR_INVALID_ARG, "n and w_pre go together");
    if (y && !f) return set_error(SB_ERR_INVALID_ARG, "y is x where f is null");
    const size_t e = c->precision == SB_BF16 ? 2 : 4;
    if (!aligned(x, e) || !aligned(f, e) || !aligned(y, e) || !aligned(n, e) || !aligned(stats, 16)) return set_error(SB_ERR_INVALID_ARG, "a matrix or stats is misaligned");
    if (!x) return set_error(SB_ERR_INVALID_ARG, "x is null");
    NormParams p = params_of(c, x, w_pre, f, w_post, gate, scale);
    p.y = y; p.n = n; p.stats = stats;
    const bool vec = vec_ok(c->d, x, f, y, n, w_pre, w_post, gate, scale);
    const Grid g = grid_of(c, false, vec);
    p.vec = vec;
    spread(p, g);
    p.status = ops_status();
    if (!p.status) return set_error(SB_ERR_CUDA, "the status word has no address on this device");
    // (two CTAs an SM where a warp holds a row)
    if (vec) { p.gate_ring = gate && p.per_group == 1; plan_ring(p, g, (int)e, pieces_of(c->d, vec) == 1 ? RING_LIMIT / 2 : RING_LIMIT); }
    const cudaError_t r = c->precision == SB_BF16 ? forward_pieces<__nv_bfloat16>(p, c->kind == SB_NORM_LAYER, g.ctas, (cudaStream_t)stream)
                                                   : forward_pieces<float>(p, c->kind == SB_NORM_LAYER, g.ctas, (cudaStream_t)stream);
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
