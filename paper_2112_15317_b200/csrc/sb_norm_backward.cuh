// Backward pass of the norms around a block: kernel and launch (formulas, layout and what bounds it: sb_norm.cu).  Each activation type is compiled in a file of
// its own (sb_norm_backward_bf16.cu, sb_norm_backward_f32.cu), which halves the time of a parallel build.
#pragma once

#include "sb_norm.cuh"

namespace sb {

namespace {

// The vectors' columns of a thread: in registers, or in shared memory in the order in which the threads read them (512 threads with 16 columns
// each, whose accumulators take their 128 registers): 16-byte pieces, neighbouring threads' next to each other.  w_pre and scale are the same for every team, and each
// writes them there; a thread only ever reads what it has written itself, or another has with the same values.
template <int V, bool SHARED> struct Held {
    F2 v[SHARED ? 1 : V][4];
    uint32_t at;             // SHARED: this thread's first piece
    int step;                // from piece to piece
    __device__ __forceinline__ void put(int c, const F2 (&a)[4])
    {
        if (!SHARED) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[SHARED ? 0 : c][j] = a[j];
            return;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at + (uint32_t)((2 * c + h) * step)), "f"(lo(a[2 * h])), "f"(hi(a[2 * h])), "f"(lo(a[2 * h + 1])), "f"(hi(a[2 * h + 1])) : "memory");
    }
    __device__ __forceinline__ void get(int c, F2 (&a)[4]) const
    {
        if (!SHARED) {
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] = v[SHARED ? 0 : c][j];
            return;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 b = lds16(at + (uint32_t)((2 * c + h) * step));
            a[2 * h] = f2(__uint_as_float(b.x), __uint_as_float(b.y));
            a[2 * h + 1] = f2(__uint_as_float(b.z), __uint_as_float(b.w));
        }
    }
};

template <typename T, int V, int BY, bool LAYER, int NT, int PARTS>
__global__ void __launch_bounds__(NT, NT == 256 && V == 1 ? 2 : 1)
norm_backward_kernel(const NormParams p)
{
    constexpr int K = LAYER ? 8 : 4;
    constexpr bool SHARED = NT == 512 && V == 2;
    SB_NORM_BEGIN(K, NT);
    // what there is: known at compile time for the two usual cases
    const bool has_f = PARTS == ALL_PARTS || (PARTS == ANY_PARTS && p.f), has_post = PARTS == ALL_PARTS || (PARTS == ANY_PARTS && p.w_post);
    const bool has_dn = PARTS != ANY_PARTS || p.dn, has_dy = PARTS != ANY_PARTS || p.dy, relu_x = PARTS == ANY_PARTS && p.relu_x;
    const bool has_dx = PARTS != ANY_PARTS || p.dx, has_df = PARTS == ALL_PARTS || (PARTS == ANY_PARTS && p.df);
    const bool idle = team_id >= p.teams;
    const F2 zero = f2(0.f);
    F2 a_pre[V][4], a_post[V][4], a_scale[V][4];
    SB_PAIRS(c, j) { a_pre[c][j] = zero; a_post[c][j] = zero; a_scale[c][j] = zero; }
    if (!idle) {
        Held<V, SHARED> w_pre, scale, q;         // q = gate * w_post
        if (SHARED) {
            const uint32_t one = (uint32_t)(V * 8 * w.width) * 4u, base = smem_u32(smem) + (uint32_t)(p.teams * p.stages * p.stage_bytes) + (uint32_t)w.t * 16u;
            w_pre.at = base; scale.at = base + one; q.at = base + (2u + (p.gate ? (uint32_t)team_id : 0u)) * one;
            w_pre.step = scale.step = q.step = w.width * 16;
        }
        F2 a_hat[V][4];                          // sum of d * fhat over the rows of the gate row held
#pragma unroll
        for (int c = 0; c < V; ++c) {
            F2 a[4];
            get_vector<T, BY>(p.w_pre, w, c, d, 1.f, a); w_pre.put(c, a);
            get_vector<T, BY>(p.scale, w, c, d, 1.f, a); scale.put(c, a);
            get_vector<T, BY>(p.w_post, w, c, d, 1.f, a); q.put(c, a);
#pragma unroll
            for (int j = 0; j < 4; ++j) a_hat[c][j] = zero;
        }
        auto use_gate = [&](const float* g) {
#pragma unroll
            for (int c = 0; c < V; ++c) {
                F2 a[4], b[4];
                get_vector<T, BY>(g, w, c, d, 1.f, a);
                get_vector<T, BY>(p.w_post, w, c, d, 1.f, b);
#pragma unroll
                for (int j = 0; j < 4; ++j) a[j] = a[j] * b[j];
                q.put(c, a);
            }
        };
        // behind the last row of a gate row (or of the turn's part of it): dg and dwpost from the sum of d * fhat
        auto close_gate = [&](const float* g, float* out) {
#pragma unroll
            for (int c = 0; c < V; ++c) {
                F2 a[4], b[4];
                get_vector<T, BY>(g, w, c, d, 1.f, a);
                get_vector<T, BY>(p.w_post, w, c, d, 1.f, b);
#pragma unroll
                for (int j = 0; j < 4; ++j) { a_post[c][j] = fma2(a[j], a_hat[c][j], a_post[c][j]); b[j] = b[j] * a_hat[c][j]; a_hat[c][j] = zero; }
                if (out) put_vector<T, BY>(out, w, c, d, b);
            }
        };
        for (int64_t t = first_turn(p, team_id); t < p.turns; t += (int64_t)gridDim.x * p.teams) {
            int64_t first, end;
            turn_rows(p, t, first, end);
            const int rows = (int)(end - first), per = BY == BY_RING ? p.stage_rows : 1;
            if (BY == BY_RING && mine)
                for (int s = 0, r = 0; s < p.stages && r < rows; ++s, r += per) ring.fill(p, (ring.slot + s) % p.stages, first + r, min(per, rows - r), (int)sizeof(T));
            int64_t group = 0, gate_end = 0;      // the gate row held, and the row behind its last
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
                    uint32_t at = stage + (uint32_t)(k * d) * (uint32_t)sizeof(T);
                    float4 st;
                    const uint32_t ring_end = stage + one * (uint32_t)p.arrays;
                    if (BY == BY_RING) {
                        const uint4 a = lds16(ring_end + (p.gate_ring ? (uint32_t)(per * d) * 4u : 0u) + (uint32_t)k * 16u);
                        st = make_float4(__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w));
                    } else st = *(const float4*)(p.stats + row * 4);
                    if (p.gate && row >= gate_end) {
                        group = p.gate_ring ? row : row / p.per_group;
                        gate_end = (group + 1) * p.per_group;
                        use_gate(p.gate_ring ? (const float*)(smem + (ring_end - smem_u32(smem))) + (size_t)k * d : p.gate + group * d);
                    }
                    F2 x[V][4], fh[V][4], e[V][4];
                    // yhat of a pair of columns, from x and fhat (columns beyond d: zero)
                    const F2 iy2 = f2(st.w), if2 = f2(st.y);
                    auto y_hat = [&](int c, int j, F2 sc, F2 qj) {
                        F2 y = has_f ? fma2(sc, x[c][j], qj * fh[c][j]) : x[c][j];
                        if (!LAYER) return y * iy2;
                        y = (y + f2(-st.z)) * iy2;
                        if (BY == BY_ELEMENT) return f2(column<T, BY>(w, c, 2 * j) < d ? lo(y) : 0.f, column<T, BY>(w, c, 2 * j + 1) < d ? hi(y) : 0.f);
                        return column<T, BY>(w, c, j / 2 * 4) < d ? y : zero;
                    };
                    // sums: 0 z yhat, 1 q fhat e, 2 q fhat yhat (3 is zero); LAYER: 3 z, 4 q fhat, 5 q e, 6 q yhat, 7 q
                    F2 s[K];
#pragma unroll
                    for (int i = 0; i < K; ++i) s[i] = zero;
#pragma unroll
                    for (int c = 0; c < V; ++c) {
                        F2 dz[4], wp[4], sc[4], qc[4];
                        uint32_t from = at;
                        auto get = [&](const void* global, F2 (&o)[4]) {
                            if (BY == BY_RING) { get_ring<T>(from, w, c, d, o); from += one; }
                            else get_row<BY>((const T*)global + row * d, w, c, d, o);
                        };
                        get(p.x, x[c]);
                        if (has_f) get(p.f, fh[c]);
                        if (has_dy) get(p.dy, e[c]);
                        if (has_dn) get(p.dn, dz);
                        w_pre.get(c, wp);
                        if (has_f) { scale.get(c, sc); q.get(c, qc); }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (!has_f) { fh[c][j] = zero; sc[j] = zero; qc[j] = zero; }
                            if (!has_dy) e[c][j] = zero;
                            if (has_post) fh[c][j] = LAYER ? (fh[c][j] + f2(-st.x)) * if2 : fh[c][j] * if2;
                            F2 yh = zero;
                            if (has_dn) {
                                yh = y_hat(c, j, sc[j], qc[j]);
                                const F2 z = wp[j] * dz[j];            // (dn is zero beyond d, and so is z)
                                a_pre[c][j] = fma2(dz[j], yh, a_pre[c][j]);
                                e[c][j] = fma2(iy2, z, e[c][j]);
                                s[0] = fma2(z, yh, s[0]);
                                if (LAYER) s[LAYER ? 3 : 0] = s[LAYER ? 3 : 0] + z;
                            }
                            if (has_post) {
                                F2 qj = qc[j];
                                if (LAYER) {
                                    if (BY == BY_ELEMENT) qj = f2(column<T, BY>(w, c, 2 * j) < d ? lo(qj) : 0.f, column<T, BY>(w, c, 2 * j + 1) < d ? hi(qj) : 0.f);
                                    else if (column<T, BY>(w, c, j / 2 * 4) >= d) qj = zero;
                                }
                                const F2 qf = qj * fh[c][j];
                                s[1] = fma2(qf, e[c][j], s[1]);
                                s[2] = fma2(qf, yh, s[2]);
                                if (LAYER) {
                                    s[LAYER ? 4 : 0] = s[LAYER ? 4 : 0] + qf;
                                    s[LAYER ? 5 : 0] = fma2(qj, e[c][j], s[LAYER ? 5 : 0]);
                                    s[LAYER ? 6 : 0] = fma2(qj, yh, s[LAYER ? 6 : 0]);
                                    s[LAYER ? 7 : 0] = s[LAYER ? 7 : 0] + qj;
                                }
                            }
                        }
                    }
                    float v[K];
#pragma unroll
                    for (int i = 0; i < K; ++i) v[i] = lo(s[i]) + hi(s[i]);
                    team_sum<K>(team, v);
                    // the means in d, then those in df
                    const float c1 = has_dn ? v[0] * p.rd : 0.f, c0 = LAYER && has_dn ? v[LAYER ? 3 : 0] * p.rd : 0.f, iy = has_dn ? st.w : 0.f;
                    const float f1 = (v[1] - iy * (c0 * (LAYER ? v[LAYER ? 4 : 0] : 0.f) + c1 * v[2])) * p.rd;
                    const float f0 = LAYER ? (v[LAYER ? 5 : 0] - iy * (c0 * v[LAYER ? 7 : 0] + c1 * v[LAYER ? 6 : 0])) * p.rd : 0.f;
                    const F2 m1 = f2(-iy * c1), m0 = f2(-iy * c0), n1 = f2(-st.y * f1), n0 = f2(-st.y * f0);
#pragma unroll
                    for (int c = 0; c < V; ++c) {
                        F2 o[4], sc[4], qc[4];
                        if (has_f) { scale.get(c, sc); q.get(c, qc); }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (!has_f) { sc[j] = zero; qc[j] = zero; }
                            F2 D = e[c][j];
                            if (has_dn) D = fma2(m1, y_hat(c, j, sc[j], qc[j]), D);
                            if (LAYER) D = D + m0;
                            e[c][j] = D;
                            a_scale[c][j] = fma2(D, x[c][j], a_scale[c][j]);
                            a_hat[c][j] = fma2(D, fh[c][j], a_hat[c][j]);
                            o[j] = has_f ? sc[j] * D : D;
                            if (relu_x) o[j] = f2(lo(x[c][j]) > 0.f ? lo(o[j]) : 0.f, hi(x[c][j]) > 0.f ? hi(o[j]) : 0.f);
                        }
                        if (has_dx) put_row<BY>((T*)p.dx + row * d, w, c, d, o);
                        if (has_df) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                o[j] = qc[j] * e[c][j];
                                if (has_post) {
                                    o[j] = fma2(if2, o[j], n1 * fh[c][j]);
                                    if (LAYER) o[j] = o[j] + n0;
                                }
                            }
                            put_row<BY>((T*)p.df + row * d, w, c, d, o);
                        }
                    }
                    // the end of a group, or of the turn's part of one
                    if (p.gate && (row + 1 == gate_end || row + 1 == end))
                        close_gate(p.gate + group * d, !p.gate_out ? nullptr : p.gate_out + (p.chunks_per_group > 1 ? t : group) * d);
                    if (BY == BY_RING && team.warps == 1) __syncwarp();
                }
            }
            if (BY == BY_RING) ring.move();
        }
        if (has_f && !p.gate) close_gate(nullptr, nullptr);
    }
    if (!p.part) return;
    // The teams' sums, one array after the other through shared memory, added in the teams' order (the ring is done with)
    float* sums = (float*)smem;
    auto join = [&](const F2 (&a)[V][4], int which) {
        __syncthreads();
        if (!idle) {
#pragma unroll
            for (int c = 0; c < V; ++c) put_vector<T, BY>(sums + (size_t)team_id * d, w, c, d, a[c]);
        }
        __syncthreads();
        float* out = p.part + ((int64_t)blockIdx.x * 3 + which) * d;
        for (int i = threadIdx.x; i < d; i += NT) {
            float v = sums[i];
            for (int k = 1; k < p.teams; ++k) v += sums[(size_t)k * d + i];
            out[i] = v;
        }
    };
    join(a_pre, 0);
    join(a_post, 1);
    join(a_scale, 2);
}

template <typename T, int V, int BY, bool LAYER, int NT, int PARTS>
cudaError_t run_backward(const NormParams& p, int64_t ctas, cudaStream_t st)
{
    const cudaError_t e = raise_smem_limit<norm_backward_kernel<T, V, BY, LAYER, NT, PARTS>>(RING_LIMIT);
    const size_t sums = (size_t)p.teams * p.d * 4, ring = ring_bytes(p) + vector_bytes(p);      // (the sums of the teams follow the ring in the same place)
    return e != cudaSuccess ? e : pdl_launch(norm_backward_kernel<T, V, BY, LAYER, NT, PARTS>, dim3((unsigned)ctas), dim3(NT), ring > sums ? ring : sums, st, p);
}
template <typename T, int V, int BY, bool LAYER, int NT>
cudaError_t backward_parts(const NormParams& p, int64_t ctas, cudaStream_t st)
{
    const bool both = p.dy && p.dn && p.dx && !p.relu_x;
    if constexpr ((BY == BY_RING || BY == BY_ELEMENT) && V <= 2)
        if (both && p.f && p.w_post && p.df) return run_backward<T, V, BY, LAYER, NT, ALL_PARTS>(p, ctas, st);
    if constexpr (BY == BY_RING && V <= 2)
        if (both && !p.f) return run_backward<T, V, BY, LAYER, NT, PRE_ONLY>(p, ctas, st);
    return run_backward<T, V, BY, LAYER, NT, ANY_PARTS>(p, ctas, st);
}
// (Up to 4096 columns a ring always fits, and element by element two pieces a thread begin there: the other combinations do not occur.)
template <typename T, int V, int BY, bool LAYER>
cudaError_t backward_threads_of(const NormParams& p, int64_t ctas, cudaStream_t st)
{
    if constexpr (V == 4 || (V == 2 && BY != BY_RING)) return backward_parts<T, V, BY, LAYER, 512>(p, ctas, st);
    else if constexpr (V == 1 && BY == BY_RING) return backward_parts<T, V, BY, LAYER, 256>(p, ctas, st);
    else return backward_threads(p.d, p.vec) == 256 ? backward_parts<T, V, BY, LAYER, 256>(p, ctas, st) : backward_parts<T, V, BY, LAYER, 512>(p, ctas, st);
}
template <typename T, int V, int BY>
cudaError_t backward_kind(const NormParams& p, bool layer, int64_t ctas, cudaStream_t st) { return layer ? backward_threads_of<T, V, BY, true>(p, ctas, st) : backward_threads_of<T, V, BY, false>(p, ctas, st); }
template <typename T, int V>
cudaError_t backward_by(const NormParams& p, bool layer, int64_t ctas, cudaStream_t st)
{
    const int by = by_of(p);
    if (by == BY_RING) return backward_kind<T, V, BY_RING>(p, layer, ctas, st);
    if constexpr (V > 1)
        if (by == BY_PIECES) return backward_kind<T, V, BY_PIECES>(p, layer, ctas, st);
    return backward_kind<T, V, BY_ELEMENT>(p, layer, ctas, st);
}
template <typename T>
cudaError_t backward_pieces(const NormParams& p, bool layer, int64_t ctas, cudaStream_t st)
{
    const int v = pieces_of(p.d, p.vec);
    return v == 1 ? backward_by<T, 1>(p, layer, ctas, st) : v == 2 ? backward_by<T, 2>(p, layer, ctas, st) : backward_by<T, 4>(p, layer, ctas, st);
}

}  // namespace

}  // namespace sb
