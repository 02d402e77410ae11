// Gated feed-forward block for few rows (bf16): products whose time is the reading of the weights.
//
// The weights are the M side of the MMA (128 of their output columns a CTA) and the rows the N side (16 to 128), so that one token pads to 16 columns
// and not to 128 rows.  What bounds it: HBM (one row, 4096 x 8192, forward: 36.6 us, 5.5 TB/s of weights; the rest is launch, set-up and the clusters'
// sums of two dependent kernels).  A CTA holds a ring of about 100 KB, two CTAs fit an SM, and the reduction is split over a cluster of up to
// eight CTAs until the machine is full: 100 to 290 CTAs with deep rings keep more bytes in flight than HBM's latency needs, whatever
// SM they sit on.  The cluster's partial tiles are added through distributed shared memory, in rank order, each CTA finishing its share of the rows: no
// second kernel, no atomics.  The forward product's tile is 64 gate columns and the 64 up columns that belong to them, so that the activation
// follows the sum directly.
// The second product of a pass fetches its first weights before it waits for the first product (which writes no weights, and whose own wait
// says that everything before it is complete).
#include "sb_ffn.h"
#include "sb_ffn_umma.h"
#include "sb_tcgen05.cuh"
#include "sb_umma.h"

#include <algorithm>

namespace sb {

namespace {

constexpr int RW_EPI = 256, RW_THREADS = 64 + RW_EPI, RW_RING = 106 * 1024, RW_CTRL = 1024, RW_MAX_STAGES = 8;
template <int NT> struct Rw {
    static constexpr int STAGE = 16384 + NT * 128;
    static constexpr int FIT = RW_RING / STAGE, STAGES = FIT < RW_MAX_STAGES ? FIT : RW_MAX_STAGES;
    static constexpr int PART = NT * 512;                                                  // one partial tile, float
    static constexpr int BODY = STAGES * STAGE > PART ? STAGES * STAGE : PART;
    static constexpr int SMEM = BODY + 1024 + RW_CTRL;
    // With this much, no kernel of CTA pairs that takes all 512 columns of tensor memory (136 KB of shared memory or more) fits beside a CTA: clusters
    // on the same SMs must not wait for each other's columns, each holding some.
    static_assert(SMEM >= 92 * 1024, "shared memory");
    static constexpr uint32_t TMEM = NT < 32 ? 32 : NT;
};
enum { RW_STORE = 0, RW_GLU = 1, RW_GLU_BACK = 2 };

struct alignas(64) RowsArgs {
    CUtensorMap w, t;          // weights, boxes of 64 x 64; rows, boxes of NT rows
    int a_mn;                  // weights as they lie: 0 = reduction along a row, 1 = down a column
    int w_split;               // RW_GLU: from a gate row to its up row
    int rows, m, chunks, early, act;
    int live;                  // RW_GLU, RW_GLU_BACK: H's columns from there on are zero
    const __nv_bfloat16* kept; // RW_GLU_BACK: GU
    __nv_bfloat16 *out, *gu;   // RW_STORE: [rows, m]; RW_GLU: H and (or nullptr) GU; RW_GLU_BACK: H and dG, dU
    uint32_t* status;
};

__device__ __forceinline__ void ld_cluster_f32x4(uint32_t caddr, float* v)
{
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(caddr) : "memory");
}
__device__ __forceinline__ void store_bf16x4(__nv_bfloat16* p, const float (&v)[4], uint2 keep = make_uint2(~0u, ~0u))
{
    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
    *(uint2*)p = make_uint2(*(const uint32_t*)&a & keep.x, *(const uint32_t*)&b & keep.y);
}
// (read-only in this kernel: such loads may go ahead of earlier stores)
__device__ __forceinline__ void load_bf16x4(const __nv_bfloat16* p, float (&v)[4])
{
    const uint2 a = __ldg((const uint2*)p);
    v[0] = __uint_as_float(a.x << 16); v[1] = __uint_as_float(a.x & 0xffff0000u);
    v[2] = __uint_as_float(a.y << 16); v[3] = __uint_as_float(a.y & 0xffff0000u);
}

template <int NT, int EPI>
__global__ void __launch_bounds__(RW_THREADS, 2)
ffn_rows_kernel(const __grid_constant__ RowsArgs a)
{
    using C = Rw<NT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* ctrl = smem + C::BODY;
    uint64_t *full = (uint64_t*)ctrl, *empty = full + RW_MAX_STAGES, *acc_full = empty + RW_MAX_STAGES;
    uint32_t* tmem_slot = (uint32_t*)(acc_full + 1);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t smem0 = smem_u32(smem);
    const int S = (int)gridDim.x, rank = (int)blockIdx.x;             // (a cluster is a row of the grid)
    const int per = (a.chunks + S - 1) / S, c0 = min(rank * per, a.chunks), c1 = min(c0 + per, a.chunks);
    const int m0 = (int)blockIdx.y * (EPI == RW_GLU ? 64 : 128), m1 = EPI == RW_GLU ? m0 + a.w_split : m0 + 64, t0 = (int)blockIdx.z * NT;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        mbar_init(acc_full, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (warp == 1) {
        tmem_alloc(tmem_slot, C::TMEM);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    uint32_t bad = 0u;

    if (warp == 0) {
        const uint32_t el = elect_one() ? 1u : 0u;
        const uint32_t full0 = smem_u32(full);
        auto weights = [&](int s, int c) {
            const uint32_t dst = smem0 + (uint32_t)(s * C::STAGE), bar = full0 + 8u * (uint32_t)s;
            mbar_expect_tx_el(bar, (uint32_t)C::STAGE, el);
            if (!a.a_mn) {
                tma_load_4d_el(&a.w, dst, bar, c * 64, m0, 0, 0, el);
                tma_load_4d_el(&a.w, dst + 8192u, bar, c * 64, m1, 0, 0, el);
            } else {
                tma_load_4d_el(&a.w, dst, bar, m0, c * 64, 0, 0, el);
                tma_load_4d_el(&a.w, dst + 8192u, bar, m1, c * 64, 0, 0, el);
            }
        };
        const int ahead = a.early ? min(C::STAGES, c1 - c0) : 0;
        for (int s = 0; s < ahead; ++s) weights(s, c0 + s);
        pdl_wait();
        pdl_trigger();
        int s = 0;
        uint32_t ph = 1u;
        bool ok = true;
        for (int c = c0; c < c1; ++c) {
            if (c - c0 >= ahead) {
                ok = __all_sync(0xffffffffu, mbar_wait(&empty[s], ph) ? 1 : 0) != 0;
                if (!ok) break;
                weights(s, c);
            }
            tma_load_4d_el(&a.t, smem0 + (uint32_t)(s * C::STAGE) + 16384u, full0 + 8u * (uint32_t)s, c * 64, t0, 0, 0, el);
            if (++s == C::STAGES) { s = 0; ph ^= 1u; }
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicMax(a.status, (uint32_t)DEV_TIMEOUT_TMA); }
        __syncwarp();
    } else if (warp == 1) {
        const uint32_t el = elect_one() ? 1u : 0u;
        const uint32_t idesc = make_idesc(NT, a.a_mn, 0);
        const uint64_t dA = make_desc(smem0, a.a_mn ? 8192 : 16), dB = make_desc(smem0 + 16384u, 16);
        const uint32_t a_hi = (uint32_t)(dA >> 32), b_hi = (uint32_t)(dB >> 32), a_step = a.a_mn ? 128u : 2u;
        int s = 0;
        uint32_t ph = 0u;
        bool ok = true;
        for (int c = c0; c < c1; ++c) {
            ok = __all_sync(0xffffffffu, mbar_wait(&full[s], ph) ? 1 : 0) != 0;
            if (!ok) break;
            tc_fence_after();
            const uint32_t off = (uint32_t)(s * C::STAGE) >> 4;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
                umma_bf16_lohi(tmem_base, (uint32_t)dA + off + a_step * kk, a_hi, (uint32_t)dB + off + 2u * kk, b_hi, idesc, (c > c0 || kk > 0) ? 1u : 0u, el);
            if (el) umma_commit(&empty[s]);
            __syncwarp();
            if (++s == C::STAGES) { s = 0; ph ^= 1u; }
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicMax(a.status, (uint32_t)DEV_TIMEOUT_MMA); }
        if (ok && el) umma_commit(acc_full);
        __syncwarp();
    } else {
        // the partial tile into shared memory, [row of the batch][output column] (the ring is done with: every MMA has read it)
        const int quad = warp % 4, r = quad * 32 + lane;      // (two warps a TMEM lane quadrant, every other 16 columns each)
        bool ok = true;
        if (lane == 0) ok = mbar_wait(acc_full, 0u);
        ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
        if (!ok && lane == 0) { *abort_flag = 1; atomicMax(a.status, (uint32_t)DEV_TIMEOUT_EPI); }
        tc_fence_after();
        float* part = (float*)smem;
#pragma unroll 1
        for (int c = (warp - 2) / 4; c < NT / 16 && ok; c += 2) {
            uint32_t v[16];
            tmem_ld16(tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(c * 16), v);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) part[(c * 16 + j) * 128 + r] = c1 > c0 ? __uint_as_float(v[j]) : 0.f;      // (no chunks: nothing was accumulated)
        }
        pdl_wait();               // (from here on global memory is read and written)
        bad = ok ? 0u : 1u;
    }
    tc_fence_before();
    if (S > 1) cluster_sync_all(); else __syncthreads();

    if (warp >= 2 && !bad) {
        // four columns a thread: a warp a row of the batch (two rows where a row is 64 pairs), rows rank, rank + S, ...
        constexpr int LANES = EPI == RW_GLU ? 16 : 32, AT_ONCE = RW_EPI / LANES;
        const int e = threadIdx.x - 64, part_col = e % LANES * 4, col = m0 + part_col;
        uint32_t peer[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) peer[s] = map_to_cta(smem0, (uint32_t)(s < S ? s : 0));
        auto sum = [&](int tok, int from, float (&v)[4]) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = 0.f;
#pragma unroll
            for (int s = 0; s < 8; ++s)
                if (s < S) {
                    float w[4];
                    ld_cluster_f32x4(peer[s] + (uint32_t)(tok * 128 + from) * 4u, w);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] += w[j];
                }
        };
        const int last = min(NT, a.rows - t0);
        // (bits of this thread's columns that are no filling: selects in the loop took 2 us of 87, backward, 4000 x 512 x 1368)
        const int live = a.live - col;
        const uint2 keep = make_uint2(live > 1 ? ~0u : live > 0 ? 0xffffu : 0u, live > 3 ? ~0u : live > 2 ? 0xffffu : 0u);
        if (col < a.m) {
#pragma unroll 4
            for (int tok = rank + S * (e / LANES); tok < last; tok += S * AT_ONCE) {
                const size_t row = (size_t)(t0 + tok), at = row * 2 * a.m + col;
                float v[4];
                if (EPI == RW_STORE) {
                    sum(tok, part_col, v);
                    store_bf16x4(a.out + row * a.m + col, v);
                } else if (EPI == RW_GLU) {
                    float up[4], h[4];
                    sum(tok, part_col, v);
                    sum(tok, 64 + part_col, up);
#pragma unroll
                    for (int j = 0; j < 4; ++j) h[j] = ffn_act<false>(v[j], a.act) * up[j];
                    store_bf16x4(a.out + row * a.m + col, h, keep);
                    if (a.gu) { store_bf16x4(a.gu + at, v); store_bf16x4(a.gu + at + a.m, up); }
                } else {
                    float g[4], up[4], dg[4], du[4], h[4];
                    load_bf16x4(a.kept + at, g);
                    load_bf16x4(a.kept + at + a.m, up);
                    sum(tok, part_col, v);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float da;
                        const float act = ffn_act_grad<false>(g[j], a.act, da);
                        dg[j] = v[j] * up[j] * da;
                        du[j] = v[j] * act;
                        h[j] = act * up[j];
                    }
                    store_bf16x4(a.gu + at, dg, keep);
                    store_bf16x4(a.gu + at + a.m, du, keep);
                    store_bf16x4(a.out + row * a.m + col, h, keep);
                }
            }
        }
    }

    // ---- teardown: nobody leaves while a peer may still read this CTA's partial tile ----
    if (S > 1) cluster_sync_all(); else __syncthreads();
    if (*abort_flag) {       // copies may be in flight: leave them time before the shared memory goes
        const uint64_t t = globaltimer_ns();
        while (globaltimer_ns() - t < 200000ull) { }
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, C::TMEM);
    }
}

int cdiv(int64_t x, int64_t y) { return (int)((x + y - 1) / y); }

// Tile width and split of the reduction: the pair with the least estimated time.  A CTA streams its stages at 70 KB/us (its ring over the
// latency), L2 gives 16 MB/us to all (10 with the reduction down the weights' columns), HBM 6.3 MB/us of weights (to narrow tiles from 165 CTAs up: one row, 4096 x 8192, 128 CTAs 41.7 us, 256 CTAs 36.7; 64 rows 43.5 and 51); two CTAs fit an SM; 3.2 us of launch, set-up and drain; 0.016 us a row for the
// partial tile and 0.036 us for each row that a CTA finishes.  (Within 20 % of what was measured for 16 to 512 rows, d and f of 512 to 8192.)
struct RowsPlan { int nt, s; double us; };
RowsPlan rows_plan(int64_t rows, int tiles, int chunks, int mn)
{
    RowsPlan best{16, 1, 1e30};
    for (int nt = 16; nt <= 128; nt *= 2) {
        if (nt > 16 && nt / 2 >= rows) break;
        const int64_t z = (rows + nt - 1) / nt;
        if (z > 65535) continue;
        for (int s = 1; s <= 8 && s <= chunks; s *= 2) {
            const double ctas = (double)tiles * z * s, per = cdiv(chunks, s), kb = 16.0 + nt / 8.0;
            const double cta = per * kb / 70.0 + 0.016 * nt + 0.036 * nt / s;
            double t = (double)(int64_t)((ctas + 295.0) / 296.0) * cta;
            t = std::max(t, ctas * per * kb / (mn ? 10000.0 : 16000.0));
            t = std::max(t, (double)tiles * chunks * 16.0 / (nt > 32 ? 6300.0 : std::min(6300.0, 1200.0 + 31.0 * ctas))) + 3.2;
            if (t < best.us) best = RowsPlan{nt, s, t};
        }
    }
    return best;
}

template <int NT, int EPI>
cudaError_t launch_rows(const RowsArgs& a, int tiles, int S, cudaStream_t st)
{
    using C = Rw<NT>;
    const int z = cdiv(a.rows, NT);
    const cudaError_t e = raise_smem_limit<ffn_rows_kernel<NT, EPI>>(C::SMEM);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(S, tiles, z);
    cfg.blockDim = dim3(RW_THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = S; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    ++kernels_launched();
    return cudaLaunchKernelEx(&cfg, ffn_rows_kernel<NT, EPI>, a);
}
template <int EPI>
sb_status launch_epi(RowsArgs& a, const void* rows, int64_t k, int tiles, cudaStream_t st)
{
    a.chunks = cdiv(k, 64);
    const RowsPlan plan = rows_plan(a.rows, tiles, a.chunks, a.a_mn);
    const int nt = plan.nt;
    if (!umma_map_rows(&a.t, rows, a.rows, (long)k, (long)k, nt)) return set_error(SB_ERR_CUDA, "ffn: %s", umma_last_error());
    a.status = ops_status();
    const cudaError_t e = nt == 16 ? launch_rows<16, EPI>(a, tiles, plan.s, st) : nt == 32 ? launch_rows<32, EPI>(a, tiles, plan.s, st)
                        : nt == 64 ? launch_rows<64, EPI>(a, tiles, plan.s, st) : launch_rows<128, EPI>(a, tiles, plan.s, st);
    return e == cudaSuccess ? SB_OK : set_error(SB_ERR_CUDA, "ffn: launch failed: %s", cudaGetErrorString(e));
}
bool weights(RowsArgs& a, const void* w, int64_t rows, int64_t cols, int mn)
{
    a.a_mn = mn;
    return umma_map_rows(&a.w, w, (long)rows, (long)cols, (long)cols, 64);
}
sb_status map_failed() { return set_error(SB_ERR_CUDA, "ffn: %s", umma_last_error()); }

}  // namespace

double ffn_rows_us(int64_t rows, int tiles, int chunks, int mn) { return rows_plan(rows, tiles, chunks, mn).us; }

sb_status ffn_rows_glu(const sb_ffn_config* c, const void* x, const void* w_gu, void* gu, __nv_bfloat16* h, int f_real, cudaStream_t st)
{
    RowsArgs a{};
    a.rows = (int)c->rows; a.m = c->f; a.live = f_real; a.w_split = c->f; a.act = c->act; a.out = h; a.gu = (__nv_bfloat16*)gu;
    if (!weights(a, w_gu, 2 * (int64_t)c->f, c->d, 0)) return map_failed();
    return launch_epi<RW_GLU>(a, x, c->d, cdiv(c->f, 64), st);
}
sb_status ffn_rows_down(const sb_ffn_config* c, const __nv_bfloat16* h, const void* w_down, void* y, cudaStream_t st)
{
    RowsArgs a{};
    a.rows = (int)c->rows; a.m = c->d; a.out = (__nv_bfloat16*)y; a.early = 1;
    if (!weights(a, w_down, c->d, c->f, 0)) return map_failed();
    return launch_epi<RW_STORE>(a, h, c->f, cdiv(c->d, 128), st);
}
sb_status ffn_rows_glu_back(const sb_ffn_config* c, const void* dy, const void* gu, const void* w_down, __nv_bfloat16* dgu, __nv_bfloat16* h, int f_real, cudaStream_t st)
{
    RowsArgs a{};
    a.rows = (int)c->rows; a.m = c->f; a.live = f_real; a.act = c->act; a.kept = (const __nv_bfloat16*)gu; a.gu = dgu; a.out = h;
    if (!weights(a, w_down, c->d, c->f, 1)) return map_failed();
    return launch_epi<RW_GLU_BACK>(a, dy, c->d, cdiv(c->f, 128), st);
}
sb_status ffn_rows_dx(const sb_ffn_config* c, const __nv_bfloat16* dgu, const void* w_gu, void* dx, cudaStream_t st)
{
    RowsArgs a{};
    a.rows = (int)c->rows; a.m = c->d; a.out = (__nv_bfloat16*)dx; a.early = 1;
    if (!weights(a, w_gu, 2 * (int64_t)c->f, c->d, 1)) return map_failed();
    return launch_epi<RW_STORE>(a, dgu, 2 * (int64_t)c->f, cdiv(c->d, 128), st);
}

}  // namespace sb
