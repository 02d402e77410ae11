// Gated feed-forward block on tensor cores (bf16; d and f multiples of eight): the products of large batches as 256 x 256 tiles on CTA pairs
// (tcgen05.mma.cta_group::2), persistent, with the activation and its derivative in the epilogue.
//
//   forward   1. GU = X Wgu^T, a tile holding 128 gate columns and the 128 up columns that belong to them; epilogue: H = a(G) * U (and GU, where the
//                backward pass will want it)
//             2. Y = H Wd^T
//   backward  1. dH = dY Wd; epilogue: dG, dU and H from dH and the kept GU
//             2. dX = [dG dU] Wgu, dWgu = [dG dU]^T X and dWd = dY^T H in one launch
//
// Operands are K-major or MN-major as they lie in memory (nothing is transposed): the shared-memory descriptors and the instruction descriptor say
// which, per problem.  A stage of the ring is 64 reduction steps: 128 x 64 of A and, since the MMA of a pair reads both CTAs' halves, 128 x 64 of B in
// each CTA.  Warps: 0 = TMA loads, 1 = TMEM and (leader) MMA, 2 .. 17 = epilogue, two groups of eight warps, each with half of the columns; two
// accumulators of 256 columns, so that a tile's epilogue runs beside the next tile's MMAs.  Epilogues stage 64-column pieces in the 128-byte swizzle and
// leave them to TMA stores, which also cut off what lies outside of the matrix.
//
// What bounds it: the tensor pipe, busy for 80 % (first product), 88 % (second) and 91 % (dX, dWgu, dWd) of the time, under the power cap when it lasts:
// 8192 rows, 4096 x 8192, forward 1095 to 1300 us (1.5 to 1.27 PFLOP/s), 4000 rows backward 1123 to 1340.  In turn with a library's plain products of the
// same operands: forward 1175 us here and 1214 there, 4000 rows 644 and 622, backward 1246 and 1254.  The derivative product (tensor pipe 62 %): the shared-memory port, which G, U, dG, dU and H pass beside the MMA's operands.  All waits are bounded and report through the operators' status word.
#include "sb_ffn.h"
#include "sb_ffn_umma.h"
#include "sb_tcgen05.cuh"
#include "sb_umma.h"

#include <algorithm>

namespace sb {

namespace {

constexpr int PT_THREADS = 64 + 512, PT_STAGE = 32768, PT_BOX = 16384, PT_CTRL = 1024, PT_MAX_STAGES = 6;
constexpr uint32_t PT_TMEM = 512;
constexpr int PT_SMEM_LIMIT = 227 * 1024;
enum { EPI_STORE = 0, EPI_GLU = 1, EPI_GLU_BACK = 2 };
__host__ __device__ constexpr int group_boxes(int epi) { return epi == EPI_STORE ? 2 : 3; }
__host__ __device__ constexpr int pair_stages(int epi) { return epi == EPI_STORE ? 5 : 4; }
__host__ __device__ constexpr int pair_smem(int epi) { return pair_stages(epi) * PT_STAGE + 2 * group_boxes(epi) * PT_BOX + 1024 + PT_CTRL; }
static_assert(pair_smem(EPI_STORE) <= PT_SMEM_LIMIT && pair_smem(EPI_GLU) <= PT_SMEM_LIMIT, "shared memory");

struct PairProblem {
    int a_mn, b_mn;            // operands as they lie: 0 = reduction along a row, 1 = reduction along a column
    int m, n, m_tiles, n_tiles, chunks, units;
    int out_f32;
    int b_split;               // rows between the two halves of a B tile (gate and up rows), or 0: 128 neighbouring columns each
};
struct alignas(64) PairArgs {
    CUtensorMap a[3], b[3], c[3];      // EPI_GLU: c = H, gate half and up half of GU; EPI_GLU_BACK: c = dG, dU, H
    CUtensorMap g, u;                  // EPI_GLU_BACK: the kept halves of GU
    PairProblem p[3];
    int count;
    // Units of the first problem go round the pairs; of its last, incomplete round the pairs without a unit take `extra` units of the other problems
    // each before these go round in turn (dX's reductions are several times as long as those of the weight gradients).
    int pairs, first, rest, odd, extra;
    int save;
    int stages, slots;                 // EPI_STORE
    uint32_t* status;
};

// The i-th unit of pair q, or -1
__device__ __forceinline__ int unit_at(const PairArgs& a, int q, int i)
{
    const int mine = q < a.first ? (a.first - q + a.pairs - 1) / a.pairs : 0;
    if (i < mine) return q + i * a.pairs;
    i -= mine;
    if (q >= a.odd) {
        if (i < a.extra) return a.first + i * (a.pairs - a.odd) + (q - a.odd);
        i -= a.extra;
    }
    const int at = a.extra * (a.pairs - a.odd) + i * a.pairs + q;
    return at < a.rest ? a.first + at : -1;
}
// Unit -> problem and tile: bands of eight row tiles, column by column, so that the pairs at work share operands in L2
__device__ __forceinline__ int tile_of(const PairArgs& a, int u, int& mt, int& nt)
{
    int k = 0;
    while (k + 1 < a.count && u >= a.p[k].units) u -= a.p[k++].units;
    const PairProblem& p = a.p[k];
    const int per = 8 * p.n_tiles, band = u / per, r = u - band * per, rows = min(8, p.m_tiles - band * 8);
    nt = r / rows;
    mt = band * 8 + (r - nt * rows);
    return k;
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *(const uint32_t*)&b;
}
__device__ __forceinline__ void st_shared16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void ld_shared16(uint32_t at, uint32_t (&v)[4])
{
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
}
// 16-byte piece c of row r in a box of 128-byte rows with the 128-byte swizzle
__device__ __forceinline__ uint32_t piece(uint32_t box, int r, int c) { return box + (uint32_t)r * 128u + (uint32_t)((c ^ (r & 7)) << 4); }

// 16 columns of one row as two pieces of bf16
__device__ __forceinline__ void stage_bf16(uint32_t box, int r, int c, const float (&v)[16])
{
    st_shared16(piece(box, r, c), pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
    st_shared16(piece(box, r, c + 1), pack2(v[8], v[9]), pack2(v[10], v[11]), pack2(v[12], v[13]), pack2(v[14], v[15]));
}

template <int EPI, int ACT>
__global__ void __launch_bounds__(PT_THREADS, 1)
ffn_pair_kernel(const __grid_constant__ PairArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    constexpr int BOXES = group_boxes(EPI);
    // (a fifth of the shared memory is a second set of staging boxes where tiles are short, else two more stages)
    const int ST = EPI == EPI_STORE ? a.stages : pair_stages(EPI), SLOTS = EPI == EPI_STORE ? a.slots : 1;
    uint8_t* stage_out = smem + ST * PT_STAGE;
    uint8_t* ctrl = smem + pair_stages(EPI) * PT_STAGE + 2 * BOXES * PT_BOX;
    uint64_t* full = (uint64_t*)ctrl;                 // [ST]
    uint64_t* empty = full + PT_MAX_STAGES;           // [ST]
    uint64_t* acc_full = empty + PT_MAX_STAGES;       // [2]
    uint64_t* acc_empty = acc_full + 2;               // [2]
    uint64_t* kept = acc_empty + 2;                   // [2]: a group's pieces of GU have arrived
    uint32_t* tmem_slot = (uint32_t*)(kept + 2);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    volatile uint32_t* epi_stop = tmem_slot + 2;      // [2]: written by the warps of one epilogue group only
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    const int q = blockIdx.x / 2;
    const uint32_t smem0 = smem_u32(smem);

    if (threadIdx.x == 0) {
        for (int s = 0; s < ST; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(&acc_full[s], 1); mbar_init(&acc_empty[s], 4); mbar_init(&kept[s], 1); epi_stop[s] = 0; }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    cluster_sync_all();    // both CTAs' barriers exist before any copy or commit can signal them
    if (warp == 1) {
        tmem_alloc_pair(tmem_slot, PT_TMEM);
        tmem_relinquish_pair();
    }
    pdl_wait();
    if (warp == 0) pdl_trigger();
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();    // the peer's accumulator columns are allocated before the leader's first MMA writes them
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    if (warp == 0) {
        // ---- loads: own 128 rows of A, own half of B ----
        const uint32_t el = elect_one() ? 1u : 0u;
        const uint32_t full0 = smem_u32(full), full_l = map_to_cta(full0, 0);
        int s = 0;
        uint32_t ph = 1u;
        bool ok = true;
        for (int i = 0; ok; ++i) {
            const int u = unit_at(a, q, i);
            if (u < 0) break;
            int mt, nt;
            const int k = tile_of(a, u, mt, nt);
            const PairProblem& p = a.p[k];
            const int m0 = mt * 256 + (int)rank * 128, n0 = p.b_split ? nt * 128 + (int)rank * p.b_split : nt * 256 + (int)rank * 128;
            const CUtensorMap *ma = &a.a[k], *mb = &a.b[k];
            const int a_mn = p.a_mn, b_mn = p.b_mn, chunks = p.chunks;
            for (int c = 0; c < chunks; ++c) {
                ok = __all_sync(0xffffffffu, mbar_wait(&empty[s], ph) ? 1 : 0) != 0;
                if (!ok) break;
                const uint32_t dst = smem0 + (uint32_t)(s * PT_STAGE), bar = full_l + 8u * (uint32_t)s;
                if (leader) mbar_expect_tx_el(full0 + 8u * (uint32_t)s, 2u * PT_STAGE, el);
                if (!a_mn) tma_load_4d_pair_el(ma, dst, bar, c * 64, m0, 0, 0, el);
                else {
                    tma_load_4d_pair_el(ma, dst, bar, m0, c * 64, 0, 0, el);
                    tma_load_4d_pair_el(ma, dst + 8192u, bar, m0 + 64, c * 64, 0, 0, el);
                }
                if (!b_mn) tma_load_4d_pair_el(mb, dst + PT_BOX, bar, c * 64, n0, 0, 0, el);
                else {
                    tma_load_4d_pair_el(mb, dst + PT_BOX, bar, n0, c * 64, 0, 0, el);
                    tma_load_4d_pair_el(mb, dst + PT_BOX + 8192u, bar, n0 + 64, c * 64, 0, 0, el);
                }
                if (++s == ST) { s = 0; ph ^= 1u; }
            }
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicMax(a.status, (uint32_t)DEV_TIMEOUT_TMA); }
        __syncwarp();
    } else if (warp == 1) {
        if (leader) {
            const uint32_t el = elect_one() ? 1u : 0u;
            // the MMA addresses both accumulators with one TMEM address: the pair must have been given the same columns
            const bool tmem_ok = ld_cluster_u32(map_to_cta(smem_u32(tmem_slot), 1)) == tmem_base;
            bool ok = tmem_ok;
            if (!ok && lane == 0) { *abort_flag = 1; atomicMax(a.status, (uint32_t)DEV_PAIR_TMEM); }
            int s = 0;
            uint32_t ph = 0u;
            for (int i = 0; ok; ++i) {
                const int u = unit_at(a, q, i);
                if (u < 0) break;
                int mt, nt;
                const PairProblem& p = a.p[tile_of(a, u, mt, nt)];
                const int chunks = p.chunks, buf = i & 1;
                const uint32_t idesc = make_idesc(256, p.a_mn, p.b_mn, 256);
                const uint64_t dA = make_desc(smem0, p.a_mn ? 8192 : 16), dB = make_desc(smem0 + PT_BOX, p.b_mn ? 8192 : 16);
                const uint32_t a_hi = (uint32_t)(dA >> 32), b_hi = (uint32_t)(dB >> 32), a_step = p.a_mn ? 128u : 2u, b_step = p.b_mn ? 128u : 2u;
                ok = __all_sync(0xffffffffu, mbar_wait(&acc_empty[buf], (uint32_t)(((i >> 1) + 1) & 1)) ? 1 : 0) != 0;
                if (!ok) break;
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + (uint32_t)(buf * 256);
                for (int c = 0; c < chunks; ++c) {
                    ok = __all_sync(0xffffffffu, mbar_wait(&full[s], ph) ? 1 : 0) != 0;
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t off = (uint32_t)(s * PT_STAGE) >> 4;
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        umma_bf16_pair_lohi(d_tmem, (uint32_t)dA + off + a_step * kk, a_hi, (uint32_t)dB + off + b_step * kk, b_hi, idesc, (c > 0 || kk > 0) ? 1u : 0u, el);
                    if (el) umma_commit_pair(&empty[s]);
                    __syncwarp();
                    if (++s == ST) { s = 0; ph ^= 1u; }
                }
                if (!ok) break;
                if (el) umma_commit_pair(&acc_full[buf]);
                __syncwarp();
            }
            if (tmem_ok && !ok && lane == 0) { *abort_flag = 1; atomicMax(a.status, (uint32_t)DEV_TIMEOUT_MMA); }
            __syncwarp();
        }
    } else {
        // ---- epilogue: own 128 rows, half of the columns a group ----
        // (two warps of a group share a TMEM lane quadrant: `side` says which columns of a 64-column piece are this one's)
        const int quad = warp % 4, group = (warp - 2) / 8, side = (warp - 2) / 4 % 2, row = quad * 32 + lane;
        const bool first = (threadIdx.x - 64) % 256 == 0;
        auto group_sync = [&]() { asm volatile("bar.sync %0, 256;" ::"r"(1 + group) : "memory"); };
        const uint32_t acc_empty_l = map_to_cta(smem_u32(acc_empty), 0), boxes = smem_u32(stage_out) + (uint32_t)(group * SLOTS * BOXES * PT_BOX);
        uint32_t box0 = boxes;
        int slot = 0;
        const uint32_t kept_bar = smem_u32(&kept[group]);
        uint32_t kept_ph = 0u;
        bool ok = true;
        // a timeout seen by one warp of the group is seen by all
        auto agree = [&]() -> bool {
            if (!ok && lane == 0) { epi_stop[group] = 1; *abort_flag = 1; atomicMax(a.status, (uint32_t)DEV_TIMEOUT_EPI); }
            group_sync();
            return epi_stop[group] == 0;
        };
        auto drained = [&](int buf) {         // this group has read its part of the accumulator
            asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(acc_empty_l + 8u * (uint32_t)buf) : "memory");
        };
        for (int i = 0;; ++i) {
            const int u = unit_at(a, q, i);
            if (u < 0) break;
            int mt, nt;
            const int k = tile_of(a, u, mt, nt);
            const PairProblem& p = a.p[k];
            const int buf = i & 1, m0 = mt * 256 + (int)rank * 128;
            const uint32_t acc = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(buf * 256);
            const bool rows_in = m0 < p.m;
            if (EPI == EPI_GLU_BACK && first) {           // the first 64 columns' G and U, into the pieces that their gradients will replace
                tma_store_wait_read();
                mbar_arrive_expect_tx(kept_bar, 2u * PT_BOX);
                tma_load_4d_el(&a.g, box0, kept_bar, nt * 256 + group * 128, m0, 0, 0, 1u);
                tma_load_4d_el(&a.u, box0 + PT_BOX, kept_bar, nt * 256 + group * 128, m0, 0, 0, 1u);
            }
            if (lane == 0) ok = mbar_wait(&acc_full[buf], (uint32_t)((i >> 1) & 1));
            ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
            // the tile that was in these staging boxes has left them
            auto boxes_free = [&]() { if (SLOTS > 1) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); else tma_store_wait_read(); };
            auto next_boxes = [&]() { if (SLOTS > 1) { slot ^= 1; box0 = boxes + (uint32_t)(slot * BOXES * PT_BOX); } };
            if (EPI != EPI_GLU_BACK && first) boxes_free();
            if (!agree()) break;
            tc_fence_after();
            if (EPI == EPI_GLU) {
                const int n0 = nt * 128 + group * 64;
#pragma unroll 1
                for (int c = 2 * side; c < 2 * side + 2; ++c) {
                    uint32_t gv[16], uv[16];
                    tmem_ld16(acc + (uint32_t)(group * 64 + c * 16), gv);
                    tmem_ld16(acc + (uint32_t)(128 + group * 64 + c * 16), uv);
                    tmem_ld_wait();
                    float g[16], up[16], h[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        g[j] = __uint_as_float(gv[j]); up[j] = __uint_as_float(uv[j]);
                        h[j] = ffn_act<false>(g[j], ACT) * up[j];
                    }
                    stage_bf16(box0, row, 2 * c, h);
                    if (a.save) { stage_bf16(box0 + PT_BOX, row, 2 * c, g); stage_bf16(box0 + 2 * PT_BOX, row, 2 * c, up); }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                tc_fence_before();
                group_sync();
                if (first) {
                    drained(buf);
                    if (rows_in && n0 < p.n)
                        for (int b = 0; b < (a.save ? 3 : 1); ++b) tma_store_4d(&a.c[b], box0 + (uint32_t)(b * PT_BOX), n0, m0, 0, 0);
                    tma_store_commit();
                }
            } else if (EPI == EPI_GLU_BACK) {
                for (int half = 0; half < 2; ++half) {
                    const int n0 = nt * 256 + group * 128 + half * 64;
                    if (half == 1) {
                        if (first) {
                            tma_store_wait_read();
                            mbar_arrive_expect_tx(kept_bar, 2u * PT_BOX);
                            tma_load_4d_el(&a.g, box0, kept_bar, n0, m0, 0, 0, 1u);
                            tma_load_4d_el(&a.u, box0 + PT_BOX, kept_bar, n0, m0, 0, 0, 1u);
                        }
                    }
                    if (lane == 0) ok = mbar_wait(&kept[group], kept_ph);
                    ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
                    kept_ph ^= 1u;
                    if (!agree()) break;
#pragma unroll 1
                    for (int c = 2 * side; c < 2 * side + 2; ++c) {
                        uint32_t dv[16], gw[8], uw[8];
                        tmem_ld16(acc + (uint32_t)(group * 128 + half * 64 + c * 16), dv);
                        ld_shared16(piece(box0, row, 2 * c), *(uint32_t(*)[4])&gw[0]);
                        ld_shared16(piece(box0, row, 2 * c + 1), *(uint32_t(*)[4])&gw[4]);
                        ld_shared16(piece(box0 + PT_BOX, row, 2 * c), *(uint32_t(*)[4])&uw[0]);
                        ld_shared16(piece(box0 + PT_BOX, row, 2 * c + 1), *(uint32_t(*)[4])&uw[4]);
                        tmem_ld_wait();
                        float dg[16], du[16], h[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const uint32_t gb = j % 2 ? gw[j / 2] & 0xffff0000u : gw[j / 2] << 16, ub = j % 2 ? uw[j / 2] & 0xffff0000u : uw[j / 2] << 16;
                            const float up = __uint_as_float(ub), dh = __uint_as_float(dv[j]);
                            float da;
                            const float act = ffn_act_grad<false>(__uint_as_float(gb), ACT, da);
                            dg[j] = dh * up * da;
                            du[j] = dh * act;
                            h[j] = act * up;
                        }
                        stage_bf16(box0, row, 2 * c, dg);
                        stage_bf16(box0 + PT_BOX, row, 2 * c, du);
                        stage_bf16(box0 + 2 * PT_BOX, row, 2 * c, h);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    tc_fence_before();
                    group_sync();
                    if (first) {
                        if (half == 1) drained(buf);
                        if (rows_in && n0 < p.n)
#pragma unroll
                            for (int b = 0; b < 3; ++b) tma_store_4d(&a.c[b], box0 + (uint32_t)(b * PT_BOX), n0, m0, 0, 0);
                        tma_store_commit();
                    }
                }
                if (!ok || epi_stop[group]) break;
            } else {
                const int n0 = nt * 256 + group * 128;
                if (!p.out_f32) {
#pragma unroll 1
                    for (int c = 4 * side; c < 4 * side + 4; ++c) {
                        uint32_t v[16];
                        tmem_ld16(acc + (uint32_t)(group * 128 + c * 16), v);
                        tmem_ld_wait();
                        float f[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) f[j] = __uint_as_float(v[j]);
                        stage_bf16(box0 + (uint32_t)(c / 4) * PT_BOX, row, 2 * (c % 4), f);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    tc_fence_before();
                    group_sync();
                    if (first) {
                        drained(buf);
                        for (int b = 0; b < 2; ++b)
                            if (rows_in && n0 + 64 * b < p.n) tma_store_4d(&a.c[k], box0 + (uint32_t)(b * PT_BOX), n0 + 64 * b, m0, 0, 0);
                        tma_store_commit();
                    }
                    next_boxes();
                } else {
                    for (int half = 0; half < 2; ++half) {       // 64 columns at a time, boxes of 32
                        if (half == 1) {
                            if (first) boxes_free();
                            group_sync();
                        }
#pragma unroll 1
                        for (int c = 2 * side; c < 2 * side + 2; ++c) {
                            uint32_t v[16];
                            tmem_ld16(acc + (uint32_t)(group * 128 + half * 64 + c * 16), v);
                            tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                st_shared16(piece(box0 + (uint32_t)(c / 2) * PT_BOX, row, 4 * (c % 2) + j), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        tc_fence_before();
                        group_sync();
                        if (first) {
                            if (half == 1) drained(buf);
                            for (int b = 0; b < 2; ++b)
                                if (rows_in && n0 + 64 * half + 32 * b < p.n) tma_store_4d(&a.c[k], box0 + (uint32_t)(b * PT_BOX), n0 + 64 * half + 32 * b, m0, 0, 0);
                            tma_store_commit();
                        }
                        next_boxes();
                    }
                }
            }
        }
        if (first) tma_store_wait_read();
    }

    // ---- teardown: everyone meets here; TMEM is released on every path ----
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {       // copies may be in flight: leave them time before the shared memory goes
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200000ull) { }
        __syncthreads();
    }
    cluster_sync_all();    // neither CTA leaves (or frees TMEM) while its partner may still signal or read it
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, PT_TMEM);
    }
}

int cdiv(int64_t x, int64_t y) { return (int)((x + y - 1) / y); }

template <int EPI, int ACT>
cudaError_t launch_pair(PairArgs& a, cudaStream_t st)
{
    a.first = a.p[0].units;
    a.rest = 0;
    for (int k = 1; k < a.count; ++k) a.rest += a.p[k].units;
    const int all = a.first + a.rest;
    if (all == 0) return cudaSuccess;
    a.pairs = std::min(74, all);
    a.odd = a.first % a.pairs;
    a.extra = 0;
    if (a.rest > 0 && a.odd > 0) a.extra = std::min((a.p[0].chunks + a.p[1].chunks / 2) / std::max(1, a.p[1].chunks), a.rest / (a.pairs - a.odd));
    // short tiles: their time is the epilogue's, which two sets of staging boxes let run on (weight gradients of 4096 x 8192 over 16 rows: 68 us with one
    // set, 60 with two; of 2048 x 2048 over 512 rows, eight chunks: 16.3 and 18)
    int longest = 0;
    for (int k = 0; k < a.count; ++k) longest = std::max(longest, a.p[k].chunks);
    a.slots = longest <= 4 ? 2 : 1;
    a.stages = a.slots == 2 ? 3 : 5;
    a.status = ops_status();
    const cudaError_t e = raise_smem_limit<ffn_pair_kernel<EPI, ACT>>(pair_smem(EPI));
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(2 * a.pairs);
    cfg.blockDim = dim3(PT_THREADS);
    cfg.dynamicSmemBytes = (size_t)pair_smem(EPI);
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    ++kernels_launched();
    return cudaLaunchKernelEx(&cfg, ffn_pair_kernel<EPI, ACT>, a);
}

template <int EPI>
cudaError_t launch_pair_act(PairArgs& a, int act, cudaStream_t st)
{
    return act == SB_ACT_SILU ? launch_pair<EPI, SB_ACT_SILU>(a, st) : act == SB_ACT_GELU ? launch_pair<EPI, SB_ACT_GELU>(a, st) : launch_pair<EPI, SB_ACT_RELU>(a, st);
}

// An operand [rows, cols] (rows ld apart): the reduction runs along its rows' columns (mn = 0: boxes of 128 rows) or down its rows (mn = 1: of 64).
bool operand(CUtensorMap* map, const void* p, int64_t rows, int64_t cols, int mn) { return umma_map_rows(map, p, (long)rows, (long)cols, (long)cols, mn ? 64 : 128); }
PairProblem problem(int64_t m, int64_t n, int64_t k, int a_mn, int b_mn)
{
    PairProblem p{};
    p.a_mn = a_mn; p.b_mn = b_mn; p.m = (int)m; p.n = (int)n; p.m_tiles = cdiv(m, 256); p.n_tiles = cdiv(n, 256); p.chunks = cdiv(k, 64);
    p.units = p.m_tiles * p.n_tiles;
    return p;
}

size_t h_bytes(const sb_ffn_config* c) { return ((size_t)c->rows * c->f * 2 + 255) / 256 * 256; }

sb_status map_failed() { return set_error(SB_ERR_CUDA, "ffn: %s", umma_last_error()); }
sb_status launched(cudaError_t e) { return e == cudaSuccess ? SB_OK : set_error(SB_ERR_CUDA, "ffn: launch failed: %s", cudaGetErrorString(e)); }

}  // namespace

// Which products run on sb_ffn_rows.cu: those whose estimate there is the shorter one.  Here: 6 us of launch, set-up and the last tile's epilogue (10 with
// the derivative), 0.33 us a chunk and 2 us (5) of epilogue that hides nothing for each round of tiles over the pairs.
// (4096 x 8192, forward: 256 rows 62.6 us there and 79.8 here, 512 rows 115 and 101; 1024 x 4096, 512 rows: 27.6 and 35.5, 1024 rows: 42.4 and 41.3.)
static bool on_rows(int64_t rows, int row_tiles, int mn, const PairProblem& p, bool back)
{
#ifdef SB_DEV_TUNING
    const int force = (int)tune("SB_FEW_ROWS", -1);
    if (force >= 0) return rows <= force;
#endif
    const double here = (back ? 10.0 : 6.0) + cdiv(p.units, 74) * (0.33 * p.chunks + (back ? 5.0 : 2.0));
    return ffn_rows_us(rows, row_tiles, p.chunks, mn) < here;
}

bool ffn_umma_ok(const sb_ffn_config* c) { return c->precision == SB_BF16 && c->d % 8 == 0 && c->f % 8 == 0; }

__nv_bfloat16* ffn_umma_h(const sb_ffn_config*, void* ws) { return (__nv_bfloat16*)ws; }
__nv_bfloat16* ffn_umma_dgu(const sb_ffn_config* c, void* ws) { return (__nv_bfloat16*)((char*)ws + h_bytes(c)); }
size_t ffn_umma_bytes(const sb_ffn_config* c, bool backward) { return backward ? 3 * h_bytes(c) : h_bytes(c); }

sb_status ffn_umma_forward(const sb_ffn_config* c, const void* x, const void* w_gu, const void* w_down, void* gu, void* y, void* ws, int f_real,
                           cudaStream_t st)
{
    const int64_t R = c->rows, D = c->d, F = c->f;
    __nv_bfloat16* h = ffn_umma_h(c, ws);
    static thread_local PairArgs a;
    a = PairArgs{};
    a.count = 1; a.save = gu != nullptr;
    a.p[0] = problem(R, F, D, 0, 0);
    a.p[0].b_split = (int)F;
    a.p[0].n_tiles = cdiv(F, 128);
    a.p[0].units = a.p[0].m_tiles * a.p[0].n_tiles;
    sb_status s = SB_OK;
    if (on_rows(R, cdiv(F, 64), 0, a.p[0], false)) s = ffn_rows_glu(c, x, w_gu, gu, h, f_real, st);
    else {
        bool ok = operand(&a.a[0], x, R, D, 0) && operand(&a.b[0], w_gu, 2 * F, D, 0) && umma_map_rows(&a.c[0], h, (long)R, f_real, (long)F, 128);
        if (ok && gu) ok = umma_map_rows(&a.c[1], gu, (long)R, (long)F, (long)(2 * F), 128) && umma_map_rows(&a.c[2], (const __nv_bfloat16*)gu + F, (long)R, (long)F, (long)(2 * F), 128);
        if (!ok) return map_failed();
        s = launched(launch_pair_act<EPI_GLU>(a, c->act, st));
    }
    if (s != SB_OK) return s;
    a = PairArgs{};
    a.count = 1;
    a.p[0] = problem(R, D, F, 0, 0);
    if (on_rows(R, cdiv(D, 128), 0, a.p[0], false)) return ffn_rows_down(c, h, w_down, y, st);
    if (!operand(&a.a[0], h, R, F, 0) || !operand(&a.b[0], w_down, D, F, 0) || !umma_map_rows(&a.c[0], y, (long)R, (long)D, (long)D, 128)) return map_failed();
    return launched(launch_pair<EPI_STORE, 0>(a, st));
}

sb_status ffn_umma_backward(const sb_ffn_config* c, const void* dy, const void* x, const void* gu, const void* w_gu, const void* w_down, void* dx, void* dw_gu,
                            void* dw_down, void* ws, int f_real, cudaStream_t st)
{
    const int64_t R = c->rows, D = c->d, F = c->f;
    __nv_bfloat16 *h = ffn_umma_h(c, ws), *dgu = ffn_umma_dgu(c, ws);
    const __nv_bfloat16* kept = (const __nv_bfloat16*)gu;
    static thread_local PairArgs a;
    a = PairArgs{};
    a.count = 1;
    a.p[0] = problem(R, F, D, 0, 1);
    sb_status s = SB_OK;
    if (on_rows(R, cdiv(F, 128), 1, a.p[0], true)) s = ffn_rows_glu_back(c, dy, gu, w_down, dgu, h, f_real, st);
    else {
        bool ok = operand(&a.a[0], dy, R, D, 0) && operand(&a.b[0], w_down, D, F, 1);
        ok = ok && umma_map_rows(&a.g, kept, (long)R, (long)F, (long)(2 * F), 128) && umma_map_rows(&a.u, kept + F, (long)R, (long)F, (long)(2 * F), 128);
        ok = ok && umma_map_rows(&a.c[0], dgu, (long)R, f_real, (long)(2 * F), 128) && umma_map_rows(&a.c[1], dgu + F, (long)R, f_real, (long)(2 * F), 128) &&
             umma_map_rows(&a.c[2], h, (long)R, f_real, (long)F, 128);
        if (!ok) return map_failed();
        s = launched(launch_pair_act<EPI_GLU_BACK>(a, c->act, st));
    }
    if (s != SB_OK) return s;
    const bool dx_rows = dx && on_rows(R, cdiv(D, 128), 1, problem(R, D, 2 * F, 0, 1), false);
    if (dx_rows && (s = ffn_rows_dx(c, dgu, w_gu, dx, st)) != SB_OK) return s;
    a = PairArgs{};
    const bool f32 = c->grad_dtype == SB_DT_F32;
    auto out = [&](CUtensorMap* map, void* p, int64_t rows, int64_t cols) {
        return f32 ? umma_map_f32_rows(map, p, (long)rows, (long)cols, 128) : umma_map_rows(map, p, (long)rows, (long)cols, (long)cols, 128);
    };
    if (dx && !dx_rows) {
        const int k = a.count++;
        a.p[k] = problem(R, D, 2 * F, 0, 1);
        if (!operand(&a.a[k], dgu, R, 2 * F, 0) || !operand(&a.b[k], w_gu, 2 * F, D, 1) || !umma_map_rows(&a.c[k], dx, (long)R, (long)D, (long)D, 128)) return map_failed();
    }
    if (dw_gu) {
        const int k = a.count++;
        a.p[k] = problem(2 * F, D, R, 1, 1);
        a.p[k].out_f32 = f32;
        if (!operand(&a.a[k], dgu, R, 2 * F, 1) || !operand(&a.b[k], x, R, D, 1) || !out(&a.c[k], dw_gu, 2 * F, D)) return map_failed();
    }
    if (dw_down) {
        const int k = a.count++;
        a.p[k] = problem(D, F, R, 1, 1);
        a.p[k].out_f32 = f32;
        if (!operand(&a.a[k], dy, R, D, 1) || !operand(&a.b[k], h, R, F, 1) || !out(&a.c[k], dw_down, D, F)) return map_failed();
    }
    return a.count ? launched(launch_pair<EPI_STORE, 0>(a, st)) : SB_OK;
}

}  // namespace sb
