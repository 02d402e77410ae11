// Device side of the norms around a block that both directions share (sb_norm.cu, sb_norm_backward.cuh): parameters, how rows fall to CTAs, loads and stores
// of a thread's columns, sums over a team of warps, the ring of rows in shared memory.
#pragma once

#include "sb_f32x2.cuh"
#include "sb_ffn.h"
#include "sb_norm.h"
#include "sb_tcgen05.cuh"

namespace sb {

constexpr int MAX_D = 16384, THREADS = 512, WARPS = THREADS / 32, MAX_STAGES = 4;
constexpr int RING_LIMIT = 208 * 1024;

struct NormParams {
    const void *x, *f, *dy, *dn;
    const float *w_pre, *w_post, *gate, *scale;
    void *y, *n, *dx, *df;
    float* stats;                 // [rows][4]: mean and inv of f, mean and inv of y
    float *part, *gate_out;       // backward: [chunk][3][d] sums of dwpre, dwpost, ds; [groups or chunks][d] of dg
    int64_t rows, per_group, chunk;      // rows of a gate; rows of a CTA's turn
    int chunks_per_group;         // > 1: a group's rows fall to that many turns (chunk of them each, the last one fewer)
    int64_t turns;
    int team, teams;              // warps of a team, teams of a CTA
    int each, extra;              // teams of a CTA that have turns: one more in the first `extra` CTAs
    int stages, stage_rows, stage_bytes;     // ring of a team (stages = 0: none)
    int vec;                      // 16-byte accesses throughout
    int arrays;                   // row arrays in it
    int gate_ring;                // the gate has a row for every row: it comes through the ring too
    uint32_t* status;
    int d, relu_x;                // relu_x: dx is zero where x <= 0 (x is the output of a ReLU layer)
    float eps, rd;                // rd = 1 / d
};

namespace {

// What a kernel computes: any of the parts (looked at as it runs), all of them (both norms, both gradients), or the norm in front of a block alone.
enum { ANY_PARTS = 0, ALL_PARTS = 1, PRE_ONLY = 2 };

// Where a thread's columns come from: the ring in shared memory, global memory in 16-byte pieces, or global memory element by element.
enum { BY_RING = 0, BY_PIECES = 1, BY_ELEMENT = 2 };
struct Place { int t, width; };              // thread of its team, threads of the team
// Column j (0 .. 7) of piece c.  bf16: eight consecutive ones; float: two runs of four; by element: `width` apart.
template <typename T, int BY> __device__ __forceinline__ int column(Place w, int c, int j)
{
    return BY == BY_ELEMENT ? (c * 8 + j) * w.width + w.t : sizeof(T) == 2 ? (c * w.width + w.t) * 8 + j : ((c * 2 + j / 4) * w.width + w.t) * 4 + j % 4;
}
__device__ __forceinline__ void unpack(const uint4& a, F2 (&o)[4])
{
    const uint32_t b[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = f2(__uint_as_float(b[j] << 16), __uint_as_float(b[j] & 0xffff0000u));
}
// A vector's columns (float, in the order of T's), `fill` beyond d or without a vector
template <typename T, int BY> __device__ __forceinline__ void get_vector(const float* p, Place w, int c, int d, float fill, F2 (&o)[4])
{
#pragma unroll
    for (int j = 0; j < 8; j += BY == BY_ELEMENT ? 2 : 4) {
        const int i = column<T, BY>(w, c, j);
        if (BY == BY_ELEMENT) {
            const int i2 = column<T, BY>(w, c, j + 1);
            o[j / 2] = f2(p && i < d ? p[i] : fill, p && i2 < d ? p[i2] : fill);
        } else {
            float4 a = make_float4(fill, fill, fill, fill);
            if (p && i < d) a = *(const float4*)(p + i);
            o[j / 2] = f2(a.x, a.y);
            o[j / 2 + 1] = f2(a.z, a.w);
        }
    }
}
template <typename T, int BY> __device__ __forceinline__ void put_vector(float* p, Place w, int c, int d, const F2 (&v)[4])
{
#pragma unroll
    for (int j = 0; j < 8; j += BY == BY_ELEMENT ? 2 : 4) {
        const int i = column<T, BY>(w, c, j);
        if (BY == BY_ELEMENT) {
            const int i2 = column<T, BY>(w, c, j + 1);
            if (i < d) p[i] = lo(v[j / 2]);
            if (i2 < d) p[i2] = hi(v[j / 2]);
        } else if (i < d) *(float4*)(p + i) = make_float4(lo(v[j / 2]), hi(v[j / 2]), lo(v[j / 2 + 1]), hi(v[j / 2 + 1]));
    }
}
// A row's columns, zero beyond d
__device__ __forceinline__ uint4 lds16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
template <typename T> __device__ __forceinline__ void get_ring(uint32_t row, Place w, int c, int d, F2 (&o)[4])
{
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    if (sizeof(T) == 2) {
        const int i = column<T, BY_RING>(w, c, 0);
        unpack(i < d ? lds16(row + (uint32_t)i * 2u) : zero, o);
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = column<T, BY_RING>(w, c, 4 * h);
            const uint4 a = i < d ? lds16(row + (uint32_t)i * 4u) : zero;
            o[2 * h] = f2(__uint_as_float(a.x), __uint_as_float(a.y));
            o[2 * h + 1] = f2(__uint_as_float(a.z), __uint_as_float(a.w));
        }
    }
}
template <int BY> __device__ __forceinline__ void get_row(const float* p, Place w, int c, int d, F2 (&o)[4]) { get_vector<float, BY>(p, w, c, d, 0.f, o); }
template <int BY> __device__ __forceinline__ void get_row(const __nv_bfloat16* p, Place w, int c, int d, F2 (&o)[4])
{
    if (BY == BY_ELEMENT) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = column<__nv_bfloat16, BY>(w, c, 2 * j), i2 = column<__nv_bfloat16, BY>(w, c, 2 * j + 1);
            o[j] = f2(i < d ? __bfloat162float(p[i]) : 0.f, i2 < d ? __bfloat162float(p[i2]) : 0.f);
        }
    } else {
        const int i = column<__nv_bfloat16, BY>(w, c, 0);
        unpack(i < d ? *(const uint4*)(p + i) : make_uint4(0u, 0u, 0u, 0u), o);
    }
}
template <int BY> __device__ __forceinline__ void put_row(float* p, Place w, int c, int d, const F2 (&v)[4]) { put_vector<float, BY>(p, w, c, d, v); }
template <int BY> __device__ __forceinline__ void put_row(__nv_bfloat16* p, Place w, int c, int d, const F2 (&v)[4])
{
    if (BY == BY_ELEMENT) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = column<__nv_bfloat16, BY>(w, c, 2 * j), i2 = column<__nv_bfloat16, BY>(w, c, 2 * j + 1);
            if (i < d) p[i] = __float2bfloat16_rn(lo(v[j]));
            if (i2 < d) p[i2] = __float2bfloat16_rn(hi(v[j]));
        }
    } else {
        uint32_t o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) { const __nv_bfloat162 b = __floats2bfloat162_rn(lo(v[j]), hi(v[j])); o[j] = *(const uint32_t*)&b; }
        const int i = column<__nv_bfloat16, BY>(w, c, 0);
        if (i < d) *(uint4*)(p + i) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// Sums over a team, through partial sums of its warps; every thread gets them.  The two halves of `buf` are used in turn, so that one barrier a call is
// enough; it also says that the whole team has read the row.  Slots of warps that a team does not have stay zero.
struct Team {
    float* buf;              // [2][K][16]
    int id, warps, warp, turn = 0;
    __device__ __forceinline__ void barrier() const { if (warps > 1) asm volatile("bar.sync %0, %1;" ::"r"(1 + id), "r"(32 * warps) : "memory"); else __syncwarp(); }
};
__device__ __forceinline__ float team_sum(Team& t, float v)
{
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (t.warps == 1) return v;
    float* b = t.buf + t.turn * 16;
    t.turn ^= 1;
    if (lane == 0) b[t.warp] = v;
    t.barrier();
    v = b[lane % 16];
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// K (4 or 8) values at once: each step of the warp's butterfly halves the values a lane still carries, so that K - 1 + log2(32 / K) shuffles do.
template <int K>
__device__ __forceinline__ void team_sum(Team& t, float (&v)[K])
{
    const int lane = threadIdx.x % 32;
    int step = 16;
#pragma unroll
    for (int n = K; n > 1; n /= 2, step /= 2) {
        const bool up = lane & step;
#pragma unroll
        for (int k = 0; k < n / 2; ++k) {
            const float keep = up ? v[k + n / 2] : v[k], give = up ? v[k] : v[k + n / 2];
            v[k] = keep + __shfl_xor_sync(0xffffffffu, give, step);
        }
    }
    // (lane / (32 / K) is now the number of the value a lane carries)
    for (int o = 16 / K; o > 0; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    constexpr int EACH = 32 / K;             // lanes of a value
    if (t.warps > 1) {
        float* b = t.buf + t.turn * (K * 16);
        t.turn ^= 1;
        if (lane % EACH == 0) b[lane / EACH * 16 + t.warp] = v[0];
        t.barrier();
        const float* mine = b + lane / EACH * 16 + lane % EACH * (16 / EACH);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 16 / EACH; ++i) s += mine[i];
        for (int o = EACH / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        v[0] = s;
    } else __syncwarp();
#pragma unroll
    for (int k = K - 1; k >= 0; --k) v[k] = __shfl_sync(0xffffffffu, v[0], k * EACH);
}

// Rows of turn t: [lo, hi)
__device__ __forceinline__ void turn_rows(const NormParams& p, int64_t t, int64_t& lo, int64_t& hi)
{
    if (p.chunks_per_group > 1) {
        const int64_t g = t / p.chunks_per_group, k = t - g * p.chunks_per_group, end = (g + 1) * p.per_group;
        lo = g * p.per_group + k * p.chunk;
        hi = lo + p.chunk < end ? lo + p.chunk : end;
    } else {
        lo = t * p.chunk;
        hi = lo + p.chunk < p.rows ? lo + p.chunk : p.rows;
    }
}

// A team's first turn (p.turns: none): neighbouring turns to the teams of a CTA, and where there are not enough for all teams, as many to each CTA.  (Filling
// CTA after CTA: 4000 x 1024, float, a gate row for each row, forward 14.5 us instead of 13.)
__device__ __forceinline__ int64_t first_turn(const NormParams& p, int team_id)
{
    const int b = (int)blockIdx.x, n = p.each + (b < p.extra ? 1 : 0);
    return team_id < n ? (int64_t)(b * p.each + min(b, p.extra) + team_id) : p.turns;
}

// A team's ring over the rows of one turn.  A stage holds `stage_rows` rows of x, f, dy, dn, the gate and the stats (those that there are), one array after the
// other.  The thread that fills it refills a slot when the team has moved on from it: each row ends with a barrier behind its last read.
struct Ring {
    uint32_t base, full;
    int stages, slot;
    uint32_t phase;
    bool dead;
    __device__ __forceinline__ void fill(const NormParams& p, int s, int64_t row, int n, int esz)
    {
        const uint32_t bytes = (uint32_t)(n * p.d * esz), one = (uint32_t)(p.stage_rows * p.d * esz), bar = full + 8u * (uint32_t)s;
        const uint32_t gate = p.gate_ring ? (uint32_t)(n * p.d * 4) : 0u, st = p.dy || p.dn ? (uint32_t)n * 16u : 0u;
        uint32_t dst = base + (uint32_t)(s * p.stage_bytes);
        mbar_arrive_expect_tx(bar, bytes * (uint32_t)p.arrays + gate + st);
        const size_t at = (size_t)row * p.d * esz;
        bulk_load(dst, (const uint8_t*)p.x + at, bytes, bar); dst += one;
        if (p.f) { bulk_load(dst, (const uint8_t*)p.f + at, bytes, bar); dst += one; }
        if (p.dy) { bulk_load(dst, (const uint8_t*)p.dy + at, bytes, bar); dst += one; }
        if (p.dn) { bulk_load(dst, (const uint8_t*)p.dn + at, bytes, bar); dst += one; }
        if (gate) { bulk_load(dst, p.gate + (size_t)row * p.d, gate, bar); dst += (uint32_t)(p.stage_rows * p.d * 4); }
        if (st) bulk_load(dst, p.stats + row * 4, st, bar);
    }
    __device__ __forceinline__ uint32_t wait(const NormParams& p)
    {
        if (!dead && !mbar_wait_at(full + 8u * (uint32_t)slot, phase)) { dead = true; atomicMax(p.status, (uint32_t)DEV_TIMEOUT_TMA); }
        return base + (uint32_t)(slot * p.stage_bytes);
    }
    __device__ __forceinline__ void move() { if (++slot == stages) { slot = 0; phase ^= 1u; } }
};

#define SB_PAIRS(c, j) _Pragma("unroll") for (int c = 0; c < V; ++c) _Pragma("unroll") for (int j = 0; j < 4; ++j)

// Sum of squares, or (LAYER) mean and sum of squared distances, of a row held in registers (columns at or beyond d are zero)
template <typename T, int V, int BY, bool LAYER>
__device__ __forceinline__ void row_stats(const F2 (&v)[V][4], const NormParams& p, Place w, Team& team, float& mean, float& inv)
{
    mean = 0.f;
    F2 s = f2(0.f);
    if (LAYER) {
        SB_PAIRS(c, j) s = s + v[c][j];
        mean = team_sum(team, lo(s) + hi(s)) * p.rd;
        s = f2(0.f);
        SB_PAIRS(c, j) {
            F2 t = v[c][j] + f2(-mean);
            if (BY == BY_ELEMENT) t = f2(column<T, BY>(w, c, 2 * j) < p.d ? lo(t) : 0.f, column<T, BY>(w, c, 2 * j + 1) < p.d ? hi(t) : 0.f);
            else if (column<T, BY>(w, c, j / 2 * 4) >= p.d) t = f2(0.f);
            s = fma2(t, t, s);
        }
    } else {
        SB_PAIRS(c, j) s = fma2(v[c][j], v[c][j], s);
    }
    inv = rsqrtf(team_sum(team, lo(s) + hi(s)) * p.rd + p.eps);
}

// What both kernels begin with: barriers of the rings, the team's place.
#define SB_NORM_BEGIN(K, NT)                                                                                        \
    extern __shared__ __align__(128) uint8_t smem[];                                                            \
    __shared__ __align__(16) float buf[NT / 32 * 2 * K * 16];                                                     \
    __shared__ uint64_t full[NT / 32 * MAX_STAGES];                                                               \
    const int warp = threadIdx.x / 32, team_id = warp / p.team, d = p.d;                                        \
    for (int i = threadIdx.x; i < NT / 32 * 2 * K * 16; i += NT) buf[i] = 0.f;                               \
    if (BY == BY_RING && threadIdx.x < NT / 32 * MAX_STAGES) {                                                    \
        mbar_init(&full[threadIdx.x], 1);                                                                       \
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");                                      \
    }                                                                                                           \
    pdl_prologue();                                                                                             \
    __syncthreads();                                                                                            \
    Team team{buf + team_id * p.team * 2 * K * 16, team_id, p.team, warp - team_id * p.team};                   \
    const Place w{team.warp * 32 + (int)threadIdx.x % 32, p.team * 32};                                         \
    const bool mine = w.t == 0;                                                                                 \
    Ring ring{smem_u32(smem) + (uint32_t)(team_id * p.stages * p.stage_bytes), smem_u32(full + team_id * MAX_STAGES), p.stages, 0, 0u, false}

// Pieces of eight columns a thread takes: two where a row fills more than a warp (what every warp does for a row, the sums above all, costs as
// much as the columns of one piece), four only where two are not enough.
// (Element by element it is the other way round: 999 x 1001, float, backward 21 us with one piece and 24 with two.)
inline int pieces_of(int d, bool vec) { return d <= (vec ? 256 : THREADS * 8) ? 1 : d <= THREADS * 16 ? 2 : 4; }
inline int team_of(int d, bool vec)
{
    const int each = 8 * 32 * pieces_of(d, vec);
    return (d + each - 1) / each;
}

// How the rows fall to teams: about `want` turns, each of whole groups or a part of one.
struct Turns { int64_t chunk, turns; int per_group; };
inline Turns turns_of(int64_t rows, int64_t groups, int64_t want)
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
// Threads of a backward CTA: 256 with up to 255 registers each hold the vectors, their gradients and a row of up to 4096 columns (512 threads of 128
// registers spill: 16384 x 4096 took 670 us, and 400 with eight columns a thread and twice the warps).
inline int backward_threads(int d, bool vec) { return d <= (vec ? 4096 : 2048) ? 256 : 512; }
struct Grid { int64_t ctas; Turns turns; int team, teams; };
inline Grid grid_of(const sb_norm_config* c, bool backward, bool vec)
{
    Grid g{};
    g.team = team_of(c->d, vec);
    const int warps = (backward ? backward_threads(c->d, vec) : THREADS) / 32, pieces = pieces_of(c->d, vec);
    g.teams = warps / g.team;
    const bool two = pieces == 1;          // CTAs on an SM
    // (as many as have two stages of a row each in shared memory, where that leaves any)
    const size_t row = (size_t)c->d * (c->precision == SB_BF16 ? 2 : 4) * (backward ? 4 : 2);
    // (backward with 16 warps and two pieces, the vectors take a part of it (see vector_bytes), but a row fills more than half of the warps: one team as it is)
    const size_t room = (size_t)RING_LIMIT / (two ? 2 : 1);
    if (room / (2 * row) >= 1 && (size_t)g.teams > room / (2 * row)) g.teams = (int)(room / (2 * row));
    const int64_t most = two ? 296 : 148;
    g.turns = turns_of(c->rows, backward ? c->groups : 0, most * g.teams);
    // few turns: one a CTA rather than several teams of few CTAs (see spread)
    g.ctas = g.turns.turns < most ? g.turns.turns : most;
    return g;
}
inline void spread(NormParams& p, const Grid& g)
{
    p.team = g.team; p.teams = g.teams; p.turns = g.turns.turns; p.chunk = g.turns.chunk;
    const bool few = p.turns < g.ctas * g.teams;
    p.each = few ? (int)(p.turns / g.ctas) : g.teams;
    p.extra = few ? (int)(p.turns % g.ctas) : 0;
}
inline size_t part_floats(const sb_norm_config* c)
{
    size_t most = 0;
    for (bool vec : {false, true}) {          // (which of the two a call is depends on its pointers as well)
        const Grid g = grid_of(c, true, vec);
        const size_t n = (size_t)g.ctas * 3 * c->d + (g.turns.per_group > 1 ? (size_t)g.turns.turns * c->d : 0) + 64;
        if (n > most) most = n;
    }
    return most;
}
// Backward with two pieces a thread: the vectors in shared memory (see Held)
inline size_t vector_bytes(const NormParams& p) { return (p.dy || p.dn) && pieces_of(p.d, p.vec) == 2 && backward_threads(p.d, p.vec) == 512 ? (size_t)(2 + (p.gate ? p.teams : 1)) * 16 * 32 * p.team * 4 : 0; }
// The ring: three stages of as many rows as fit, at most eight; none where not even two stages of a row do.
inline void plan_ring(NormParams& p, const Grid& g, int esz, int limit)
{
    limit -= (int)vector_bytes(p);
    p.arrays = 1 + (p.f != nullptr) + (p.dy != nullptr) + (p.dn != nullptr);
    const size_t row = (size_t)p.d * (p.arrays * esz + (p.gate_ring ? 4 : 0)) + (p.arrays > 2 || !p.f ? 16 : 0), room = limit > 0 ? (size_t)limit / g.teams : 0;
    p.stages = room / row >= 3 ? 3 : room / row >= 2 ? 2 : 0;
    if (!p.stages) { p.gate_ring = 0; return; }
    size_t rows = room / p.stages / row;
    if (rows > 8) rows = 8;
    if ((int64_t)rows > p.chunk) rows = (size_t)p.chunk;
    p.stage_rows = (int)rows;
    p.stage_bytes = (int)(rows * row);
}
inline size_t ring_bytes(const NormParams& p) { return (size_t)p.teams * p.stages * p.stage_bytes; }

inline int by_of(const NormParams& p) { return !p.vec ? BY_ELEMENT : p.stages > 0 ? BY_RING : BY_PIECES; }

}  // namespace

cudaError_t launch_norm_backward_bf16(const NormParams& p, bool layer, int64_t ctas, cudaStream_t st);
cudaError_t launch_norm_backward_f32(const NormParams& p, bool layer, int64_t ctas, cudaStream_t st);

}  // namespace sb
