// Norm over rows, forward and backward (formulas in tsr.h).  Both passes are bound by HBM: forward reads x and writes y, backward reads
// x and dy and writes dx, each once; a row stays in registers between its sums and its results.
//
// Rows up to 32 KB are worked on by a group of lanes or a team of warps, the next ones in flight.  The mean is found in two steps: one sum gives m,
// the mean to FP32 accuracy, then the distances d = x - m, each rounded to its own size, are summed together with their squares, which
// corrects mean and variance:  mean = m + e,  e = sum d / n,  variance = sum d^2 / n - e^2  (e is below a unit of m's last place or below 2^-12 of the deviation,
// so that next to nothing is taken away; where rows are a few units of last place wide, a bit).  Neither a large mean nor single large entries, wherever they stand,
// cost the others digits.  The first sum is that of distances from the row's first entry, which makes m of a row of equal entries exact and its variance zero.
// Backward: lanes keep their columns
// from row to row, so that the sums for dweight and dbias stay in registers; a cluster of CTAs leaves one partial row of them, and
// column_finish_kernel adds those in order.
// Measured: forward 16384 x 2048 BF16 25.5 us (5.3 TB/s of 6.6 that a copy reaches), backward 8192 x 1024 FP32 23 us (4.3), backward without mean 6007 x
// 5461 BF16 59 us (3.4: the rows start at eight different places, teams of eight warps wait for each other, and first and last rows of a CTA are alone).
// Wider rows, and matrices that do not start at the same place in 16 bytes, are read several times (from L2, mostly), entry by entry; their column
// sums take a pass of their own.  Those are bound by instructions: 6007 x 5461 from a pitch of 5464 into one of 5461 takes 152 us forward, 220 us
// backward with mean and dbias, against 41 and 73 with both alike.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "tsr_layers.cuh"
#include "tsr_umma.cuh"

namespace tsr {

__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// Sum over the CTA; `slot` (a float per warp) must not be in use by an earlier sum that a thread may still read.
__device__ __forceinline__ float cta_sum(float x, float *slot)
{
    const int warps = (blockDim.x + 31) >> 5;
    x = warp_sum(x);
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = x;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return warp_sum(lane < warps ? slot[lane] : 0.f);
}
// Two sums at once.
__device__ __forceinline__ float2 cta_sums(float2 x, float2 *slot)
{
    const int warps = (blockDim.x + 31) >> 5;
    x = make_float2(warp_sum(x.x), warp_sum(x.y));
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = x;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const float2 s = lane < warps ? slot[lane] : make_float2(0.f, 0.f);
    return make_float2(warp_sum(s.x), warp_sum(s.y));
}
// Variance from the means of the squares and of the distances; rounding may leave it below zero, and NaN stays.
__device__ __forceinline__ float variance_of(float squares, float rest)
{
    const float v = fmaf(-rest, rest, squares);
    return v < 0.f ? 0.f : v;
}
__device__ __forceinline__ float finite_or_zero(float x) { return fabsf(x) < INFINITY ? x : 0.f; }
// The mean as the statistics hold it; that of a row with an infinity is the infinity.
__device__ __forceinline__ float whole_mean(float mean, float rest) { return fabsf(mean) == INFINITY ? mean : mean + rest; }

constexpr int NORM_STAGES = 8;      // most stages of a ring
constexpr int MOST_CLUSTER = 8;     // CTAs that add their column sums

struct NormArgs {
    const void *x, *dy, *weight, *bias;
    void *y;                        // y, or dx
    float *stats;
    const float *stats_in;
    float *partial;                 // [parts][cols] of dweight, then of dbias; NULL: one part, the sums go to dw and db
    void *dw, *db;
    int32_t g_bf16, accumulate;
    int64_t ldx, lddy, ldy, rows;
    int32_t cols, p_bf16, center, want_dw, want_db;
    int32_t team;                   // warps of a row
    int32_t period;                 // classes of rows that start at the same place in a unit; 0: the matrices differ in that
    float eps, inv_n;
};

// ---- rows in aligned vectors ------------------------------------------------------------------------------------------
//
// A UNIT is 16 aligned bytes, V entries.  Rows whose pitch is no multiple of 16 bytes start anywhere in a unit, but rows that are `period` apart
// start at the same place, and so do the rows of other matrices with the same offset and pitch modulo 16 bytes.  A CTA takes the rows
// of one such class: unit j of each of them holds columns j V - shift ..., for the whole life of the CTA, so that everything is read and written in
// aligned vectors, weight and column sums belong to fixed registers or addresses, and only the first and the last unit of a row need care.
// Rows come as bulk copies of whole units into a ring in shared memory, a few rows ahead of where they are used: what is in flight then costs no
// registers and no instructions.  (Every unit copied holds an entry of the row, so none lies outside of what may be read.)

template <typename T> struct Unit { static constexpr int V = 16 / (int)sizeof(T); };

struct RowClass { int shift, units; int64_t first, step; };    // rows first, first + step, ... of the matrix

// The class of this CTA; its rows are shared out among the CTAs of the class, `rows` side by side.
template <typename T>
__device__ __forceinline__ RowClass row_class(const void *x, int64_t ldx, int cols, int period, int cta, int ctas)
{
    constexpr int V = Unit<T>::V;
    RowClass c;
    const int cls = cta % period;
    c.shift = (int)((((uintptr_t)x / sizeof(T)) + (uint64_t)cls * (uint64_t)ldx) % V);
    c.units = (c.shift + cols + V - 1) / V;
    c.first = cls + (int64_t)period * (cta / period);
    c.step = (int64_t)period * (ctas / period);
    return c;
}

// Asks for a row: `units` units from the start of the one that holds its first entry.
template <typename T>
__device__ __forceinline__ void ask_row(uint32_t dst, const T *row, const RowClass &rc, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"((uint64_t)__cvta_generic_to_global(row - rc.shift)), "r"((uint32_t)rc.units * 16u), "r"(bar) : "memory");
}
// Waits for a stage of the ring; once a wait has run out nothing is waited for any more (the outputs are then undefined).
__device__ __forceinline__ void await_row(uint32_t bar, uint32_t parity, bool &gave_up)
{
    if (!gave_up && !mbar_wait(bar, parity, UM_WAIT_CLOCKS)) gave_up = true;
}
__device__ int g_norm_status;
__device__ __forceinline__ void note_gave_up(bool gave_up)
{
    if (!gave_up) return;
    atomicMax(&g_norm_status, (int)TSR_ERR_TIMEOUT);
    __nanosleep(2000000);      // let copies in flight land before the CTA goes away
}

// Where the entries of a row lie in its first and its last unit: bits that are set for them, kept in shared memory.  Only the units u = 0 and u = last of a
// lane can be those, so that all others of a row are taken and stored without a look.
struct Edges { uint4 first, last; };
template <typename T>
__device__ __forceinline__ uint4 unit_mask(int col, int cols)
{
    constexpr int V = Unit<T>::V;
    uint32_t m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (V == 4) m[i] = col + i >= 0 && col + i < cols ? 0xffffffffu : 0u;
        else m[i] = (col + 2 * i >= 0 && col + 2 * i < cols ? 0xffffu : 0u) | (col + 2 * i + 1 >= 0 && col + 2 * i + 1 < cols ? 0xffff0000u : 0u);
    }
    return make_uint4(m[0], m[1], m[2], m[3]);
}
template <typename T>
__device__ __forceinline__ void find_edges(Edges *e, const RowClass &rc, int cols)      // by one thread
{
    e->first = unit_mask<T>(-rc.shift, cols);
    e->last = unit_mask<T>((rc.units - 1) * Unit<T>::V - rc.shift, cols);
}
// Whether unit u of the lanes may hold an edge, and the mask of this lane's unit j there.
__device__ __forceinline__ bool at_edge(int u, int last_u) { return u == 0 || u == last_u; }
__device__ __forceinline__ uint4 edge_mask(const Edges &e, int j, int units)
{
    uint4 m = make_uint4(0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu);
    if (j == 0) m = e.first;
    if (j == units - 1) {
        const uint4 l = e.last;
        m = make_uint4(m.x & l.x, m.y & l.y, m.z & l.z, m.w & l.w);
    }
    return m;
}
// The places that hold no entry become `fill` (a value, or two of them in a word).
__device__ __forceinline__ uint4 filled(const uint4 &r, const uint4 &m, uint32_t fill)
{
    return make_uint4((r.x & m.x) | (fill & ~m.x), (r.y & m.y) | (fill & ~m.y), (r.z & m.z) | (fill & ~m.z), (r.w & m.w) | (fill & ~m.w));
}
__device__ __forceinline__ uint32_t fill_word(float x) { return __float_as_uint(x); }
__device__ __forceinline__ uint32_t fill_word(bf16 x) { return (uint32_t)__bfloat16_as_ushort(x) * 0x10001u; }
// A unit as pairs of FP32 values, and back.
__device__ __forceinline__ float2 bf16_pair(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ void unit_pairs(const uint4 &r, float2 (&v)[4]) { v[0] = bf16_pair(r.x); v[1] = bf16_pair(r.y); v[2] = bf16_pair(r.z); v[3] = bf16_pair(r.w); }
__device__ __forceinline__ void unit_pairs(const uint4 &r, float2 (&v)[2])
{
    v[0] = make_float2(__uint_as_float(r.x), __uint_as_float(r.y));
    v[1] = make_float2(__uint_as_float(r.z), __uint_as_float(r.w));
}
__device__ __forceinline__ uint4 unit_of(const float2 (&v)[4])
{
    return make_uint4(pack_bf16(v[0].x, v[0].y), pack_bf16(v[1].x, v[1].y), pack_bf16(v[2].x, v[2].y), pack_bf16(v[3].x, v[3].y));
}
__device__ __forceinline__ uint4 unit_of(const float2 (&v)[2])
{
    return make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x), __float_as_uint(v[1].y));
}
// To the unit that begins with column col; with `edge` the places that hold no entry are left alone.
template <typename T>
__device__ __forceinline__ void store_unit(T *row, int col, int cols, bool edge, const float2 (&v)[Unit<T>::V / 2])
{
    constexpr int V = Unit<T>::V;
    const uint4 r = unit_of(v);
    if (!edge || (col >= 0 && col + V <= cols)) *(uint4 *)(row + col) = r;
    else {
        T t[V];
        memcpy(t, &r, 16);
#pragma unroll
        for (int i = 0; i < V; ++i) if (col + i >= 0 && col + i < cols) row[col + i] = t[i];
    }
}
__device__ __forceinline__ float param(const void *p, int c, bool is_bf16, float none) { return p ? load_as(p, c, is_bf16) : none; }

// The entries of a unit less `from`.
template <int P>
__device__ __forceinline__ void less(float2 (&v)[P], float from)
{
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = add2(v[i], pair(-from));
}

// weight and bias of a row's units in shared memory, units * V values each: the first four values of every unit, then (BF16) the last four, so that
// the lanes of a warp read 16 bytes side by side.
__device__ __forceinline__ int shared_at(int unit, int half, int units) { return (half * units + unit) * 4; }
template <typename T>
__device__ __forceinline__ void share_params(const NormArgs &a, const RowClass &rc, float *w, float *b)
{
    constexpr int V = Unit<T>::V;
    constexpr int AT_ONCE = 8;      // loads in flight: one after the other they took 9 us of a row of 5461 columns
    for (int i0 = threadIdx.x; i0 < rc.units * V; i0 += AT_ONCE * blockDim.x) {
        float wv[AT_ONCE], bv[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int c = i0 + k * blockDim.x - rc.shift;
            const bool in = c >= 0 && c < a.cols;
            wv[k] = in ? param(a.weight, c, a.p_bf16, 1.f) : 0.f;
            bv[k] = in && b ? param(a.bias, c, a.p_bf16, 0.f) : 0.f;
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int i = i0 + k * blockDim.x, at = shared_at(i / V, i % V / 4, rc.units) + i % 4;
            if (i >= rc.units * V) break;
            w[at] = wv[k];
            if (b) b[at] = bv[k];
        }
    }
}
// Sums of distances and squares without those of `empty` places, each at distance `from`.  That is the first entry's own distance, so that at most 2 V - 2
// squares are taken away from a sum that keeps one more of them: four bits at the worst (a row of two BF16 entries), none of a long row without outliers.
template <bool EDGE>
__device__ __forceinline__ float2 less_empty(float2 s, float from, float empty)
{
    if (!EDGE) return s;
    const float e = empty * from;
    return make_float2(s.x - e, fmaf(-e, from, s.y));
}
// v <- (v rstd + shift) w + b over unit j
template <int P>
__device__ __forceinline__ void normed(float2 (&v)[P], float rstd, float shift, const float *w, const float *b, int j, int units)
{
#pragma unroll
    for (int i = 0; i < P; i += 2) {
        const float4 ww = *(const float4 *)(w + shared_at(j, i / 2, units)), bb = *(const float4 *)(b + shared_at(j, i / 2, units));
        v[i] = fma2(fma2(v[i], pair(rstd), pair(shift)), make_float2(ww.x, ww.y), make_float2(bb.x, bb.y));
        v[i + 1] = fma2(fma2(v[i + 1], pair(rstd), pair(shift)), make_float2(ww.z, ww.w), make_float2(bb.z, bb.w));
    }
}

// The sum over a row's L lanes.
template <int L>
__device__ __forceinline__ float lanes_sum(float x)
{
#pragma unroll
    for (int o = L / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// Two sums at once: the lanes share them out with the first exchange.
template <int L>
__device__ __forceinline__ float2 lanes_sum(float2 x, int lane)
{
    const bool hi = lane & (L / 2);
    float k = (hi ? x.y : x.x) + __shfl_xor_sync(0xffffffffu, hi ? x.x : x.y, L / 2);
#pragma unroll
    for (int o = L / 4; o; o >>= 1) k += __shfl_xor_sync(0xffffffffu, k, o);
    const float other = __shfl_xor_sync(0xffffffffu, k, L / 2);
    return hi ? make_float2(other, k) : make_float2(k, other);
}

// Who works on a row: L lanes of a warp (32 / L rows side by side in it), or (TEAMS) several whole warps, U units per lane.  The groups do not wait for
// one another; each has a ring of `stages` rows.  Of all groups of a class of rows, the g-th takes every n-th row.
constexpr int ROW_WARPS = 8;       // warps of a CTA, and most groups of them
template <int L, bool TEAMS>
struct Rows {
    int lane, lanes, group, groups;    // within the row; of the CTA
    int warps;                     // ... of a team
    int left, turns;               // rows of the group, and the most of a group of the warp
    int64_t row, step;
    RowClass rc;
};
template <typename T, int L, bool TEAMS>
__device__ __forceinline__ Rows<L, TEAMS> rows_of(const NormArgs &a, int cta, int ctas)
{
    Rows<L, TEAMS> r;
    r.rc = row_class<T>(a.x, a.ldx, a.cols, a.period, cta, ctas);
    r.warps = TEAMS ? a.team : 1;
    r.lanes = TEAMS ? 32 * r.warps : L;
    r.group = (int)threadIdx.x / r.lanes;
    r.groups = (int)blockDim.x / r.lanes;
    r.lane = (int)threadIdx.x - r.group * r.lanes;
    r.step = r.rc.step * r.groups;           // (`step` of the class is that of a CTA with one row)
    r.row = r.rc.first + r.rc.step * r.group;
    const int64_t left = r.row < a.rows ? (a.rows - r.row + r.step - 1) / r.step : 0;
    r.left = (int)left;                      // (at most 2^40 rows among the groups of a full grid)
    r.turns = __shfl_sync(0xffffffffu, r.left, 0);      // (the first group of a warp has the most)
    return r;
}
// Waits for the other warps of the team (barrier 0 is the CTA's).
__device__ __forceinline__ void team_sync(int team, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(threads) : "memory"); }

template <typename T, int L, int U, bool EDGE, bool TEAMS>
__global__ void __launch_bounds__(256, U > 4 ? 2 : U > 2 ? 3 : 4)
norm_forward_kernel(const NormArgs a, int stages)
{
    constexpr int V = Unit<T>::V, P = V / 2, G = 32 / L;      // G: groups of a warp (or of a team)
    extern __shared__ float4 shared[];       // w, b, rings
    __shared__ uint64_t bars[ROW_WARPS * NORM_STAGES];
    __shared__ Edges edges;
    __shared__ float2 slots[TEAMS ? 2 : 1][ROW_WARPS];     // sums of a team's warps: the first and the second of a row, or those of one row and the next
    pdl_trigger();
    pdl_wait();
    const int warp = threadIdx.x >> 5;
    const Rows<L, TEAMS> rows = rows_of<T, L, TEAMS>(a, blockIdx.x, gridDim.x);
    const RowClass &rc = rows.rc;
    const int lane = rows.lane, left = rows.left, lanes = rows.lanes, ring_at = TEAMS ? rows.group : warp;
    float *w = (float *)shared, *b = w + rc.units * V;
    const uint4 *ring = (const uint4 *)(b + rc.units * V) + (ring_at * stages * G + rows.group % G) * rc.units;
    uint64_t *bar = bars + ring_at * NORM_STAGES;
    const float empty = (float)(rc.units * V - a.cols);      // places of a row's units that hold no entry
    const T *ask = (const T *)a.x + rows.row * a.ldx;
    const int64_t next_ask = rows.step * a.ldx, next_y = rows.step * a.ldy;
    int asked = 0;
    auto request = [&](int stage) {      // the next row, by the first lane of a group
        const bool any = asked++ < left;
        mbar_expect_tx(smem_u32(bar + stage), any ? (uint32_t)rc.units * 16u : 0u);
        if (!any) return;
        ask_row<T>(smem_u32(ring + stage * G * rc.units), ask, rc, smem_u32(bar + stage));
        ask += next_ask;
    };
    // over the whole row, from every lane's sum; or two at once.  (A team's lanes read its warps' sums side by side: one after the other they took 8000 x 8192
    // BF16 from 68 to 72 us.)
    auto row_sum = [&](float x, float2 *slot) -> float {
        x = lanes_sum<L>(x);
        if constexpr (TEAMS) {      // (slots are written again after another barrier at the earliest)
            if ((threadIdx.x & 31) == 0) slot[warp].x = x;
            team_sync(rows.group, lanes);
            x = slot[rows.group * rows.warps + (lane & (rows.warps - 1))].x;
            for (int o = rows.warps / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        }
        return x;
    };
    auto row_sums = [&](float2 x, float2 *slot) -> float2 {
        x = lanes_sum<L>(x, lane);
        if constexpr (TEAMS) {
            if ((threadIdx.x & 31) == 0) slot[warp] = x;
            team_sync(rows.group, lanes);
            x = slot[rows.group * rows.warps + (lane & (rows.warps - 1))];
            for (int o = rows.warps / 2; o; o >>= 1) {
                x.x += __shfl_xor_sync(0xffffffffu, x.x, o);
                x.y += __shfl_xor_sync(0xffffffffu, x.y, o);
            }
        }
        return x;
    };
    if (TEAMS ? lane == 0 : (threadIdx.x & 31) == 0) {
        for (int i = 0; i < stages; ++i) mbar_init(smem_u32(bar + i), G);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (EDGE && threadIdx.x == 0) find_edges<T>(&edges, rc, a.cols);
    const int last_u = (rc.units - 1) / lanes;
    __syncwarp();
    if (lane == 0)
        for (int i = 0; i < stages && i < rows.turns; ++i) request(i);
    share_params<T>(a, rc, w, b);
    __syncthreads();
    bool gave_up = false;
    int stage = 0;
    uint32_t phase = 0;
    T *y = (T *)a.y + rows.row * a.ldy;
    float *stats = a.stats ? a.stats + 2 * rows.row : nullptr;
    for (int turn = 0; turn < rows.turns; ++turn) {
        await_row(smem_u32(bar + stage), phase, gave_up);
        const uint4 *row = ring + stage * G * rc.units;
        const bool mine = G == 1 || turn < left;      // (what a group without a row computes goes nowhere)
        const T pivot = a.center ? *((const T *)row + rc.shift) : T(0.f);      // the first entry; also stands in the places that hold none
        const float x0 = finite_or_zero(load_f(&pivot));
        float2 v[U][P], sum = pair(0.f), q = pair(0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * lanes + lane;
            uint4 r = make_uint4(0, 0, 0, 0);
            if (j < rc.units) {
                r = row[j];
                if (EDGE && at_edge(u, last_u)) r = filled(r, edge_mask(edges, j, rc.units), fill_word(pivot));
            }
            unit_pairs(r, v[u]);
        }
        if constexpr (!TEAMS) {      // (a team: after its barrier)
            __syncwarp();
            if (lane == 0 && turn + stages < rows.turns) request(stage);
        }
        float mean = 0.f, rest = 0.f, shift = 0.f, rstd;
        if (a.center) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u * lanes + lane >= rc.units) continue;
#pragma unroll
                for (int i = 0; i < P; ++i) sum = add2(sum, add2(v[u][i], pair(-x0)));
            }
            mean = fmaf(row_sum(sum.x + sum.y, slots[0]), a.inv_n, x0);
            sum = pair(0.f);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u * lanes + lane >= rc.units) continue;
                less(v[u], mean);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    sum = add2(sum, v[u][i]);
                    q = fma2(v[u][i], v[u][i], q);
                }
            }
            const float2 s = less_empty<EDGE>(row_sums(make_float2(sum.x + sum.y, q.x + q.y), slots[TEAMS ? 1 : 0]), x0 - mean, empty);
            rest = s.x * a.inv_n;
            rstd = rsqrtf(variance_of(s.y * a.inv_n, rest) + a.eps);
            shift = -rest * rstd;
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u * lanes + lane >= rc.units) continue;
#pragma unroll
                for (int i = 0; i < P; ++i) q = fma2(v[u][i], v[u][i], q);
            }
            rstd = rsqrtf(fmaf(row_sum(q.x + q.y, slots[TEAMS ? turn & 1 : 0]), a.inv_n, a.eps));
        }
        if (TEAMS && lane == 0 && turn + stages < rows.turns) request(stage);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
        if (stats && lane == 0 && mine) *(float2 *)stats = make_float2(whole_mean(mean, rest), rstd);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * lanes + lane;
            if (j >= rc.units || !mine) continue;
            normed(v[u], rstd, shift, w, b, j, rc.units);
            store_unit<T>(y, j * V - rc.shift, a.cols, EDGE && at_edge(u, last_u), v[u]);
        }
        y += next_y;
        if (stats) stats += 2 * rows.step;
    }
    note_gave_up(gave_up);
}

// Any width and alignment: three passes over the row.
template <typename T>
__global__ void __launch_bounds__(1024)
norm_forward_wide_kernel(const NormArgs a)
{
    __shared__ float slots[32];
    __shared__ float2 pairs[32];
    pdl_trigger();
    pdl_wait();
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = (const T *)a.x + r * a.ldx;
        float mean = 0.f, rest = 0.f, sum = 0.f, q = 0.f;
        if (a.center) {
            const float x0 = finite_or_zero(load_f(x));
            for (int c = threadIdx.x; c < a.cols; c += blockDim.x) sum += load_f(x + c) - x0;
            mean = fmaf(cta_sum(sum, slots), a.inv_n, x0);
        }
        sum = 0.f;
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
            const float d = load_f(x + c) - mean;
            sum += d;
            q = fmaf(d, d, q);
        }
        const float2 s = cta_sums(make_float2(sum, q), pairs);
        if (a.center) rest = s.x * a.inv_n;
        const float rstd = rsqrtf(variance_of(s.y * a.inv_n, rest) + a.eps), shift = a.center ? -rest * rstd : 0.f;
        if (a.stats && threadIdx.x == 0) { a.stats[2 * r] = whole_mean(mean, rest); a.stats[2 * r + 1] = rstd; }
        T *y = (T *)a.y + r * a.ldy;
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x)
            store_f(y + c, fmaf(fmaf(load_f(x + c) - mean, rstd, shift), param(a.weight, c, a.p_bf16, 1.f), param(a.bias, c, a.p_bf16, 0.f)));
        __syncthreads();
    }
}

// Column sums at the end of a backward kernel.  A unit's, to shared memory:
__device__ __forceinline__ void keep_sums(float *to, const float2 (&v)[4])
{
    *(float4 *)to = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
    *(float4 *)(to + 4) = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
}
__device__ __forceinline__ void keep_sums(float *to, const float2 (&v)[2]) { *(float4 *)to = make_float4(v[0].x, v[0].y, v[1].x, v[1].y); }
// The sums of a CTA lie by unit, dweight's, then dbias's.  Each CTA of the cluster (along z) adds a share of the columns over all of them (whose units
// may start elsewhere), so that fewer partial rows are left: 740 of 2048 columns took longer to write and read than the sums.
template <typename T, bool DB>
__device__ __forceinline__ void add_up(const NormArgs &a, const float *sums)
{
    constexpr int V = Unit<T>::V;
    const int cluster = gridDim.z, rank = blockIdx.z, ctas = gridDim.x * cluster, first = blockIdx.x * cluster;
    if (cluster > 1) cluster_sync();
    else __syncthreads();
    int from[MOST_CLUSTER], half[MOST_CLUSTER];
#pragma unroll
    for (int k = 0; k < MOST_CLUSTER; ++k) {
        const RowClass other = row_class<T>(a.x, a.ldx, a.cols, a.period, first + k, ctas);
        from[k] = other.shift;
        half[k] = other.units * V;
    }
#pragma unroll 2
    for (int c = rank * blockDim.x + threadIdx.x; c < a.cols; c += cluster * blockDim.x) {
        float w = 0.f, b = 0.f;
#pragma unroll
        for (int k = 0; k < MOST_CLUSTER; ++k) {
            if (k >= cluster) break;
            if (a.want_dw) w += shared_of(sums + from[k] + c, k);
            if (DB) b += shared_of(sums + half[k] + from[k] + c, k);
        }
        if (a.partial) {
            if (a.want_dw) a.partial[(int64_t)blockIdx.x * a.cols + c] = w;
            if (DB) a.partial[((int64_t)(a.want_dw ? gridDim.x : 0) + blockIdx.x) * a.cols + c] = b;
        } else {
            if (a.want_dw) store_as(a.dw, c, a.g_bf16, a.accumulate ? w + load_as(a.dw, c, a.g_bf16) : w);
            if (DB) store_as(a.db, c, a.g_bf16, a.accumulate ? b + load_as(a.db, c, a.g_bf16) : b);
        }
    }
    if (cluster > 1) cluster_sync();      // no CTA leaves while its sums are read
}

// Units of x and dy of one row in the ring; groups of four lanes, two of which are served at a time, get slots half a cycle of the banks apart.
template <int L>
__host__ __device__ __forceinline__ int slot_units(int units) { return 2 * units + (L == 4 ? (4 - 2 * units % 8 + 8) % 8 : 0); }

// Groups and rings as in the forward pass; x and dy come through the ring.  A lane keeps its columns from row to row, so that the column sums stay in
// registers (128 of them at U = 8 and BF16: eight warps per SM, whose eight units per lane hide what little there is to wait for; two units per thread
// in five CTAs of four warps per row took 69 us for 16384 x 2048, where half of the instructions were those of barriers and sums).  Weight is in
// registers up to two units, else in shared memory.  DB: the sums of dy are wanted too.
template <typename T, int L, int U, bool DB, bool EDGE, bool TEAMS, int CTAS, int WARPS = ROW_WARPS>
__global__ void __launch_bounds__(32 * WARPS, CTAS)
norm_backward_kernel(const NormArgs a, int stages)
{
    constexpr int V = Unit<T>::V, P = V / 2, G = 32 / L;
    constexpr bool KEEP = U <= 2;
    extern __shared__ float4 shared[];       // weight (unless kept), rings; at the end the column sums
    __shared__ uint64_t bars[ROW_WARPS * NORM_STAGES];
    __shared__ Edges edges;
    __shared__ float2 slots[2][TEAMS ? WARPS : 1];      // sums of a team's warps
    pdl_trigger();
    pdl_wait();
    const int warp = threadIdx.x >> 5;
    const int cta = blockIdx.x * gridDim.z + blockIdx.z;
    const Rows<L, TEAMS> rows = rows_of<T, L, TEAMS>(a, cta, gridDim.x * gridDim.z);
    const RowClass &rc = rows.rc;
    const int lane = rows.lane, left = rows.left, lanes = rows.lanes, ring_at = TEAMS ? rows.group : warp;
    float *weight = (float *)shared;
    const int slot = slot_units<L>(rc.units);
    const uint4 *ring = (const uint4 *)(KEEP ? weight : weight + rc.units * V) + (ring_at * stages * G + rows.group % G) * slot;
    uint64_t *bar = bars + ring_at * NORM_STAGES;
    const T *ask_x = (const T *)a.x + rows.row * a.ldx, *ask_dy = (const T *)a.dy + rows.row * a.lddy;
    const int64_t next_x = rows.step * a.ldx, next_dy = rows.step * a.lddy, next_y = rows.step * a.ldy;
    int asked = 0;
    auto request = [&](int stage) {      // the next row, by the first lane of a group
        const bool any = asked++ < left;
        const uint32_t to = smem_u32(bar + stage), bytes = (uint32_t)rc.units * 16u, at = smem_u32(ring + stage * G * slot);
        mbar_expect_tx(to, any ? 2 * bytes : 0u);
        if (!any) return;
        ask_row<T>(at, ask_x, rc, to);
        ask_row<T>(at + bytes, ask_dy, rc, to);
        ask_x += next_x;
        ask_dy += next_dy;
    };
    if (TEAMS ? lane == 0 : (threadIdx.x & 31) == 0) {
        for (int i = 0; i < stages; ++i) mbar_init(smem_u32(bar + i), G);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (EDGE && threadIdx.x == 0) find_edges<T>(&edges, rc, a.cols);
    const int last_u = (rc.units - 1) / lanes;
    __syncwarp();
    if (lane == 0)
        for (int i = 0; i < stages && i < rows.turns; ++i) request(i);
    float2 kept[KEEP ? U : 1][P], dw[U][P], db[DB ? U : 1][P];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < P; ++i) {
            dw[u][i] = pair(0.f);
            if (DB) db[u][i] = pair(0.f);
            if (KEEP) {
                const int c = (u * lanes + lane) * V - rc.shift + 2 * i;
                kept[u][i] = make_float2(c >= 0 && c < a.cols ? param(a.weight, c, a.p_bf16, 1.f) : 0.f, c + 1 >= 0 && c + 1 < a.cols ? param(a.weight, c + 1, a.p_bf16, 1.f) : 0.f);
            }
        }
    if (!KEEP) share_params<T>(a, rc, weight, nullptr);
    if (!KEEP || EDGE) __syncthreads();      // (teams keep none: their other warps see the barriers initialised)
    auto weights = [&](int u, float2 (&w)[P]) {
#pragma unroll
        for (int i = 0; i < P; i += 2) {
            if constexpr (KEEP) {
                w[i] = kept[u][i];
                w[i + 1] = kept[u][i + 1];
            } else {
                const float4 t = *(const float4 *)(weight + shared_at(u * lanes + lane, i / 2, rc.units));
                w[i] = make_float2(t.x, t.y);
                w[i + 1] = make_float2(t.z, t.w);
            }
        }
    };
    bool gave_up = false;
    int stage = 0;
    uint32_t phase = 0;
    T *y = (T *)a.y + rows.row * a.ldy;
    const float2 *stats = (const float2 *)a.stats_in + rows.row;
    float2 next = left > 0 ? *stats : pair(0.f);
    for (int turn = 0; turn < rows.turns; ++turn) {
        const float2 st = next;
        stats += rows.step;
        next = turn + 1 < left ? *stats : pair(0.f);
        await_row(smem_u32(bar + stage), phase, gave_up);
        const uint4 *row = ring + stage * G * slot;
        const bool mine = G == 1 || turn < left;
        uint4 x[U], g[U];
        float2 s1 = pair(0.f), s2 = pair(0.f);
        const float2 less_mu = pair(-st.x), r = pair(st.y);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * lanes + lane;
            if (j >= rc.units || !mine) continue;
            x[u] = row[j];
            g[u] = row[rc.units + j];
            if (EDGE && at_edge(u, last_u)) {
                const uint4 m = edge_mask(edges, j, rc.units);
                x[u] = filled(x[u], m, 0u);
                g[u] = filled(g[u], m, 0u);
            }
            float2 w[P], xv[P], gv[P];
            weights(u, w);
            unit_pairs(x[u], xv);
            unit_pairs(g[u], gv);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float2 h = mul2(add2(xv[i], less_mu), r);
                dw[u][i] = fma2(gv[i], h, dw[u][i]);
                if (DB) db[u][i] = add2(db[u][i], gv[i]);
                const float2 gw = mul2(gv[i], w[i]);
                s1 = add2(s1, gw);
                s2 = fma2(gw, h, s2);
            }
        }
        float2 s = lanes_sum<L>(make_float2(s1.x + s1.y, s2.x + s2.y), lane);
        if constexpr (TEAMS) {      // (one barrier per turn: the slots of the turn before last are written again only after the last one's)
            if ((threadIdx.x & 31) == 0) slots[turn & 1][warp] = s;
            team_sync(rows.group, lanes);
            s = pair(0.f);
            for (int i = 0; i < rows.warps; ++i) s = add2(s, slots[turn & 1][rows.group * rows.warps + i]);
        }
        if (lane == 0 && turn + stages < rows.turns) request(stage);      // (after shuffles or barrier: every lane has read its units)
        if (++stage == stages) { stage = 0; phase ^= 1u; }
        if (a.y && mine) {
            // dx = r g w - r mean(g w) - (x - mu) r^2 mean(g w h)
            const float2 c1 = pair(a.center ? -s.x * a.inv_n * st.y : 0.f), c2 = pair(-s.y * a.inv_n * st.y * st.y);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = u * lanes + lane;
                if (j >= rc.units) continue;
                float2 w[P], xv[P], gv[P];
                weights(u, w);
                unit_pairs(x[u], xv);
                unit_pairs(g[u], gv);
#pragma unroll
                for (int i = 0; i < P; ++i) gv[i] = fma2(mul2(gv[i], w[i]), r, fma2(add2(xv[i], less_mu), c2, c1));
                store_unit<T>(y, j * V - rc.shift, a.cols, EDGE && at_edge(u, last_u), gv);
            }
        }
        y += next_y;
    }
    note_gave_up(gave_up);
    if (!a.want_dw && !DB) return;
    // The column sums: over the groups of a warp, then (in the place of weight and rings) over warps or teams.
    const int width = rc.units * V, set = DB ? 2 * width : width;
    float *sums = (float *)shared;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int j = u * lanes + lane;
#pragma unroll
        for (int o = L; o < 32; o <<= 1)
#pragma unroll
            for (int i = 0; i < P; ++i) {
                dw[u][i] = add2(dw[u][i], make_float2(__shfl_xor_sync(0xffffffffu, dw[u][i].x, o), __shfl_xor_sync(0xffffffffu, dw[u][i].y, o)));
                if (DB) db[DB ? u : 0][i] = add2(db[DB ? u : 0][i], make_float2(__shfl_xor_sync(0xffffffffu, db[DB ? u : 0][i].x, o), __shfl_xor_sync(0xffffffffu, db[DB ? u : 0][i].y, o)));
            }
        if (j >= rc.units || (!TEAMS && rows.group % G)) continue;
        keep_sums(sums + ring_at * set + j * V, dw[u]);
        if (DB) keep_sums(sums + ring_at * set + width + j * V, db[DB ? u : 0]);
    }
    __syncthreads();
    const int sets = rows.groups / G;
#pragma unroll 4
    for (int i = threadIdx.x; i < set; i += blockDim.x) {
        float t = sums[i];
#pragma unroll
        for (int k = 1; k < ROW_WARPS; ++k) if (k < sets) t += sums[k * set + i];
        sums[i] = t;
    }
    add_up<T, DB>(a, sums);
}

// Any width and alignment: dx alone, two passes over the row (after the column sums, as it may replace dy), ...
template <typename T>
__global__ void __launch_bounds__(1024)
norm_backward_wide_kernel(const NormArgs a)
{
    __shared__ float slots[2][32];
    pdl_trigger();
    pdl_wait();
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = (const T *)a.x + r * a.ldx, *dy = (const T *)a.dy + r * a.lddy;
        const float mu = a.stats_in[2 * r], rs = a.stats_in[2 * r + 1];
        float c1 = 0.f, c2 = 0.f;
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
            const float g = load_f(dy + c) * param(a.weight, c, a.p_bf16, 1.f);
            c1 += g;
            c2 = fmaf(g, (load_f(x + c) - mu) * rs, c2);
        }
        c1 = cta_sum(c1, slots[0]);
        c2 = cta_sum(c2, slots[1]) * a.inv_n;
        c1 = a.center ? c1 * a.inv_n : 0.f;
        T *dx = (T *)a.y + r * a.ldy;
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
            const float g = load_f(dy + c) * param(a.weight, c, a.p_bf16, 1.f);
            store_f(dx + c, rs * (g - fmaf((load_f(x + c) - mu) * rs, c2, c1)));
        }
        __syncthreads();
    }
}
// ... and the column sums: 256 columns per CTA, a range of rows.
template <typename T>
__global__ void __launch_bounds__(256)
norm_columns_kernel(const NormArgs a, int64_t rows_per)
{
    pdl_trigger();
    pdl_wait();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    const int64_t r0 = blockIdx.y * rows_per, r1 = min(a.rows, r0 + rows_per);
    float dw = 0.f, db = 0.f;
#pragma unroll 4
    for (int64_t r = r0; r < r1; ++r) {
        const float g = load_f((const T *)a.dy + r * a.lddy + c);
        dw = fmaf(g, (load_f((const T *)a.x + r * a.ldx + c) - a.stats_in[2 * r]) * a.stats_in[2 * r + 1], dw);
        db += g;
    }
    if (a.want_dw) a.partial[(int64_t)blockIdx.y * a.cols + c] = dw;
    if (a.want_db) a.partial[((int64_t)(a.want_dw ? gridDim.y : 0) + blockIdx.y) * a.cols + c] = db;
}

cudaError_t norm_status_read(int32_t *status, cudaStream_t stream)
{
    int zero = 0, v = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(&v, g_norm_status, sizeof(int), 0, cudaMemcpyDeviceToHost, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    if (e == cudaSuccess && v) e = cudaMemcpyToSymbolAsync(g_norm_status, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    *status = v;
    return e;
}

namespace {

constexpr int64_t ROW_UNITS = 2048;         // widest row that the row kernels hold

// Classes of rows (see above) that a set of matrices has in common, and the most units a row of theirs covers; 0: none in common.
int common_period(const tsr_norm_desc &d, const tsr_matrix *const *m, int n, int *units)
{
    const int es = type_bytes(d.dtype), V = 16 / es;
    const int64_t at = (int64_t)(((uintptr_t)m[0]->data / es) % V), ld = d.rows > 1 ? m[0]->ld % V : 0;
    for (int i = 1; i < n; ++i) {
        if (!m[i]->data) continue;
        if ((int64_t)(((uintptr_t)m[i]->data / es) % V) != at || (d.rows > 1 && m[i]->ld % V != ld)) return 0;
    }
    int period = 1;
    while (ld * period % V) period *= 2;
    *units = 0;
    for (int c = 0; c < period; ++c) *units = std::max(*units, (int)(((at + c * ld) % V + d.cols + V - 1) / V));
    return period;
}

int64_t shared_out(int64_t rows, int period, int64_t rows_each, int64_t ctas)      // CTAs, a multiple of the period
{
    const int64_t per_class = (rows + period - 1) / period;
    return period * std::max<int64_t>(1, std::min<int64_t>((per_class + rows_each - 1) / rows_each, ctas / period));
}
int any_threads(int64_t cols) { return (int)std::min<int64_t>(1024, std::max<int64_t>(32, round_up(cols, 32))); }

// Rows of whole units have no edges to look at.
bool has_edges(const NormArgs &a, int V) { return a.period != 1 || a.cols % V || (uintptr_t)a.x % 16; }

// Shared memory of an SM that its CTAs may share out, and a ring's stages in what one of them gets.
constexpr int SM_SHARED = 216 * 1024;
int ring_stages(int per_sm, size_t fixed, size_t stage)
{
    const int64_t n = (SM_SHARED / per_sm - (int64_t)fixed) / (int64_t)stage;
    return (int)std::max<int64_t>(1, std::min<int64_t>(NORM_STAGES, n));
}
template <typename Kern>
cudaError_t launch_with(Kern kernel, dim3 grid, int threads, size_t smem, cudaStream_t s, const NormArgs &a, int stages, int cluster = 1)
{
    if (smem > 40 * 1024) {      // (48 KB less what is static; the limit belongs to the kernel, so all calls set the same: other threads may be between here and their launch)
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SM_SHARED);
        if (e != cudaSuccess) return e;
    }
    return launch_dependent(kernel, grid, dim3(threads), smem, s, cluster, a, stages);
}

// Rows of more units than a warp takes: two, four or eight warps with up to eight units per lane (five or six where that is enough).
struct Team { int warps, teams, per_lane; };
Team team_of(int64_t units)
{
    Team t;
    t.warps = units <= 512 ? 2 : units <= 1024 ? 4 : 8;
    t.teams = ROW_WARPS / t.warps;
    t.per_lane = units <= 160 * t.warps ? 5 : units <= 192 * t.warps ? 6 : 8;
    return t;
}

template <typename T, bool EDGE>
cudaError_t forward_as(const NormArgs &a, int units, int sms, cudaStream_t s)
{
    constexpr int V = Unit<T>::V;
    const size_t params = (size_t)units * V * 8, row = (size_t)units * 16;
    if (a.period && units <= 256) {
        const int u = (units + 31) / 32, per_sm = u > 4 ? 2 : u > 2 ? 3 : 4;      // as many as are resident
        const int beside = units <= 4 ? 8 : units <= 8 ? 4 : units <= 16 ? 2 : 1; // rows side by side in a warp
        const dim3 grid((unsigned)shared_out(a.rows, a.period, ROW_WARPS * beside, sms * per_sm));
        const int stages = ring_stages(per_sm, params, ROW_WARPS * beside * row);
        const size_t smem = params + ROW_WARPS * beside * stages * row;
        if (beside == 8) return launch_with(norm_forward_kernel<T, 4, 1, EDGE, false>, grid, 256, smem, s, a, stages);
        if (beside == 4) return launch_with(norm_forward_kernel<T, 8, 1, EDGE, false>, grid, 256, smem, s, a, stages);
        if (beside == 2) return launch_with(norm_forward_kernel<T, 16, 1, EDGE, false>, grid, 256, smem, s, a, stages);
        if (u <= 1) return launch_with(norm_forward_kernel<T, 32, 1, EDGE, false>, grid, 256, smem, s, a, stages);
        if (u <= 2) return launch_with(norm_forward_kernel<T, 32, 2, EDGE, false>, grid, 256, smem, s, a, stages);
        if (u <= 4) return launch_with(norm_forward_kernel<T, 32, 4, EDGE, false>, grid, 256, smem, s, a, stages);
        return launch_with(norm_forward_kernel<T, 32, 8, EDGE, false>, grid, 256, smem, s, a, stages);
    }
    if (a.period && units <= ROW_UNITS) {
        const Team t = team_of(units);
        NormArgs b = a;
        b.team = t.warps;
        const int per_sm = std::max(1, std::min(2, (int)(SM_SHARED / (params + 2 * t.teams * row))));
        const dim3 grid((unsigned)shared_out(a.rows, a.period, t.teams, sms * per_sm));
        const int stages = ring_stages(per_sm, params, t.teams * row);
        const size_t smem = params + t.teams * stages * row;
        if (t.per_lane == 5) return launch_with(norm_forward_kernel<T, 32, 5, EDGE, true>, grid, 32 * t.warps * t.teams, smem, s, b, stages);
        if (t.per_lane == 6) return launch_with(norm_forward_kernel<T, 32, 6, EDGE, true>, grid, 32 * t.warps * t.teams, smem, s, b, stages);
        return launch_with(norm_forward_kernel<T, 32, 8, EDGE, true>, grid, 32 * t.warps * t.teams, smem, s, b, stages);
    }
    const int threads = any_threads(a.cols);
    const dim3 grid((unsigned)std::min<int64_t>(a.rows, (int64_t)sms * (2048 / threads)));
    return launch_dependent(norm_forward_wide_kernel<T>, grid, dim3(threads), 0, s, 1, a);
}

// The backward row kernel's form for rows of that many units: rows at a time in a CTA, lanes per row (eight units per lane: with fewer, what a row costs
// besides them counted for more; 32768 x 1024 in four units 75 us, in eight 40), threads and CTAs per SM (by their registers), and CTAs of a cluster: as many as fill the SMs of a GPC whatever its number of SMs.
struct BackwardForm { int rows, lanes, per_lane, threads, team, per_sm, cluster; };
BackwardForm backward_form(int64_t units)
{
    BackwardForm f = {1, 32, 8, 32 * ROW_WARPS, 1, 1, 0};
    if (units <= 256) {
        f.lanes = units <= 32 ? 4 : units <= 64 ? 8 : units <= 128 ? 16 : 32;
        f.rows = ROW_WARPS * 32 / f.lanes;
        f.per_lane = units <= 4 ? 1 : units <= 8 ? 2 : units <= 16 ? 4 : 8;
        f.per_sm = f.per_lane == 1 ? 3 : f.per_lane < 8 ? 2 : 1;
    } else {
        const Team t = team_of(units);
        f.rows = t.teams;
        f.per_lane = t.per_lane;
        f.team = t.warps;
        f.threads = 32 * t.warps * t.teams;
        // Sixteen warps of three units in place of eight of six: BF16 up to 12 % less time, FP32 from 8 % less to 5 % longer, at 320 to 1536 units (6007 x 5461 BF16 without dbias
        // 64 -> 58 us).  In place of five units they take up to 15 % longer (at 320 units with dbias 44 %), of eight (as four) 14 % less to 13 % longer: not there.
        if (t.per_lane == 6) { f.per_lane = 3; f.team *= 2; f.threads *= 2; }
    }
    f.cluster = f.per_sm == 1 ? 2 : f.per_sm == 2 ? 4 : 8;
    return f;
}
// CTAs of the backward row kernel, a multiple of its classes and, where there are enough, of its clusters.
int64_t backward_ctas(int64_t rows, int64_t units, int period, int sms, int *cluster)
{
    const BackwardForm f = backward_form(units);
    int64_t ctas = shared_out(rows, period, 2 * f.rows, (int64_t)sms * f.per_sm);
    *cluster = ctas >= 2 * f.cluster ? f.cluster : 1;
    const int64_t by = std::max<int64_t>(*cluster, period);
    if (ctas > by) ctas = ctas / by * by;
    if (ctas % *cluster) *cluster = 1;
    return ctas;
}
// Partial rows of column sums that a backward pass leaves.
int backward_parts(int64_t rows, int64_t units, int period, int sms)
{
    if (units > ROW_UNITS || period == 0) return (int)std::max<int64_t>(1, std::min<int64_t>((rows + 31) / 32, 2 * sms));
    int cluster;
    const int64_t ctas = backward_ctas(rows, units, period, sms, &cluster);
    return (int)(ctas / cluster);
}
// ... and the most for any alignment of the matrices.
int most_parts(const tsr_norm_desc &d, int sms)
{
    const int V = 16 / type_bytes(d.dtype);
    int most = backward_parts(d.rows, 0, 0, sms);
    for (int period = 1; period <= V; period *= 2)
        for (int shift = 0; shift < V; ++shift) most = std::max(most, backward_parts(d.rows, (d.cols + shift + V - 1) / V, period, sms));
    return most;
}

template <typename T, bool DB, bool EDGE>
cudaError_t backward_as(const NormArgs &a, int units, int sms, cudaStream_t s)
{
    constexpr int V = Unit<T>::V;
    const BackwardForm f = backward_form(units);
    int cluster;
    const int64_t ctas = backward_ctas(a.rows, units, a.period, sms, &cluster);
    const size_t fixed = f.per_lane > 2 ? (size_t)units * V * 4 : 0, stage = (size_t)16 * f.rows * (f.lanes == 4 ? slot_units<4>(units) : 2 * units);
    const int stages = ring_stages(f.per_sm, fixed, stage);
    // (the sums at the end take up to two stages)
    const int sets = f.team > 1 ? f.rows : ROW_WARPS;
    const size_t smem = std::max(fixed + stages * stage, (size_t)units * V * sets * (DB ? 8 : 4));
    const dim3 grid((unsigned)(ctas / cluster), 1, cluster);
    NormArgs b = a;
    b.team = f.team;
    const auto launch = [&](auto kernel) { return launch_with(kernel, grid, f.threads, smem, s, b, stages, cluster); };
    if (units <= 4) return launch(norm_backward_kernel<T, 4, 1, DB, EDGE, false, 3>);
    if (units <= 8) return launch(norm_backward_kernel<T, 4, 2, DB, EDGE, false, 2>);
    if (units <= 16) return launch(norm_backward_kernel<T, 4, 4, DB, EDGE, false, 2>);
    if (units <= 32) return launch(norm_backward_kernel<T, 4, 8, DB, EDGE, false, 1>);
    if (units <= 64) return launch(norm_backward_kernel<T, 8, 8, DB, EDGE, false, 1>);
    if (units <= 128) return launch(norm_backward_kernel<T, 16, 8, DB, EDGE, false, 1>);
    if (units <= 256) return launch(norm_backward_kernel<T, 32, 8, DB, EDGE, false, 1>);
    if (f.per_lane == 3) return launch(norm_backward_kernel<T, 32, 3, DB, EDGE, true, 1, 16>);
    if (f.per_lane == 5) return launch(norm_backward_kernel<T, 32, 5, DB, EDGE, true, 1>);
    return launch(norm_backward_kernel<T, 32, 8, DB, EDGE, true, 1>);
}

template <typename T>
cudaError_t forward_of(const NormArgs &a, int units, int sms, cudaStream_t s)
{
    return has_edges(a, Unit<T>::V) ? forward_as<T, true>(a, units, sms, s) : forward_as<T, false>(a, units, sms, s);
}
template <typename T>
cudaError_t backward_of(const NormArgs &a, int units, int sms, cudaStream_t s)
{
    if (has_edges(a, Unit<T>::V)) return a.want_db ? backward_as<T, true, true>(a, units, sms, s) : backward_as<T, false, true>(a, units, sms, s);
    return a.want_db ? backward_as<T, true, false>(a, units, sms, s) : backward_as<T, false, false>(a, units, sms, s);
}

template <typename T>
cudaError_t backward_wide(const NormArgs &a, int parts, int sms, cudaStream_t s)
{
    if (a.want_dw || a.want_db) {      // first: dx may replace dy
        const cudaError_t e = launch_dependent(norm_columns_kernel<T>, dim3((unsigned)((a.cols + 255) / 256), (unsigned)parts), dim3(256), 0, s, 1, a, (a.rows + parts - 1) / parts);
        if (e != cudaSuccess) return e;
    }
    if (!a.y) return cudaSuccess;
    const int threads = any_threads(a.cols);
    return launch_dependent(norm_backward_wide_kernel<T>, dim3((unsigned)std::min<int64_t>(a.rows, (int64_t)sms * (2048 / threads))), dim3(threads), 0, s, 1, a);
}

constexpr int64_t MOST_COLS = 0x7fffffff - 1023, MOST_ROWS = (int64_t)1 << 40;

tsr_status check_norm(const tsr_norm_desc *d)
{
    if (!d) return TSR_ERR_INVALID_ARG;
    if (!type_ok(d->dtype) || !type_ok(d->p_dtype) || !type_ok(d->g_dtype)) return TSR_ERR_UNSUPPORTED;
    if (d->rows < 0 || d->cols < 0 || d->rows > MOST_ROWS || d->cols > MOST_COLS) return TSR_ERR_SHAPE;
    if (!(d->eps >= 0.f) || !isfinite(d->eps) || (d->center != 0 && d->center != 1)) return TSR_ERR_INVALID_ARG;
    return TSR_OK;
}
tsr_status check_rows(const tsr_matrix &m, const tsr_norm_desc &d, bool want)
{
    if (!m.data) return want && d.rows > 0 && d.cols > 0 ? TSR_ERR_INVALID_ARG : TSR_OK;
    if (!extent_ok(d.rows, d.cols, m.ld)) return TSR_ERR_SHAPE;
    return aligned_to(m.data, type_bytes(d.dtype)) ? TSR_OK : TSR_ERR_ALIGNMENT;
}

}  // namespace
}  // namespace tsr

using namespace tsr;

extern "C" tsr_status tsr_norm_forward(const tsr_norm_desc *desc, tsr_matrix x, const void *weight, const void *bias, tsr_matrix y, float *stats, void *stream)
{
    tsr_status st = check_norm(desc);
    if (st != TSR_OK) return st;
    const tsr_norm_desc &d = *desc;
    if ((st = check_rows(x, d, true)) != TSR_OK || (st = check_rows(y, d, true)) != TSR_OK) return st;
    if (!aligned_to(weight, type_bytes(d.p_dtype)) || !aligned_to(bias, type_bytes(d.p_dtype)) || !aligned_to(stats, 8)) return TSR_ERR_ALIGNMENT;
    if (d.rows == 0 || d.cols == 0) return TSR_OK;
    const int sms = device_sms();
    if (!sms) return TSR_ERR_CUDA;
    NormArgs a = {};
    a.x = x.data; a.ldx = x.ld; a.y = y.data; a.ldy = y.ld;
    a.weight = weight; a.bias = bias; a.p_bf16 = d.p_dtype == TSR_BF16;
    a.stats = stats; a.rows = d.rows; a.cols = (int)d.cols; a.center = d.center; a.eps = d.eps; a.inv_n = 1.f / (float)d.cols;
    const tsr_matrix *all[2] = {&x, &y};
    int units = 0;
    a.period = common_period(d, all, 2, &units);
    cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = d.dtype == TSR_BF16 ? forward_of<bf16>(a, units, sms, s) : forward_of<float>(a, units, sms, s);
    return e == cudaSuccess ? TSR_OK : TSR_ERR_CUDA;
}

extern "C" tsr_status tsr_norm_workspace_bytes(const tsr_norm_desc *desc, size_t *bytes)
{
    const tsr_status st = check_norm(desc);
    if (st != TSR_OK) return st;
    if (!bytes) return TSR_ERR_INVALID_ARG;
    const int sms = device_sms();
    *bytes = (size_t)2 * 4 * (size_t)desc->cols * (size_t)most_parts(*desc, sms ? sms : 148);
    return TSR_OK;
}

extern "C" tsr_status tsr_norm_backward(const tsr_norm_desc *desc, tsr_matrix dy, tsr_matrix x, const void *weight, const float *stats, tsr_matrix dx,
                                        void *dweight, void *dbias, void *workspace, size_t workspace_bytes, void *stream)
{
    tsr_status st = check_norm(desc);
    if (st != TSR_OK) return st;
    const tsr_norm_desc &d = *desc;
    if ((st = check_rows(dy, d, true)) != TSR_OK || (st = check_rows(x, d, true)) != TSR_OK || (st = check_rows(dx, d, false)) != TSR_OK) return st;
    if (!stats && d.rows > 0 && d.cols > 0) return TSR_ERR_INVALID_ARG;
    if (!aligned_to(weight, type_bytes(d.p_dtype)) || !aligned_to(dweight, type_bytes(d.g_dtype)) || !aligned_to(dbias, type_bytes(d.g_dtype)) || !aligned_to(stats, 8))
        return TSR_ERR_ALIGNMENT;
    const int known = device_sms(), sms = known ? known : 148;
    if (dweight || dbias) {
        const size_t need = (size_t)2 * 4 * (size_t)d.cols * (size_t)most_parts(d, sms);
        if (need && (!workspace || workspace_bytes < need)) return TSR_ERR_WORKSPACE;
        if (need && !aligned_to(workspace, 256)) return TSR_ERR_ALIGNMENT;
    }
    if (d.cols == 0) return TSR_OK;
    if (!known) return TSR_ERR_CUDA;
    cudaStream_t s = (cudaStream_t)stream;
    NormArgs a = {};
    a.dy = dy.data; a.lddy = dy.ld; a.x = x.data; a.ldx = x.ld; a.y = dx.data; a.ldy = dx.ld;
    a.weight = weight; a.p_bf16 = d.p_dtype == TSR_BF16;
    a.stats_in = stats; a.partial = (float *)workspace; a.rows = d.rows; a.cols = (int)d.cols; a.center = d.center; a.inv_n = 1.f / (float)d.cols;
    a.want_dw = dweight != nullptr; a.want_db = dbias != nullptr;
    const tsr_matrix *all[3] = {&x, &dy, &dx};
    int units = 0;
    a.period = d.rows > 0 ? common_period(d, all, 3, &units) : 0;
    const int parts = backward_parts(d.rows, units, a.period, sms);
    bool direct = false;      // a single part of the row kernel: its sums are the result
    if (d.rows > 0) {
        const bool bf = d.dtype == TSR_BF16;
        direct = parts == 1 && a.period && units <= ROW_UNITS;
        if (direct) a.partial = nullptr;
        a.dw = dweight; a.db = dbias; a.g_bf16 = d.g_dtype == TSR_BF16; a.accumulate = d.accumulate;
        cudaError_t e;
        if (a.period == 0 || units > ROW_UNITS) e = bf ? backward_wide<bf16>(a, parts, sms, s) : backward_wide<float>(a, parts, sms, s);
        else e = bf ? backward_of<bf16>(a, units, sms, s) : backward_of<float>(a, units, sms, s);
        if (e != cudaSuccess) return TSR_ERR_CUDA;
    }
    const bool gb = d.g_dtype == TSR_BF16;
    void *one = dweight ? dweight : dbias, *two = dweight ? dbias : nullptr;
    if (one && !direct && column_finish((const float *)workspace, d.rows ? parts : 0, d.cols, d.cols, one, gb, two, gb, d.accumulate != 0, s) != cudaSuccess) return TSR_ERR_CUDA;
    return TSR_OK;
}
