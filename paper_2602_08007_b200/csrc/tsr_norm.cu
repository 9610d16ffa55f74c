// Norm over rows, forward and backward (formulas in tsr.h).  Both passes are bound by HBM: forward reads x and writes y, backward reads
// x and dy and writes dx, each once; a row stays in registers between its sums and its results.
//
// Forward and backward: rows up to 32 KB are worked on by a warp or a CTA, the next ones in flight.  Distances are formed from the
// row's first entry and then from means: a large mean costs no digits, and a row of equal entries has variance zero.
// Backward: threads keep their columns from row to row, so that the sums for dweight and dbias stay in registers; a CTA leaves one partial row each, and
// column_finish adds them in order.
// Wider rows, and matrices that do not start at the same place in 16 bytes, are read several times (from L2, mostly); their column sums take a
// pass of their own.
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
    float s = 0.f;
    for (int w = 0; w < warps; ++w) s += slot[w];
    return s;
}

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

// Unit j of a row in shared memory; EDGE: the places that hold no entry are `fill`.
template <typename T, bool EDGE>
__device__ __forceinline__ uint4 take_unit(const uint4 *row, int j, int col, int cols, T fill)
{
    constexpr int V = Unit<T>::V;
    uint4 r = row[j];
    if (EDGE && (col < 0 || col + V > cols)) {
        T t[V];
        memcpy(t, &r, 16);
#pragma unroll
        for (int i = 0; i < V; ++i) if (col + i < 0 || col + i >= cols) t[i] = fill;
        memcpy(&r, t, 16);
    }
    return r;
}
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
// EDGE: the places that hold no entry are left alone.
template <typename T, bool EDGE>
__device__ __forceinline__ void store_unit(T *row, int col, int cols, const float2 (&v)[Unit<T>::V / 2])
{
    constexpr int V = Unit<T>::V;
    const uint4 r = unit_of(v);
    if (!EDGE || (col >= 0 && col + V <= cols)) *(uint4 *)(row + col) = r;
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
    for (int i = threadIdx.x; i < rc.units * V; i += blockDim.x) {
        const int c = i - rc.shift, at = shared_at(i / V, i % V / 4, rc.units) + i % 4;
        const bool in = c >= 0 && c < a.cols;
        w[at] = in ? param(a.weight, c, a.p_bf16, 1.f) : 0.f;
        if (b) b[at] = in ? param(a.bias, c, a.p_bf16, 0.f) : 0.f;
    }
}
// Squares without those of `empty` places, each of which had distance `mean` from the mean.  The pivot is an entry of the row, so that what is taken
// away is at most (2 V - 2) mean^2 <= (2 V - 2) squares: four bits at the worst (a row of two entries), none of a row that is long.
template <bool EDGE>
__device__ __forceinline__ float less_empty(float squares, float mean, float empty)
{
    if (!EDGE) return squares;
    const float s = fmaf(-empty * mean, mean, squares);
    return s < 0.f ? 0.f : s;      // (NaN stays)
}
// v <- v rstd w + b over unit j
template <int P>
__device__ __forceinline__ void normed(float2 (&v)[P], float rstd, const float *w, const float *b, int j, int units)
{
#pragma unroll
    for (int i = 0; i < P; i += 2) {
        const float4 ww = *(const float4 *)(w + shared_at(j, i / 2, units)), bb = *(const float4 *)(b + shared_at(j, i / 2, units));
        v[i] = fma2(mul2(v[i], pair(rstd)), make_float2(ww.x, ww.y), make_float2(bb.x, bb.y));
        v[i + 1] = fma2(mul2(v[i + 1], pair(rstd)), make_float2(ww.z, ww.w), make_float2(bb.z, bb.w));
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

// Narrow and middling rows: L lanes per row (32 / L rows side by side in a warp), U units per lane, a ring of `stages` turns per warp; warps do not wait
// for one another.  `Rows` says which rows a group of lanes works on: of all groups of the class, the g-th takes every n-th row.
constexpr int ROW_WARPS = 8;
template <int L>
struct Rows {
    int lane, group;               // within the row; of the CTA
    int left, turns;               // rows of the group, and the most of a group of the warp
    int64_t row, step;
    RowClass rc;
};
template <typename T, int L>
__device__ __forceinline__ Rows<L> rows_of(const NormArgs &a, int cta, int ctas)
{
    constexpr int G = 32 / L;
    Rows<L> r;
    r.rc = row_class<T>(a.x, a.ldx, a.cols, a.period, cta, ctas);
    r.lane = threadIdx.x & (L - 1);
    r.group = threadIdx.x / L;
    r.step = r.rc.step * ROW_WARPS * G;      // (`step` of the class is that of a CTA with one row)
    r.row = r.rc.first + r.rc.step * r.group;
    const int64_t left = r.row < a.rows ? (a.rows - r.row + r.step - 1) / r.step : 0;
    r.left = (int)left;                      // (at most 2^40 rows among the groups of a full grid)
    r.turns = __shfl_sync(0xffffffffu, r.left, 0);      // (the first group of a warp has the most)
    return r;
}

template <typename T, int L, int U, bool EDGE>
__global__ void __launch_bounds__(256, U > 4 ? 2 : U > 2 ? 3 : 4)
norm_forward_kernel(const NormArgs a, int stages)
{
    constexpr int V = Unit<T>::V, P = V / 2, G = 32 / L;
    extern __shared__ float4 shared[];       // w, b, rings
    __shared__ uint64_t bars[ROW_WARPS * NORM_STAGES];
    pdl_trigger();
    pdl_wait();
    const int warp = threadIdx.x >> 5;
    const Rows<L> rows = rows_of<T, L>(a, blockIdx.x, gridDim.x);
    const RowClass &rc = rows.rc;
    const int lane = rows.lane, left = rows.left;
    float *w = (float *)shared, *b = w + rc.units * V;
    const uint4 *ring = (const uint4 *)(b + rc.units * V) + (warp * stages * G + rows.group % G) * rc.units;
    uint64_t *bar = bars + warp * NORM_STAGES;
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
    if ((threadIdx.x & 31) == 0) {
        for (int i = 0; i < stages; ++i) mbar_init(smem_u32(bar + i), G);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
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
        const T pivot = a.center ? *((const T *)row + rc.shift) : T(0.f);      // also stands in the places that hold no entry
        const float x0 = load_f(&pivot);
        float2 v[U][P], sum = pair(0.f), q = pair(0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * L + lane;
            unit_pairs(j < rc.units ? take_unit<T, EDGE>(row, j, j * V - rc.shift, a.cols, pivot) : make_uint4(0, 0, 0, 0), v[u]);
        }
        __syncwarp();
        if (lane == 0 && turn + stages < rows.turns) request(stage);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u * L + lane >= rc.units) continue;
            less(v[u], x0);
#pragma unroll
            for (int i = 0; i < P; ++i) sum = add2(sum, v[u][i]);
        }
        const float mean = a.center ? lanes_sum<L>(sum.x + sum.y) * a.inv_n : 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u * L + lane >= rc.units) continue;
            less(v[u], mean);
#pragma unroll
            for (int i = 0; i < P; ++i) q = fma2(v[u][i], v[u][i], q);
        }
        const float rstd = rsqrtf(less_empty<EDGE>(lanes_sum<L>(q.x + q.y), mean, empty) * a.inv_n + a.eps);
        if (stats && lane == 0 && mine) *(float2 *)stats = make_float2(x0 + mean, rstd);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * L + lane;
            if (j >= rc.units || !mine) continue;
            normed(v[u], rstd, w, b, j, rc.units);
            store_unit<T, EDGE>(y, j * V - rc.shift, a.cols, v[u]);
        }
        y += next_y;
        if (stats) stats += 2 * rows.step;
    }
    note_gave_up(gave_up);
}

// Wider rows: a CTA per row, U units per thread.  Each thread forms mean and sum of squared distances of its own entries; two sets of n1 and n2
// entries join by
//     mean = mean1 + d n2 / (n1 + n2),   squares = squares1 + squares2 + d^2 n1 n2 / (n1 + n2),   d = mean2 - mean1
// (T. Chan, G. Golub, R. LeVeque 1979), so that a row takes one round of exchanges and one barrier, and digits are lost to neither a large mean nor an
// outlier.  The factors are the same for every row.
template <typename T, int U, bool EDGE, int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS)
norm_forward_row_kernel(const NormArgs a, int stages)
{
    constexpr int V = Unit<T>::V, P = V / 2;
    extern __shared__ float4 shared[];       // w, b, ring
    __shared__ uint64_t bars[NORM_STAGES];
    __shared__ float2 slots[2][16], factors[16];
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 31, warp = tid >> 5, warps = threads >> 5;
    const RowClass rc = row_class<T>(a.x, a.ldx, a.cols, a.period, blockIdx.x, gridDim.x);
    float *w = (float *)shared, *b = w + rc.units * V;
    const uint4 *ring = (const uint4 *)(b + rc.units * V);
    int64_t left = rc.first < a.rows ? (a.rows - rc.first + rc.step - 1) / rc.step : 0;
    const T *ask = (const T *)a.x + rc.first * a.ldx;
    auto request = [&](int stage) {      // the next row, by one thread
        mbar_expect_tx(smem_u32(bars + stage), (uint32_t)rc.units * 16u);
        ask_row<T>(smem_u32(ring + stage * rc.units), ask, rc, smem_u32(bars + stage));
        ask += rc.step * a.ldx;
    };
    if (tid == 0) {
        for (int i = 0; i < stages; ++i) mbar_init(smem_u32(bars + i), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int i = 0; i < stages && i < left; ++i) request(i);
    }
    share_params<T>(a, rc, w, b);
    int own = 0, places = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int j = u * threads + tid, col = j * V - rc.shift;
        own += max(0, min(col + V, a.cols) - max(col, 0));
        if (j < rc.units) places += V;
    }
    const float empty = (float)(places - own);
    const float inv_own = own ? 1.f / (float)own : 0.f;
    float f2[5], f12[5], count = (float)own;      // n2 / (n1 + n2) and n1 n2 / (n1 + n2) of the five exchanges within a warp
#pragma unroll
    for (int k = 0; k < 5; ++k) {
        const float other = __shfl_xor_sync(0xffffffffu, count, 1 << k), both = count + other;
        f2[k] = both > 0.f ? other / both : 0.f;
        f12[k] = count * f2[k];
        count = both;
    }
    if (lane == 0) slots[0][warp].x = count;
    __syncthreads();
    if (tid == 0) {
        float before = 0.f;
        for (int i = 0; i < warps; ++i) {
            const float n = slots[0][i].x, both = before + n, f = both > 0.f ? n / both : 0.f;
            factors[i] = make_float2(f, before * f);
            before = both;
        }
    }
    __syncthreads();
    bool gave_up = false;
    int turn = 0, stage = 0;
    uint32_t phase = 0;
    T *y = (T *)a.y + rc.first * a.ldy;
    float *stats = a.stats ? a.stats + 2 * rc.first : nullptr;
    for (; left > 0; --left, turn ^= 1) {
        await_row(smem_u32(bars + stage), phase, gave_up);
        const uint4 *row = ring + stage * rc.units;
        const T pivot = a.center ? *((const T *)row + rc.shift) : T(0.f);      // also stands in the places that hold no entry
        const float x0 = load_f(&pivot);
        float2 v[U][P], sum = pair(0.f), q = pair(0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * threads + tid;
            if (j >= rc.units) continue;
            unit_pairs(take_unit<T, EDGE>(row, j, j * V - rc.shift, a.cols, pivot), v[u]);
            less(v[u], x0);
#pragma unroll
            for (int i = 0; i < P; ++i) sum = add2(sum, v[u][i]);
        }
        const float mine = a.center ? (sum.x + sum.y) * inv_own : 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u * threads + tid >= rc.units) continue;
            less(v[u], mine);
#pragma unroll
            for (int i = 0; i < P; ++i) q = fma2(v[u][i], v[u][i], q);
        }
        float mean = mine, squares = less_empty<EDGE>(q.x + q.y, mine, empty);
#pragma unroll
        for (int k = 0; k < 5; ++k) {
            const float d = __shfl_xor_sync(0xffffffffu, mean, 1 << k) - mean;
            squares = fmaf(d * d, f12[k], squares + __shfl_xor_sync(0xffffffffu, squares, 1 << k));
            mean = fmaf(d, f2[k], mean);
        }
        if (lane == 0) slots[turn][warp] = make_float2(mean, squares);
        // One barrier per turn: the slots of the turn before last are written again only after the last one's, and the row has left its stage.
        __syncthreads();
        if (tid == 0 && left > stages) request(stage);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
        mean = slots[turn][0].x;
        squares = slots[turn][0].y;
        for (int i = 1; i < warps; ++i) {
            const float2 t = slots[turn][i], f = factors[i];
            const float d = t.x - mean;
            squares = fmaf(d * d, f.y, squares + t.y);
            mean = fmaf(d, f.x, mean);
        }
        const float rstd = rsqrtf(squares * a.inv_n + a.eps);
        if (stats && tid == 0) *(float2 *)stats = make_float2(x0 + mean, rstd);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * threads + tid;
            if (j >= rc.units) continue;
            less(v[u], mean - mine);
            normed(v[u], rstd, w, b, j, rc.units);
            store_unit<T, EDGE>(y, j * V - rc.shift, a.cols, v[u]);
        }
        y += rc.step * a.ldy;
        if (stats) stats += 2 * rc.step;
    }
    note_gave_up(gave_up);
}

// Any width and alignment: three passes over the row.
template <typename T>
__global__ void __launch_bounds__(1024)
norm_forward_wide_kernel(const NormArgs a)
{
    __shared__ float slots[2][32];
    pdl_trigger();
    pdl_wait();
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = (const T *)a.x + r * a.ldx;
        float x0 = 0.f, m0 = 0.f, q = 0.f;
        if (a.center) {
            x0 = load_f(x);
            for (int c = threadIdx.x; c < a.cols; c += blockDim.x) m0 += load_f(x + c) - x0;
            m0 = cta_sum(m0, slots[0]) * a.inv_n;
        }
        const float mu = x0 + m0;
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) { const float d = load_f(x + c) - x0 - m0; q = fmaf(d, d, q); }
        const float rstd = rsqrtf(cta_sum(q, slots[1]) * a.inv_n + a.eps);
        if (a.stats && threadIdx.x == 0) { a.stats[2 * r] = mu; a.stats[2 * r + 1] = rstd; }
        T *y = (T *)a.y + r * a.ldy;
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x)
            store_f(y + c, fmaf((load_f(x + c) - x0 - m0) * rstd, param(a.weight, c, a.p_bf16, 1.f), param(a.bias, c, a.p_bf16, 0.f)));
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

// Rows of up to 256 units: L lanes per row, U units per lane, as in the forward pass; x and dy come through the ring.  A lane keeps its columns from
// row to row, so that the column sums stay in registers (128 of them at U = 8 and BF16).  Weight is in registers up to two units, else in shared
// memory.  DB: the sums of dy are wanted too.
template <typename T, int L, int U, bool DB, bool EDGE, int CTAS>
__global__ void __launch_bounds__(256, CTAS)
norm_backward_lanes_kernel(const NormArgs a, int stages)
{
    constexpr int V = Unit<T>::V, P = V / 2, G = 32 / L;
    constexpr bool KEEP = U <= 2;
    extern __shared__ float4 shared[];       // weight (unless kept), rings; at the end the column sums
    __shared__ uint64_t bars[ROW_WARPS * NORM_STAGES];
    pdl_trigger();
    pdl_wait();
    const int warp = threadIdx.x >> 5;
    const int cta = blockIdx.x * gridDim.z + blockIdx.z;
    const Rows<L> rows = rows_of<T, L>(a, cta, gridDim.x * gridDim.z);
    const RowClass &rc = rows.rc;
    const int lane = rows.lane, left = rows.left;
    float *weight = (float *)shared;
    const uint4 *ring = (const uint4 *)(KEEP ? weight : weight + rc.units * V) + (warp * stages * G + rows.group % G) * 2 * rc.units;
    uint64_t *bar = bars + warp * NORM_STAGES;
    const T *ask_x = (const T *)a.x + rows.row * a.ldx, *ask_dy = (const T *)a.dy + rows.row * a.lddy;
    const int64_t next_x = rows.step * a.ldx, next_dy = rows.step * a.lddy, next_y = rows.step * a.ldy;
    int asked = 0;
    auto request = [&](int stage) {      // the next row, by the first lane of a group
        const bool any = asked++ < left;
        const uint32_t to = smem_u32(bar + stage), bytes = (uint32_t)rc.units * 16u, at = smem_u32(ring + stage * G * 2 * rc.units);
        mbar_expect_tx(to, any ? 2 * bytes : 0u);
        if (!any) return;
        ask_row<T>(at, ask_x, rc, to);
        ask_row<T>(at + bytes, ask_dy, rc, to);
        ask_x += next_x;
        ask_dy += next_dy;
    };
    if ((threadIdx.x & 31) == 0) {
        for (int i = 0; i < stages; ++i) mbar_init(smem_u32(bar + i), G);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
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
                const int c = (u * L + lane) * V - rc.shift + 2 * i;
                kept[u][i] = make_float2(c >= 0 && c < a.cols ? param(a.weight, c, a.p_bf16, 1.f) : 0.f, c + 1 >= 0 && c + 1 < a.cols ? param(a.weight, c + 1, a.p_bf16, 1.f) : 0.f);
            }
        }
    if (!KEEP) {
        share_params<T>(a, rc, weight, nullptr);
        __syncthreads();
    }
    auto weights = [&](int u, float2 (&w)[P]) {
#pragma unroll
        for (int i = 0; i < P; i += 2) {
            if constexpr (KEEP) {
                w[i] = kept[u][i];
                w[i + 1] = kept[u][i + 1];
            } else {
                const float4 t = *(const float4 *)(weight + shared_at(u * L + lane, i / 2, rc.units));
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
        const uint4 *row = ring + stage * G * 2 * rc.units;
        const bool mine = G == 1 || turn < left;
        uint4 x[U], g[U];
        float2 s1 = pair(0.f), s2 = pair(0.f);
        const float2 less_mu = pair(-st.x), r = pair(st.y);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * L + lane, col = j * V - rc.shift;
            if (j >= rc.units || !mine) continue;
            x[u] = take_unit<T, EDGE>(row, j, col, a.cols, T(0.f));
            g[u] = take_unit<T, EDGE>(row + rc.units, j, col, a.cols, T(0.f));
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
        const float2 s = lanes_sum<L>(make_float2(s1.x + s1.y, s2.x + s2.y), lane);
        if (lane == 0 && turn + stages < rows.turns) request(stage);      // (after the shuffles: every lane has read its units)
        if (++stage == stages) { stage = 0; phase ^= 1u; }
        if (a.y && mine) {
            // dx = r g w - r mean(g w) - (x - mu) r^2 mean(g w h)
            const float2 c1 = pair(a.center ? -s.x * a.inv_n * st.y : 0.f), c2 = pair(-s.y * a.inv_n * st.y * st.y);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = u * L + lane;
                if (j >= rc.units) continue;
                float2 w[P], xv[P], gv[P];
                weights(u, w);
                unit_pairs(x[u], xv);
                unit_pairs(g[u], gv);
#pragma unroll
                for (int i = 0; i < P; ++i) gv[i] = fma2(mul2(gv[i], w[i]), r, fma2(add2(xv[i], less_mu), c2, c1));
                store_unit<T, EDGE>(y, j * V - rc.shift, a.cols, gv);
            }
        }
        y += next_y;
    }
    note_gave_up(gave_up);
    if (!a.want_dw && !DB) return;
    // The column sums: over the groups of a warp, then (in the place of weight and rings) over the warps.
    const int width = rc.units * V, set = DB ? 2 * width : width;
    float *sums = (float *)shared;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int j = u * L + lane;
#pragma unroll
        for (int o = L; o < 32; o <<= 1)
#pragma unroll
            for (int i = 0; i < P; ++i) {
                dw[u][i] = add2(dw[u][i], make_float2(__shfl_xor_sync(0xffffffffu, dw[u][i].x, o), __shfl_xor_sync(0xffffffffu, dw[u][i].y, o)));
                if (DB) db[DB ? u : 0][i] = add2(db[DB ? u : 0][i], make_float2(__shfl_xor_sync(0xffffffffu, db[DB ? u : 0][i].x, o), __shfl_xor_sync(0xffffffffu, db[DB ? u : 0][i].y, o)));
            }
        if (j >= rc.units || rows.group % G) continue;
        keep_sums(sums + warp * set + j * V, dw[u]);
        if (DB) keep_sums(sums + warp * set + width + j * V, db[DB ? u : 0]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < set; i += 256) {
        float t = sums[i];
#pragma unroll
        for (int k = 1; k < ROW_WARPS; ++k) t += sums[k * set + i];
        sums[i] = t;
    }
    add_up<T, DB>(a, sums);
}

// Wider rows: a CTA walks over rows of its class, R of them at a time; U units per thread, whose columns stay the same, so that weight and column sums
// stay in registers.  x and dy come through a ring of `stages`, R rows of each in one.  Two rows at a time share one wait, one barrier, and six shuffles
// (instead of twenty) for their four sums: what surrounds the arithmetic was half of the instructions with one.
//
// The sums of a warp, R pairs (s1, s2), over its lanes: with each exchange a lane keeps half of the values; lane 8 k has the k-th at last.
template <int R>
__device__ __forceinline__ float sums_of_warp(const float (&v)[2 * R], int lane)
{
    float k0, k1;
    if constexpr (R == 2) {
        const bool hi = lane & 16;
        k0 = (hi ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, hi ? v[0] : v[2], 16);
        k1 = (hi ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, hi ? v[1] : v[3], 16);
    } else {
        k0 = v[0] + __shfl_xor_sync(0xffffffffu, v[0], 16);
        k1 = v[1] + __shfl_xor_sync(0xffffffffu, v[1], 16);
    }
    const bool hi = lane & 8;
    float k = (hi ? k1 : k0) + __shfl_xor_sync(0xffffffffu, hi ? k0 : k1, 8);
#pragma unroll
    for (int o = 4; o; o >>= 1) k += __shfl_xor_sync(0xffffffffu, k, o);
    return k;
}
template <typename T, int U, bool DB, bool EDGE, int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS)
norm_backward_kernel(const NormArgs a, int stages)
{
    constexpr int V = Unit<T>::V, P = V / 2, R = U <= 2 ? 2 : 1;      // (rows of four units per thread fill the registers one at a time)
    constexpr bool KEEP = U <= 2;                                     // weight in registers; otherwise in shared memory
    extern __shared__ float4 shared[];       // weight (unless kept), ring; at the end the column sums
    __shared__ uint64_t bars[NORM_STAGES];
    __shared__ float4 slots[2][THREADS / 32];      // the sums of every warp, (s1, s2) of R rows
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x, threads = blockDim.x, warp = tid >> 5, lane = tid & 31, warps = threads >> 5;
    const int ctas = gridDim.x * gridDim.z, cta = blockIdx.x * gridDim.z + blockIdx.z;
    const RowClass rc = row_class<T>(a.x, a.ldx, a.cols, a.period, cta, ctas);
    float *weight = (float *)shared;
    const uint4 *ring = (const uint4 *)(KEEP ? weight : weight + rc.units * V);      // per stage and row x, then dy
    int64_t left = rc.first < a.rows ? (a.rows - rc.first + rc.step - 1) / rc.step : 0;
    int64_t to_ask = left;
    const T *ask_x = (const T *)a.x + rc.first * a.ldx, *ask_dy = (const T *)a.dy + rc.first * a.lddy;
    auto request = [&](int stage) {      // the next rows, by one thread
        const uint32_t bar = smem_u32(bars + stage), bytes = (uint32_t)rc.units * 16u;
        uint32_t at = smem_u32(ring + stage * R * 2 * rc.units);
        const int n = to_ask < R ? (int)to_ask : R;
        mbar_expect_tx(bar, n * 2 * bytes);
        for (int k = 0; k < n; ++k, at += 2 * bytes) {
            ask_row<T>(at, ask_x, rc, bar);
            ask_row<T>(at + bytes, ask_dy, rc, bar);
            ask_x += rc.step * a.ldx;
            ask_dy += rc.step * a.lddy;
        }
        to_ask -= n;
    };
    if (tid == 0) {
        for (int i = 0; i < stages; ++i) mbar_init(smem_u32(bars + i), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int i = 0; i < stages && to_ask > 0; ++i) request(i);
    }
    float2 kept[KEEP ? U : 1][P], dw[U][P], db[DB ? U : 1][P];
    if constexpr (KEEP) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int c = (u * threads + tid) * V - rc.shift + 2 * i;
                kept[u][i] = make_float2(c >= 0 && c < a.cols ? param(a.weight, c, a.p_bf16, 1.f) : 0.f, c + 1 >= 0 && c + 1 < a.cols ? param(a.weight, c + 1, a.p_bf16, 1.f) : 0.f);
            }
    } else share_params<T>(a, rc, weight, nullptr);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < P; ++i) {
            dw[u][i] = pair(0.f);
            if (DB) db[u][i] = pair(0.f);
        }
    auto weights = [&](int u, float2 (&w)[P]) {
#pragma unroll
        for (int i = 0; i < P; i += 2) {
            if constexpr (KEEP) {
                w[i] = kept[u][i];
                w[i + 1] = kept[u][i + 1];
            } else {
                const float4 t = *(const float4 *)(weight + shared_at(u * threads + tid, i / 2, rc.units));
                w[i] = make_float2(t.x, t.y);
                w[i + 1] = make_float2(t.z, t.w);
            }
        }
    };
    __syncthreads();
    bool gave_up = false;
    int turn = 0, stage = 0;
    uint32_t phase = 0;
    T *y = (T *)a.y + rc.first * a.ldy;
    const int64_t next_y = rc.step * a.ldy;
    const float2 *stats = (const float2 *)a.stats_in + rc.first;
    float2 next[R];
    auto ask_stats = [&](int64_t n) {      // of the coming rows, n of which exist
#pragma unroll
        for (int k = 0; k < R; ++k) next[k] = k < n ? stats[k * rc.step] : pair(0.f);
        stats += R * rc.step;
    };
    ask_stats(left);
    for (; left > 0; left -= R, turn ^= 1) {
        float2 st[R];
#pragma unroll
        for (int k = 0; k < R; ++k) st[k] = next[k];
        ask_stats(left - R);
        await_row(smem_u32(bars + stage), phase, gave_up);
        const uint4 *row = ring + stage * R * 2 * rc.units;
        const bool both = left > 1;
        uint4 x[R][U], g[R][U];
        float2 s1[R], s2[R];
#pragma unroll
        for (int k = 0; k < R; ++k) s1[k] = s2[k] = pair(0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * threads + tid, col = j * V - rc.shift;
            if (j >= rc.units) continue;
            float2 w[P];
            weights(u, w);
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (k == 0 || both) {
                    x[k][u] = take_unit<T, EDGE>(row + 2 * k * rc.units, j, col, a.cols, T(0.f));
                    g[k][u] = take_unit<T, EDGE>(row + (2 * k + 1) * rc.units, j, col, a.cols, T(0.f));
                } else x[k][u] = g[k][u] = make_uint4(0, 0, 0, 0);
                float2 xv[P], gv[P];
                unit_pairs(x[k][u], xv);
                unit_pairs(g[k][u], gv);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float2 h = mul2(add2(xv[i], pair(-st[k].x)), pair(st[k].y));
                    dw[u][i] = fma2(gv[i], h, dw[u][i]);
                    if (DB) db[u][i] = add2(db[u][i], gv[i]);
                    const float2 gw = mul2(gv[i], w[i]);
                    s1[k] = add2(s1[k], gw);
                    s2[k] = fma2(gw, h, s2[k]);
                }
            }
        }
        float v[2 * R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            v[2 * k] = s1[k].x + s1[k].y;
            v[2 * k + 1] = s2[k].x + s2[k].y;
        }
        // One barrier per turn: the slots of the turn before last are written again only after the last one's, and the rows have left their stage.
        const float mine = sums_of_warp<R>(v, lane);
        if ((lane & 7) == 0 && (lane >> 3) < 2 * R) ((float *)&slots[turn][warp])[lane >> 3] = mine;
        if (warps > 1) __syncthreads();
        else __syncwarp();
        if (tid == 0 && to_ask > 0) request(stage);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
        if (a.y) {
            float2 c1 = pair(0.f), c2 = pair(0.f);      // of the two rows
            for (int i = 0; i < warps; ++i) {
                const float4 t = slots[turn][i];
                c1 = add2(c1, make_float2(t.x, R == 2 ? t.z : 0.f));
                c2 = add2(c2, make_float2(t.y, R == 2 ? t.w : 0.f));
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (k && !both) break;
                // dx = r g w - r mean(g w) - (x - mu) r^2 mean(g w h)
                const float f1 = a.center ? -(k ? c1.y : c1.x) * a.inv_n * st[k].y : 0.f, f2 = -(k ? c2.y : c2.x) * a.inv_n * st[k].y * st[k].y;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int j = u * threads + tid;
                    if (j >= rc.units) continue;
                    float2 w[P], xv[P], gv[P];
                    weights(u, w);
                    unit_pairs(x[k][u], xv);
                    unit_pairs(g[k][u], gv);
#pragma unroll
                    for (int i = 0; i < P; ++i) gv[i] = fma2(mul2(gv[i], w[i]), pair(st[k].y), fma2(add2(xv[i], pair(-st[k].x)), pair(f2), pair(f1)));
                    store_unit<T, EDGE>(y, j * V - rc.shift, a.cols, gv);
                }
                y += next_y;
            }
        }
    }
    note_gave_up(gave_up);
    if (!a.want_dw && !DB) return;
    // Column sums of this CTA, by unit: dweight's, then dbias's, in the place of weight and ring.
    __syncthreads();
    float *sums = (float *)shared;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int j = u * threads + tid;
        if (j >= rc.units) continue;
        keep_sums(sums + j * V, dw[u]);
        if (DB) keep_sums(sums + rc.units * V + j * V, db[DB ? u : 0]);
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
    if (smem > 40 * 1024) {      // (48 KB less what is static)
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    return launch_dependent(kernel, grid, dim3(threads), smem, s, cluster, a, stages);
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
        if (beside == 8) return launch_with(norm_forward_kernel<T, 4, 1, EDGE>, grid, 256, smem, s, a, stages);
        if (beside == 4) return launch_with(norm_forward_kernel<T, 8, 1, EDGE>, grid, 256, smem, s, a, stages);
        if (beside == 2) return launch_with(norm_forward_kernel<T, 16, 1, EDGE>, grid, 256, smem, s, a, stages);
        if (u <= 1) return launch_with(norm_forward_kernel<T, 32, 1, EDGE>, grid, 256, smem, s, a, stages);
        if (u <= 2) return launch_with(norm_forward_kernel<T, 32, 2, EDGE>, grid, 256, smem, s, a, stages);
        if (u <= 4) return launch_with(norm_forward_kernel<T, 32, 4, EDGE>, grid, 256, smem, s, a, stages);
        return launch_with(norm_forward_kernel<T, 32, 8, EDGE>, grid, 256, smem, s, a, stages);
    }
    if (a.period && units <= ROW_UNITS) {
        constexpr int U = 32 / V, CTAS = V == 8 ? 3 : 2;
        const int threads = (int)round_up((units + U - 1) / U, 32);
        const int per_sm = std::max(1, std::min(256 * CTAS / threads, (int)(SM_SHARED / (params + 2 * row))));
        const dim3 grid((unsigned)shared_out(a.rows, a.period, 1, sms * per_sm));
        const int stages = ring_stages(per_sm, params, row);
        if constexpr (V == 8)
            if (threads > 256) return launch_with(norm_forward_row_kernel<T, U, EDGE, 512, 1>, grid, threads, params + stages * row, s, a, stages);
        return launch_with(norm_forward_row_kernel<T, U, EDGE, 256, CTAS>, grid, threads, params + stages * row, s, a, stages);
    }
    const int threads = any_threads(a.cols);
    const dim3 grid((unsigned)std::min<int64_t>(a.rows, (int64_t)sms * (2048 / threads)));
    return launch_dependent(norm_forward_wide_kernel<T>, grid, dim3(threads), 0, s, 1, a);
}

// The backward row kernels' form for rows of that many units: rows at a time in a CTA, units per thread, threads and CTAs per SM (by their registers), and
// CTAs of a cluster: as many as fill the SMs of a GPC whatever its number of SMs.
struct BackwardForm { int rows, per_thread, threads, per_sm, cluster; };
BackwardForm backward_form(int64_t units)
{
    BackwardForm f;
    if (units <= 256) {
        f.rows = ROW_WARPS * (units <= 4 ? 8 : units <= 8 ? 4 : units <= 16 ? 2 : 1);
        f.per_thread = units <= 32 ? 1 : units <= 64 ? 2 : units <= 128 ? 4 : 8;
        f.threads = 32 * ROW_WARPS;
        f.per_sm = f.per_thread == 1 ? 3 : f.per_thread < 8 ? 2 : 1;
    } else {
        f.per_thread = units <= 768 ? 1 : units <= 1024 ? 2 : 4;
        f.rows = f.per_thread == 4 ? 1 : 2;
        f.threads = (int)round_up((units + f.per_thread - 1) / f.per_thread, 32);
        f.per_sm = units <= 384 ? 2 : 1;
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
    const size_t fixed = f.per_thread > 2 ? (size_t)units * V * 4 : 0, stage = (size_t)units * 32 * f.rows;
    const int stages = ring_stages(f.per_sm, fixed, stage);
    // (the sums of eight warps need two stages)
    const size_t smem = std::max(fixed + stages * stage, units <= 256 ? (size_t)units * V * (DB ? 64 : 32) : 0);
    const dim3 grid((unsigned)(ctas / cluster), 1, cluster);
    const auto launch = [&](auto kernel) { return launch_with(kernel, grid, f.threads, smem, s, a, stages, cluster); };
    if (units <= 4) return launch(norm_backward_lanes_kernel<T, 4, 1, DB, EDGE, 3>);
    if (units <= 8) return launch(norm_backward_lanes_kernel<T, 8, 1, DB, EDGE, 3>);
    if (units <= 16) return launch(norm_backward_lanes_kernel<T, 16, 1, DB, EDGE, 3>);
    if (units <= 32) return launch(norm_backward_lanes_kernel<T, 32, 1, DB, EDGE, 3>);
    if (units <= 64) return launch(norm_backward_lanes_kernel<T, 32, 2, DB, EDGE, 2>);
    if (units <= 128) return launch(norm_backward_lanes_kernel<T, 32, 4, DB, EDGE, 2>);
    if (units <= 256) return launch(norm_backward_lanes_kernel<T, 32, 8, DB, EDGE, 1>);
    if (units <= 384) return launch(norm_backward_kernel<T, 1, DB, EDGE, 384, 2>);
    if (units <= 768) return launch(norm_backward_kernel<T, 1, DB, EDGE, 768, 1>);
    if (units <= 1024) return launch(norm_backward_kernel<T, 2, DB, EDGE, 512, 1>);
    return launch(norm_backward_kernel<T, 4, DB, EDGE, 512, 1>);
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
