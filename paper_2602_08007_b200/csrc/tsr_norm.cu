// Norm over rows, forward and backward (formulas in tsr.h).  Both passes are bound by HBM: forward reads x and writes y, backward reads
// x and dy and writes dx, each once; a row stays in registers between its sums and its results.
//
// Forward and backward: rows up to 8192 columns are worked on by a warp or a CTA, the next ones in flight.  Distances are formed from the
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

struct NormArgs {
    const void *x, *dy, *weight, *bias;
    void *y;                        // y, or dx
    float *stats;
    const float *stats_in;
    float *partial;                 // [parts][cols] of dweight, then of dbias; NULL: one CTA, the sums go to dw and db
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

// Unit j of a row in shared memory; EDGE: the places that hold no entry are zero.
template <typename T, bool EDGE>
__device__ __forceinline__ uint4 take_unit(const uint4 *row, int j, int col, int cols)
{
    constexpr int V = Unit<T>::V;
    uint4 r = row[j];
    if (EDGE && (col < 0 || col + V > cols)) {
        T t[V];
        memcpy(t, &r, 16);
#pragma unroll
        for (int i = 0; i < V; ++i) if (col + i < 0 || col + i >= cols) t[i] = T(0.f);
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
    if (!EDGE || (col >= 0 && col + V <= cols)) *(uint4 *)(row + col) = unit_of(v);
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) if (col + i >= 0 && col + i < cols) store_f(row + col + i, i & 1 ? v[i / 2].y : v[i / 2].x);
    }
}
__device__ __forceinline__ float param(const void *p, int c, bool is_bf16, float none) { return p ? load_as(p, c, is_bf16) : none; }

// The entries of a unit less `from`; places that hold no entry become zero.  Without EDGE only whole units are missing.
template <bool EDGE, int P>
__device__ __forceinline__ void less(float2 (&v)[P], float from, int col, int cols)
{
    if (EDGE ? col >= 0 && col + 2 * P <= cols : col < cols) {
#pragma unroll
        for (int i = 0; i < P; ++i) v[i] = add2(v[i], pair(-from));
    } else {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            v[i].x = EDGE && col + 2 * i >= 0 && col + 2 * i < cols ? v[i].x - from : 0.f;
            v[i].y = EDGE && col + 2 * i + 1 >= 0 && col + 2 * i + 1 < cols ? v[i].y - from : 0.f;
        }
    }
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
// v <- (v - mean) rstd w + b over unit j
template <int P>
__device__ __forceinline__ void normed(float2 (&v)[P], float mean, float rstd, const float *w, const float *b, int j, int units)
{
#pragma unroll
    for (int i = 0; i < P; i += 2) {
        const float4 ww = *(const float4 *)(w + shared_at(j, i / 2, units)), bb = *(const float4 *)(b + shared_at(j, i / 2, units));
        v[i] = fma2(mul2(add2(v[i], pair(-mean)), pair(rstd)), make_float2(ww.x, ww.y), make_float2(bb.x, bb.y));
        v[i + 1] = fma2(mul2(add2(v[i + 1], pair(-mean)), pair(rstd)), make_float2(ww.z, ww.w), make_float2(bb.z, bb.w));
    }
}

// A warp per row, U units per lane, a ring of `stages` rows per warp.
template <typename T, int U, bool EDGE>
__global__ void __launch_bounds__(256, U > 4 ? 2 : U > 2 ? 3 : 4)
norm_forward_kernel(const NormArgs a, int stages)
{
    constexpr int V = Unit<T>::V, P = V / 2;
    extern __shared__ float4 shared[];       // w, b, rings
    __shared__ uint64_t bars[8 * NORM_STAGES];
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const RowClass rc = row_class<T>(a.x, a.ldx, a.cols, a.period, blockIdx.x, gridDim.x);
    float *w = (float *)shared, *b = w + rc.units * V;
    const uint4 *ring = (const uint4 *)(b + rc.units * V) + warp * stages * rc.units;
    uint64_t *bar = bars + warp * NORM_STAGES;
    const int64_t step = rc.step * 8, start = rc.first + rc.step * warp;
    int64_t left = start < a.rows ? (a.rows - start + step - 1) / step : 0;     // rows of this warp
    const T *ask = (const T *)a.x + start * a.ldx;
    auto request = [&](int stage) {      // the next row, by lane 0
        mbar_expect_tx(smem_u32(bar + stage), (uint32_t)rc.units * 16u);
        ask_row<T>(smem_u32(ring + stage * rc.units), ask, rc, smem_u32(bar + stage));
        ask += step * a.ldx;
    };
    if (lane == 0) {
        for (int i = 0; i < stages; ++i) mbar_init(smem_u32(bar + i), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int i = 0; i < stages && i < left; ++i) request(i);
    }
    share_params<T>(a, rc, w, b);
    __syncthreads();
    bool gave_up = false;
    int stage = 0;
    uint32_t phase = 0;
    T *y = (T *)a.y + start * a.ldy;
    float *stats = a.stats ? a.stats + 2 * start : nullptr;
    for (; left > 0; --left) {
        await_row(smem_u32(bar + stage), phase, gave_up);
        const uint4 *row = ring + stage * rc.units;
        const float x0 = a.center ? load_f((const T *)row + rc.shift) : 0.f;
        float2 v[U][P], sum = pair(0.f), q = pair(0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * 32 + lane, col = j * V - rc.shift;
            unit_pairs(j < rc.units ? take_unit<T, EDGE>(row, j, col, a.cols) : make_uint4(0, 0, 0, 0), v[u]);
        }
        __syncwarp();
        if (lane == 0 && left > stages) request(stage);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            less<EDGE>(v[u], x0, (u * 32 + lane) * V - rc.shift, a.cols);
#pragma unroll
            for (int i = 0; i < P; ++i) sum = add2(sum, v[u][i]);
        }
        const float mean = a.center ? warp_sum(sum.x + sum.y) * a.inv_n : 0.f;
        // squared distances from the mean; what holds no entry is left out
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = (u * 32 + lane) * V - rc.shift;
            if (EDGE ? col >= 0 && col + V <= a.cols : col < a.cols) {
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float2 d = add2(v[u][i], pair(-mean));
                    q = fma2(d, d, q);
                }
            } else if (EDGE) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = (i & 1 ? v[u][i / 2].y : v[u][i / 2].x) - mean;
                    if (col + i >= 0 && col + i < a.cols) q.x = fmaf(d, d, q.x);
                }
            }
        }
        const float rstd = rsqrtf(warp_sum(q.x + q.y) * a.inv_n + a.eps);
        if (stats && lane == 0) *(float2 *)stats = make_float2(x0 + mean, rstd);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * 32 + lane;
            if (j >= rc.units) continue;
            normed(v[u], mean, rstd, w, b, j, rc.units);
            store_unit<T, EDGE>(y, j * V - rc.shift, a.cols, v[u]);
        }
        y += step * a.ldy;
        if (stats) stats += 2 * step;
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
    int own = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int col = (u * threads + tid) * V - rc.shift;
        own += max(0, min(col + V, a.cols) - max(col, 0));
    }
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
        const float x0 = a.center ? load_f((const T *)row + rc.shift) : 0.f;
        float2 v[U][P], sum = pair(0.f), q = pair(0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * threads + tid, col = j * V - rc.shift;
            unit_pairs(j < rc.units ? take_unit<T, EDGE>(row, j, col, a.cols) : make_uint4(0, 0, 0, 0), v[u]);
            less<EDGE>(v[u], x0, col, a.cols);
#pragma unroll
            for (int i = 0; i < P; ++i) sum = add2(sum, v[u][i]);
        }
        const float mine = a.center ? (sum.x + sum.y) * inv_own : 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            less<EDGE>(v[u], mine, (u * threads + tid) * V - rc.shift, a.cols);
#pragma unroll
            for (int i = 0; i < P; ++i) q = fma2(v[u][i], v[u][i], q);
        }
        float mean = mine, squares = q.x + q.y;
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
            normed(v[u], mean - mine, rstd, w, b, j, rc.units);
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

// A CTA walks over rows of its class; U units per thread, whose columns stay the same, so that the column sums stay in registers.  x and dy come
// through a ring of `stages` rows; weight is in shared memory, by unit.  DB: the sums of dy are wanted too.
template <typename T, int U, bool DB, bool EDGE, int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS)
norm_backward_kernel(const NormArgs a, int stages)
{
    constexpr int V = Unit<T>::V, P = V / 2;
    extern __shared__ float4 shared[];       // weight, ring
    __shared__ uint64_t bars[NORM_STAGES];
    __shared__ float4 slots[2][16];          // the warps' pairs of sums, two in a vector
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x, threads = blockDim.x, warp = tid >> 5, lane = tid & 31, warps = threads >> 5;
    const RowClass rc = row_class<T>(a.x, a.ldx, a.cols, a.period, blockIdx.x, gridDim.x);
    float *weight = (float *)shared;
    const uint4 *ring = (const uint4 *)(weight + rc.units * V);      // per stage x, then dy
    int64_t left = rc.first < a.rows ? (a.rows - rc.first + rc.step - 1) / rc.step : 0;
    const T *ask_x = (const T *)a.x + rc.first * a.ldx, *ask_dy = (const T *)a.dy + rc.first * a.lddy;
    auto request = [&](int stage) {      // the next row, by one thread
        const uint32_t bar = smem_u32(bars + stage), at = smem_u32(ring + stage * 2 * rc.units);
        mbar_expect_tx(bar, (uint32_t)rc.units * 32u);
        ask_row<T>(at, ask_x, rc, bar);
        ask_row<T>(at + (uint32_t)rc.units * 16u, ask_dy, rc, bar);
        ask_x += rc.step * a.ldx;
        ask_dy += rc.step * a.lddy;
    };
    if (tid == 0) {
        for (int i = 0; i < stages; ++i) mbar_init(smem_u32(bars + i), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int i = 0; i < stages && i < left; ++i) request(i);
    }
    share_params<T>(a, rc, weight, nullptr);
    for (int i = tid; i < 2 * 16; i += threads) ((float4 *)slots)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    float2 dw[U][P], db[DB ? U : 1][P];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < P; ++i) {
            dw[u][i] = pair(0.f);
            if (DB) db[u][i] = pair(0.f);
        }
    auto weights = [&](int u, float2 (&w)[P]) {
        const int j = min(u * threads + tid, rc.units - 1);      // (a thread without a unit has dy = 0)
#pragma unroll
        for (int i = 0; i < P; i += 2) {
            const float4 t = *(const float4 *)(weight + shared_at(j, i / 2, rc.units));
            w[i] = make_float2(t.x, t.y);
            w[i + 1] = make_float2(t.z, t.w);
        }
    };
    __syncthreads();
    bool gave_up = false;
    int turn = 0, stage = 0;
    uint32_t phase = 0;
    T *y = (T *)a.y + rc.first * a.ldy;
    const float2 *stats = (const float2 *)a.stats_in + rc.first;
    float2 next = left > 0 ? *stats : pair(0.f);
    for (; left > 0; --left, turn ^= 1) {
        const float2 st = next;
        stats += rc.step;
        if (left > 1) next = *stats;
        await_row(smem_u32(bars + stage), phase, gave_up);
        const uint4 *row = ring + stage * 2 * rc.units;
        uint4 x[U], g[U];
        float2 s1 = pair(0.f), s2 = pair(0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * threads + tid, col = j * V - rc.shift;
            x[u] = g[u] = make_uint4(0, 0, 0, 0);
            if (j < rc.units) {
                x[u] = take_unit<T, EDGE>(row, j, col, a.cols);
                g[u] = take_unit<T, EDGE>(row + rc.units, j, col, a.cols);
            }
            float2 w[P], xv[P], gv[P];
            weights(u, w);
            unit_pairs(x[u], xv);
            unit_pairs(g[u], gv);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float2 h = mul2(add2(xv[i], pair(-st.x)), pair(st.y));
                dw[u][i] = fma2(gv[i], h, dw[u][i]);
                if (DB) db[u][i] = add2(db[u][i], gv[i]);
                const float2 gw = mul2(gv[i], w[i]);
                s1 = add2(s1, gw);
                s2 = fma2(gw, h, s2);
            }
        }
        float2 s = make_float2(s1.x + s1.y, s2.x + s2.y);
#pragma unroll
        for (int o = 16; o; o >>= 1) s = add2(s, make_float2(__shfl_xor_sync(0xffffffffu, s.x, o), __shfl_xor_sync(0xffffffffu, s.y, o)));
        // One barrier per turn: the slots of the turn before last are written again only after the last one's, and the rows have left their stage.
        if (warps > 1) {
            if (lane == 0) ((float2 *)slots[turn])[warp] = s;
            __syncthreads();
            s = pair(0.f);
            for (int i = 0; i < (warps + 1) / 2; ++i) {
                const float4 t = slots[turn][i];
                s = add2(s, add2(make_float2(t.x, t.y), make_float2(t.z, t.w)));
            }
        } else __syncwarp();
        if (tid == 0 && left > stages) request(stage);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
        if (a.y) {
            // dx = r g w - r mean(g w) - (x - mu) r^2 mean(g w h)
            const float2 c1 = pair(a.center ? -s.x * a.inv_n * st.y : 0.f), c2 = pair(-s.y * a.inv_n * st.y * st.y);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = u * threads + tid;
                if (j >= rc.units) continue;
                float2 w[P], xv[P], gv[P];
                weights(u, w);
                unit_pairs(x[u], xv);
                unit_pairs(g[u], gv);
#pragma unroll
                for (int i = 0; i < P; ++i) gv[i] = fma2(mul2(gv[i], w[i]), pair(st.y), fma2(add2(xv[i], pair(-st.x)), c2, c1));
                store_unit<T, EDGE>(y, j * V - rc.shift, a.cols, gv);
            }
            y += rc.step * a.ldy;
        }
    }
    note_gave_up(gave_up);
    // column sums of this CTA
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (u * threads + tid) * V - rc.shift + i;
            if (c < 0 || c >= a.cols) continue;
            const float w = i & 1 ? dw[u][i / 2].y : dw[u][i / 2].x, b = !DB ? 0.f : i & 1 ? db[DB ? u : 0][i / 2].y : db[DB ? u : 0][i / 2].x;
            if (a.partial) {
                if (a.want_dw) a.partial[(int64_t)blockIdx.x * a.cols + c] = w;
                if (DB) a.partial[((int64_t)(a.want_dw ? gridDim.x : 0) + blockIdx.x) * a.cols + c] = b;
            } else {
                if (a.want_dw) store_as(a.dw, c, a.g_bf16, a.accumulate ? w + load_as(a.dw, c, a.g_bf16) : w);
                if (DB) store_as(a.db, c, a.g_bf16, a.accumulate ? b + load_as(a.db, c, a.g_bf16) : b);
            }
        }
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

constexpr int64_t ROW_COLS = 8192;          // widest row that the row kernels hold, in whole units

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
cudaError_t launch_with(Kern kernel, dim3 grid, int threads, size_t smem, cudaStream_t s, const NormArgs &a, int stages)
{
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    return launch_dependent(kernel, grid, dim3(threads), smem, s, 1, a, stages);
}

template <typename T, bool EDGE>
cudaError_t forward_as(const NormArgs &a, int units, int sms, cudaStream_t s)
{
    constexpr int V = Unit<T>::V;
    const size_t params = (size_t)units * V * 8, row = (size_t)units * 16;
    if (a.period && units <= 256) {
        const int u = (units + 31) / 32, per_sm = u > 4 ? 2 : u > 2 ? 3 : 4;      // as many as are resident
        const dim3 grid((unsigned)shared_out(a.rows, a.period, 8, sms * per_sm));
        const int stages = ring_stages(per_sm, params, 8 * row);
        const size_t smem = params + 8 * stages * row;
        if (u <= 1) return launch_with(norm_forward_kernel<T, 1, EDGE>, grid, 256, smem, s, a, stages);
        if (u <= 2) return launch_with(norm_forward_kernel<T, 2, EDGE>, grid, 256, smem, s, a, stages);
        if (u <= 4) return launch_with(norm_forward_kernel<T, 4, EDGE>, grid, 256, smem, s, a, stages);
        return launch_with(norm_forward_kernel<T, 8, EDGE>, grid, 256, smem, s, a, stages);
    }
    if (a.period && units * V <= ROW_COLS) {
        constexpr int U = 32 / V, CTAS = V == 8 ? 3 : 2;
        const int threads = (int)round_up((units + U - 1) / U, 32);
        const int per_sm = std::max(1, std::min(256 * CTAS / threads, (int)(SM_SHARED / (params + 2 * row))));
        const dim3 grid((unsigned)shared_out(a.rows, a.period, 1, sms * per_sm));
        const int stages = ring_stages(per_sm, params, row);
        return launch_with(norm_forward_row_kernel<T, U, EDGE, 256, CTAS>, grid, threads, params + stages * row, s, a, stages);
    }
    const int threads = any_threads(a.cols);
    const dim3 grid((unsigned)std::min<int64_t>(a.rows, (int64_t)sms * (2048 / threads)));
    return launch_dependent(norm_forward_wide_kernel<T>, grid, dim3(threads), 0, s, 1, a);
}

// The backward row kernel's form for a row of that many units: units per thread, threads, CTAs per SM.
struct BackwardForm { int per_thread, threads, per_sm; };
BackwardForm backward_form(int64_t units, int V)
{
    BackwardForm f;
    f.per_thread = units <= 32 ? 1 : units <= 1024 ? 2 : 4;
    f.threads = (int)std::max<int64_t>(32, round_up((units + f.per_thread - 1) / f.per_thread, 32));
    f.per_sm = f.per_thread == 4 ? 1 : std::min(24, (f.threads > 128 ? 768 : V == 8 ? 640 : 896) / f.threads);      // by their registers
    const int64_t least = units * (V * 4 + 2 * 32);      // weight and two stages
    if (least > 0) f.per_sm = (int)std::min<int64_t>(f.per_sm, SM_SHARED / least);
    f.per_sm = std::max(1, f.per_sm);
    return f;
}
// Partial rows of column sums that a backward pass leaves.
int backward_parts(int64_t rows, int64_t units, int V, int period, int sms)
{
    if (units * V > ROW_COLS || period == 0) return (int)std::max<int64_t>(1, std::min<int64_t>((rows + 31) / 32, 2 * sms));
    return (int)shared_out(rows, period, 2, (int64_t)sms * backward_form(units, V).per_sm);
}
// ... and the most for any alignment of the matrices.
int most_parts(const tsr_norm_desc &d, int sms)
{
    const int V = 16 / type_bytes(d.dtype);
    int most = backward_parts(d.rows, 0, V, 0, sms);
    for (int period = 1; period <= V; period *= 2)
        for (int shift = 0; shift < V; ++shift) most = std::max(most, backward_parts(d.rows, (d.cols + shift + V - 1) / V, V, period, sms));
    return most;
}

template <typename T, bool DB, bool EDGE>
cudaError_t backward_as(const NormArgs &a, int units, int parts, cudaStream_t s)
{
    constexpr int V = Unit<T>::V;
    const BackwardForm f = backward_form(units, V);
    const size_t fixed = (size_t)units * V * 4, stage = (size_t)units * 32;
    const int stages = ring_stages(f.per_sm, fixed, stage);
    const size_t smem = fixed + stages * stage;
    if (f.per_thread == 1) return launch_with(norm_backward_kernel<T, 1, DB, EDGE, 32, 24>, dim3(parts), f.threads, smem, s, a, stages);
    if (f.per_thread == 4) return launch_with(norm_backward_kernel<T, 4, DB, EDGE, 512, 1>, dim3(parts), f.threads, smem, s, a, stages);
    if (f.threads <= 128) return launch_with(norm_backward_kernel<T, 2, DB, EDGE, 128, V == 8 ? 5 : 7>, dim3(parts), f.threads, smem, s, a, stages);
    if (f.threads <= 384) return launch_with(norm_backward_kernel<T, 2, DB, EDGE, 384, 2>, dim3(parts), f.threads, smem, s, a, stages);
    return launch_with(norm_backward_kernel<T, 2, DB, EDGE, 512, 1>, dim3(parts), f.threads, smem, s, a, stages);
}

template <typename T>
cudaError_t forward_of(const NormArgs &a, int units, int sms, cudaStream_t s)
{
    return has_edges(a, Unit<T>::V) ? forward_as<T, true>(a, units, sms, s) : forward_as<T, false>(a, units, sms, s);
}
template <typename T>
cudaError_t backward_of(const NormArgs &a, int units, int parts, cudaStream_t s)
{
    if (has_edges(a, Unit<T>::V)) return a.want_db ? backward_as<T, true, true>(a, units, parts, s) : backward_as<T, false, true>(a, units, parts, s);
    return a.want_db ? backward_as<T, true, false>(a, units, parts, s) : backward_as<T, false, false>(a, units, parts, s);
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
    const int V = 16 / type_bytes(d.dtype);
    const int parts = backward_parts(d.rows, units, V, a.period, sms);
    bool direct = false;      // a single CTA of the row kernel: its sums are the result
    if (d.rows > 0) {
        const bool bf = d.dtype == TSR_BF16;
        direct = parts == 1 && a.period && units * V <= ROW_COLS;
        if (direct) a.partial = nullptr;
        a.dw = dweight; a.db = dbias; a.g_bf16 = d.g_dtype == TSR_BF16; a.accumulate = d.accumulate;
        cudaError_t e;
        if (a.period == 0 || units * V > ROW_COLS) e = bf ? backward_wide<bf16>(a, parts, sms, s) : backward_wide<float>(a, parts, sms, s);
        else e = bf ? backward_of<bf16>(a, units, parts, s) : backward_of<float>(a, units, parts, s);
        if (e != cudaSuccess) return TSR_ERR_CUDA;
    }
    const bool gb = d.g_dtype == TSR_BF16;
    void *one = dweight ? dweight : dbias, *two = dweight ? dbias : nullptr;
    if (one && !direct && column_finish((const float *)workspace, d.rows ? parts : 0, d.cols, d.cols, one, gb, two, gb, d.accumulate != 0, s) != cudaSuccess) return TSR_ERR_CUDA;
    return TSR_OK;
}
