// Norm over rows, forward and backward (formulas in tsr.h).  Both passes are bound by HBM: forward reads x and writes y, backward reads
// x and dy and writes dx, each once; a row stays in registers between its sums and its results.
//
// Forward: a warp per row up to 2048 columns (FP32 1024; no barrier), a CTA per row up to 8192.  The mean is formed from the distances from the
// row's first entry and the variance from the distances from the mean, both from registers: a large mean costs no digits, and a row
// of equal entries has variance zero.
// Backward: a CTA walks over rows with fixed columns per thread, so that the sums for dweight and dbias stay in its registers; it leaves one
// partial row each, and column_finish adds them in order.  Narrow rows share the barrier of their reductions two by two.
// Wider rows, and matrices that do not start at the same place in 16 bytes, are read several times (from L2, mostly); their column sums take a
// pass of their own.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "tsr_layers.cuh"

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

struct NormArgs {
    const void *x, *dy, *weight, *bias;
    void *y;                        // y, or dx
    float *stats;
    const float *stats_in;
    float *partial;                 // [parts][cols] of dweight, then of dbias
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
// aligned vectors, weight and column sums belong to fixed registers or addresses, and only the first and the last unit of a row go entry by entry.

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

// EDGE: units may hang over an end of the row; the places that do read as `fill` and are not written.
template <typename T, bool EDGE>
__device__ __forceinline__ uint4 load_unit(const T *row, int col, int cols, T fill)
{
    constexpr int V = Unit<T>::V;
    if (!EDGE || (col >= 0 && col + V <= cols)) return *(const uint4 *)(row + col);
    T t[V];
#pragma unroll
    for (int i = 0; i < V; ++i) t[i] = col + i >= 0 && col + i < cols ? row[col + i] : fill;
    uint4 r;
    memcpy(&r, t, 16);
    return r;
}
__device__ __forceinline__ void unit_values(const uint4 &r, float (&v)[8]) { unpack8(r, v); }
__device__ __forceinline__ void unit_values(const uint4 &r, float (&v)[4])
{
    v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ uint4 unit_of(const float (&v)[8])
{
    return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}
__device__ __forceinline__ uint4 unit_of(const float (&v)[4])
{
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
template <typename T, bool EDGE>
__device__ __forceinline__ void store_unit(T *row, int col, int cols, const float (&v)[Unit<T>::V])
{
    constexpr int V = Unit<T>::V;
    if (!EDGE || (col >= 0 && col + V <= cols)) *(uint4 *)(row + col) = unit_of(v);
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) if (col + i >= 0 && col + i < cols) store_f(row + col + i, v[i]);
    }
}
__device__ __forceinline__ float param(const void *p, int c, bool is_bf16, float none) { return p ? load_as(p, c, is_bf16) : none; }

// Places of a unit that hang over an end of the row read as the row's first entry x0: their distance from it is zero and the mean right; from the
// mean m0 of the distances they are m0 away, which is taken out of the sum of squares again.  (That sum is m0^2 at least, by
// the first entry itself, so the difference keeps its digits.)
__device__ __forceinline__ float variance_of(float squares, float m0, const NormArgs &a, const int units, int V)
{
    return fmaxf(squares - (float)(units * V - a.cols) * m0 * m0, 0.f) * a.inv_n;
}

// A warp per row, eight rows of the class per CTA at a time, U units per lane; weight and bias in shared memory, by unit.
template <typename T, int U, bool EDGE>
__global__ void __launch_bounds__(256, 2)
norm_forward_kernel(const NormArgs a)
{
    constexpr int V = Unit<T>::V;
    __shared__ __align__(16) float w[U * 32 * V], b[U * 32 * V];
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const RowClass rc = row_class<T>(a.x, a.ldx, a.cols, a.period, blockIdx.x, gridDim.x);
    for (int i = threadIdx.x; i < rc.units * V; i += 256) {
        const int c = i - rc.shift;
        const bool in = c >= 0 && c < a.cols;
        w[i] = in ? param(a.weight, c, a.p_bf16, 1.f) : 0.f;
        b[i] = in ? param(a.bias, c, a.p_bf16, 0.f) : 0.f;
    }
    __syncthreads();
    for (int64_t r = rc.first + rc.step * warp; r < a.rows; r += rc.step * 8) {
        const T *x = (const T *)a.x + r * a.ldx;
        const T first = a.center ? *x : T(0.f);
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * 32 + lane;
            raw[u] = j < rc.units ? load_unit<T, EDGE>(x, j * V - rc.shift, a.cols, first) : make_uint4(0, 0, 0, 0);
        }
        const float x0 = load_f(&first);
        float v[U][V], m0 = 0.f, q = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float from = u * 32 + lane < rc.units ? x0 : 0.f;
            unit_values(raw[u], v[u]);
#pragma unroll
            for (int i = 0; i < V; ++i) { v[u][i] -= from; m0 += v[u][i]; }
        }
        m0 = a.center ? warp_sum(m0) * a.inv_n : 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float from = u * 32 + lane < rc.units ? m0 : 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) { v[u][i] -= from; q = fmaf(v[u][i], v[u][i], q); }
        }
        const float rstd = 1.f / sqrtf((EDGE ? variance_of(warp_sum(q), m0, a, rc.units, V) : warp_sum(q) * a.inv_n) + a.eps);
        if (a.stats && lane == 0) *(float2 *)(a.stats + 2 * r) = make_float2(x0 + m0, rstd);
        T *y = (T *)a.y + r * a.ldy;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * 32 + lane;
            if (j >= rc.units) continue;
            float o[V];
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                const float4 ww = *(const float4 *)(w + j * V + i), bb = *(const float4 *)(b + j * V + i);
                o[i] = fmaf(v[u][i] * rstd, ww.x, bb.x);
                o[i + 1] = fmaf(v[u][i + 1] * rstd, ww.y, bb.y);
                o[i + 2] = fmaf(v[u][i + 2] * rstd, ww.z, bb.z);
                o[i + 3] = fmaf(v[u][i + 3] * rstd, ww.w, bb.w);
            }
            store_unit<T, EDGE>(y, j * V - rc.shift, a.cols, o);
        }
    }
}

// A CTA per row, eight entries per thread; weight and bias in registers, the next row on its way while one is worked on.
template <typename T, bool EDGE>
__global__ void __launch_bounds__(1024, 1)
norm_forward_row_kernel(const NormArgs a)
{
    constexpr int V = Unit<T>::V, U = 8 / V;
    __shared__ float slots[2][32];
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x, threads = blockDim.x;
    const RowClass rc = row_class<T>(a.x, a.ldx, a.cols, a.period, blockIdx.x, gridDim.x);
    float w[U][V], b[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (u * threads + tid) * V - rc.shift + i;
            const bool in = c >= 0 && c < a.cols;
            w[u][i] = in ? param(a.weight, c, a.p_bf16, 1.f) : 0.f;
            b[u][i] = in ? param(a.bias, c, a.p_bf16, 0.f) : 0.f;
        }
    uint4 raw[U];
    T first = T(0.f);
    auto fetch = [&](int64_t r) {
        if (r >= a.rows) return;
        const T *x = (const T *)a.x + r * a.ldx;
        if (a.center) first = *x;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * threads + tid;
            raw[u] = j < rc.units ? load_unit<T, EDGE>(x, j * V - rc.shift, a.cols, first) : make_uint4(0, 0, 0, 0);
        }
    };
    fetch(rc.first);
    for (int64_t r = rc.first; r < a.rows; r += rc.step) {
        float v[U][V], m0 = 0.f, q = 0.f;
        const float x0 = load_f(&first);
#pragma unroll
        for (int u = 0; u < U; ++u) unit_values(raw[u], v[u]);
        fetch(r + rc.step);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float from = u * threads + tid < rc.units ? x0 : 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) { v[u][i] -= from; m0 += v[u][i]; }
        }
        if (a.center) m0 = cta_sum(m0, slots[0]) * a.inv_n;
        else m0 = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float from = u * threads + tid < rc.units ? m0 : 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) { v[u][i] -= from; q = fmaf(v[u][i], v[u][i], q); }
        }
        q = cta_sum(q, slots[1]);
        const float rstd = 1.f / sqrtf((EDGE ? variance_of(q, m0, a, rc.units, V) : q * a.inv_n) + a.eps);
        if (a.stats && tid == 0) *(float2 *)(a.stats + 2 * r) = make_float2(x0 + m0, rstd);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = u * threads + tid;
            if (j >= rc.units) continue;
#pragma unroll
            for (int i = 0; i < V; ++i) v[u][i] = fmaf(v[u][i] * rstd, w[u][i], b[u][i]);
            store_unit<T, EDGE>((T *)a.y + r * a.ldy, j * V - rc.shift, a.cols, v[u]);
        }
        if (!a.center) __syncthreads();     // (the slot of the only sum is free again)
    }
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
        const float rstd = 1.f / sqrtf(cta_sum(q, slots[1]) * a.inv_n + a.eps);
        if (a.stats && threadIdx.x == 0) { a.stats[2 * r] = mu; a.stats[2 * r + 1] = rstd; }
        T *y = (T *)a.y + r * a.ldy;
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x)
            store_f(y + c, fmaf((load_f(x + c) - x0 - m0) * rstd, param(a.weight, c, a.p_bf16, 1.f), param(a.bias, c, a.p_bf16, 0.f)));
        __syncthreads();
    }
}

// A CTA (up to 1024 threads) on R rows of its class at a time; U units per thread, whose columns stay the same, so that the column sums
// stay in registers.  The next R rows are on their way while these are worked on.  DB: the sums of dy are wanted too.
template <typename T, int U, int R, bool DB, bool EDGE, int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS)
norm_backward_kernel(const NormArgs a)
{
    constexpr int V = Unit<T>::V;
    __shared__ float2 slots[2][R][32];
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x, threads = blockDim.x, warp = tid >> 5, lane = tid & 31, warps = threads >> 5;
    const RowClass rc = row_class<T>(a.x, a.ldx, a.cols, a.period, blockIdx.x, gridDim.x);
    float w[U][V], dw[U][V], db[DB ? U : 1][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (u * threads + tid) * V - rc.shift + i;
            w[u][i] = c >= 0 && c < a.cols ? param(a.weight, c, a.p_bf16, 1.f) : 0.f;
            dw[u][i] = 0.f;
            if (DB) db[u][i] = 0.f;
        }
    uint4 nx[R][U], ng[R][U];
    float2 nst[R];
    auto fetch = [&](int64_t r0) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int64_t r = r0 + k * rc.step;
            const bool live = r < a.rows;       // a row that does not exist reads as dy = 0 with finite statistics: it adds nothing
            nst[k] = live ? *(const float2 *)(a.stats_in + 2 * r) : make_float2(0.f, 0.f);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = u * threads + tid;
                nx[k][u] = ng[k][u] = make_uint4(0, 0, 0, 0);
                if (live && j < rc.units) {
                    nx[k][u] = load_unit<T, EDGE>((const T *)a.x + r * a.ldx, j * V - rc.shift, a.cols, T(0.f));
                    ng[k][u] = load_unit<T, EDGE>((const T *)a.dy + r * a.lddy, j * V - rc.shift, a.cols, T(0.f));
                }
            }
        }
    };
    fetch(rc.first);
    int turn = 0;
    for (int64_t r0 = rc.first; r0 < a.rows; r0 += R * rc.step, turn ^= 1) {
        float x[R][U][V], g[R][U][V];
        float2 s[R], st[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            st[k] = nst[k];
#pragma unroll
            for (int u = 0; u < U; ++u) { unit_values(nx[k][u], x[k][u]); unit_values(ng[k][u], g[k][u]); }
        }
        fetch(r0 + R * rc.step);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            s[k] = make_float2(0.f, 0.f);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float h = (x[k][u][i] - st[k].x) * st[k].y;
                    x[k][u][i] = h;
                    dw[u][i] = fmaf(g[k][u][i], h, dw[u][i]);
                    if (DB) db[u][i] += g[k][u][i];
                    g[k][u][i] *= w[u][i];
                    s[k].x += g[k][u][i];
                    s[k].y = fmaf(g[k][u][i], h, s[k].y);
                }
            s[k].x = warp_sum(s[k].x);
            s[k].y = warp_sum(s[k].y);
        }
        if (warps > 1) {
            if (lane == 0) {
#pragma unroll
                for (int k = 0; k < R; ++k) slots[turn][k][warp] = s[k];
            }
            __syncthreads();      // one per turn: the slots of the turn before last are written again only after the last one's barrier
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const float2 t = lane < warps ? slots[turn][k][lane] : make_float2(0.f, 0.f);
                s[k].x = warp_sum(t.x);
                s[k].y = warp_sum(t.y);
            }
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int64_t r = r0 + k * rc.step;
            if (!a.y || r >= a.rows) continue;
            const float c1 = a.center ? s[k].x * a.inv_n : 0.f, c2 = s[k].y * a.inv_n;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = u * threads + tid;
                if (j >= rc.units) continue;
#pragma unroll
                for (int i = 0; i < V; ++i) g[k][u][i] = st[k].y * (g[k][u][i] - fmaf(x[k][u][i], c2, c1));
                store_unit<T, EDGE>((T *)a.y + r * a.ldy, j * V - rc.shift, a.cols, g[k][u]);
            }
        }
    }
    // column sums of this CTA
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (u * threads + tid) * V - rc.shift + i;
            if (c < 0 || c >= a.cols) continue;
            if (a.want_dw) a.partial[(int64_t)blockIdx.x * a.cols + c] = dw[u][i];
            if (DB) a.partial[((int64_t)(a.want_dw ? gridDim.x : 0) + blockIdx.x) * a.cols + c] = db[u][i];
        }
}

// Any width and alignment: dx alone, two passes over the row, ...
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

template <typename T, bool EDGE>
cudaError_t forward_as(const NormArgs &a, int units, int sms, cudaStream_t s)
{
    constexpr int V = Unit<T>::V;
    if (a.period && units * V <= 2048) {
        const int u = (units + 31) / 32;
        const dim3 grid((unsigned)shared_out(a.rows, a.period, 8, sms * 4));
        if (u <= 1) return launch_dependent(norm_forward_kernel<T, 1, EDGE>, grid, dim3(256), 0, s, 1, a);
        if (u <= 2) return launch_dependent(norm_forward_kernel<T, 2, EDGE>, grid, dim3(256), 0, s, 1, a);
        if (u <= 4) return launch_dependent(norm_forward_kernel<T, 4, EDGE>, grid, dim3(256), 0, s, 1, a);
        if (V == 8 || u <= 8) return launch_dependent(norm_forward_kernel<T, 8, EDGE>, grid, dim3(256), 0, s, 1, a);
    }
    if (a.period && units * V <= ROW_COLS) {
        const int threads = (int)round_up((units * V + 7) / 8, 32);
        return launch_dependent(norm_forward_row_kernel<T, EDGE>, dim3((unsigned)shared_out(a.rows, a.period, 1, sms * std::max(1, 1024 / threads))), dim3(threads), 0, s, 1, a);
    }
    const int threads = any_threads(a.cols);
    const dim3 grid((unsigned)std::min<int64_t>(a.rows, (int64_t)sms * (2048 / threads)));
    return launch_dependent(norm_forward_wide_kernel<T>, grid, dim3(threads), 0, s, 1, a);
}

// The backward row kernel's form for a row of that many entries (whole units): entries per thread, threads, CTAs per SM.
struct BackwardForm { int entries, threads, per_sm; };
BackwardForm backward_form(int64_t entries_in_units)
{
    BackwardForm f;
    f.entries = entries_in_units <= 4096 ? 8 : 16;
    f.threads = (int)std::max<int64_t>(32, round_up((entries_in_units + f.entries - 1) / f.entries, 32));
    f.per_sm = f.threads <= 256 ? std::min(16, 768 / f.threads) : f.threads <= 384 ? 2 : 1;
    return f;
}
// Partial rows of column sums that a backward pass leaves.
int backward_parts(int64_t rows, int64_t entries_in_units, int period, int sms)
{
    if (entries_in_units > ROW_COLS || period == 0) return (int)std::max<int64_t>(1, std::min<int64_t>((rows + 31) / 32, 2 * sms));
    return (int)shared_out(rows, period, 2, (int64_t)sms * backward_form(entries_in_units).per_sm);
}
// ... and the most for any alignment of the matrices.
int most_parts(const tsr_norm_desc &d, int sms)
{
    const int V = 16 / type_bytes(d.dtype);
    int most = backward_parts(d.rows, 0, 0, sms);
    for (int period = 1; period <= V; period *= 2)
        for (int shift = 0; shift < V; ++shift) most = std::max(most, backward_parts(d.rows, round_up(d.cols + shift, V), period, sms));
    return most;
}

template <typename T, bool DB, bool EDGE>
cudaError_t backward_as(const NormArgs &a, int units, int parts, cudaStream_t s)
{
    constexpr int V = Unit<T>::V, U8 = 8 / V, U16 = 16 / V;
    const BackwardForm f = backward_form((int64_t)units * V);
    const dim3 grid(parts), block(f.threads);
    if (f.entries == 16) {
        if (f.threads <= 384) return launch_dependent(norm_backward_kernel<T, U16, 1, DB, EDGE, 384, DB ? 1 : 2>, grid, block, 0, s, 1, a);
        return launch_dependent(norm_backward_kernel<T, U16, 1, DB, EDGE, 512, 1>, grid, block, 0, s, 1, a);
    }
    if (f.threads <= 256) return launch_dependent(norm_backward_kernel<T, U8, 2, DB, EDGE, 256, V == 8 ? 3 : 2>, grid, block, 0, s, 1, a);
    return launch_dependent(norm_backward_kernel<T, U8, 1, DB, EDGE, 512, V == 8 ? 2 : 1>, grid, block, 0, s, 1, a);
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
    if (a.y) {
        const int threads = any_threads(a.cols);
        const cudaError_t e = launch_dependent(norm_backward_wide_kernel<T>, dim3((unsigned)std::min<int64_t>(a.rows, (int64_t)sms * (2048 / threads))), dim3(threads), 0, s, 1, a);
        if (e != cudaSuccess) return e;
    }
    if (!a.want_dw && !a.want_db) return cudaSuccess;
    return launch_dependent(norm_columns_kernel<T>, dim3((unsigned)((a.cols + 255) / 256), (unsigned)parts), dim3(256), 0, s, 1, a, (a.rows + parts - 1) / parts);
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
    if (!aligned_to(weight, type_bytes(d.p_dtype)) || !aligned_to(bias, type_bytes(d.p_dtype)) || !aligned_to(stats, 4)) return TSR_ERR_ALIGNMENT;
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
    if (!aligned_to(weight, type_bytes(d.p_dtype)) || !aligned_to(dweight, type_bytes(d.g_dtype)) || !aligned_to(dbias, type_bytes(d.g_dtype)) || !aligned_to(stats, 4))
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
    const int64_t entries = (int64_t)units * (16 / type_bytes(d.dtype));
    const int parts = backward_parts(d.rows, entries, a.period, sms);
    if (d.rows > 0) {
        const bool bf = d.dtype == TSR_BF16;
        cudaError_t e;
        if (a.period == 0 || entries > ROW_COLS) e = bf ? backward_wide<bf16>(a, parts, sms, s) : backward_wide<float>(a, parts, sms, s);
        else e = bf ? backward_of<bf16>(a, units, parts, s) : backward_of<float>(a, units, parts, s);
        if (e != cudaSuccess) return TSR_ERR_CUDA;
    }
    const bool gb = d.g_dtype == TSR_BF16;
    void *one = dweight ? dweight : dbias, *two = dweight ? dbias : nullptr;
    if (one && column_finish((const float *)workspace, d.rows ? parts : 0, d.cols, d.cols, one, gb, two, gb, d.accumulate != 0, s) != cudaSuccess) return TSR_ERR_CUDA;
    return TSR_OK;
}
