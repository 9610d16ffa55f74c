// Norm over rows, forward and backward (formulas in tsr.h).  Both passes are bound by HBM: forward reads x and writes y, backward reads
// x and dy and writes dx, each once; a row stays in registers between its sums and its results.
//
// Forward: a warp per row up to 2048 columns (no barrier), a CTA per row up to 16384.  The mean is formed from the distances from the
// row's first entry and the variance from the distances from the mean, both from registers: a large mean costs no digits, and a row
// of equal entries has variance zero.
// Backward: a CTA walks over rows with eight columns per thread, so that the sums for dweight and dbias stay in its registers; it leaves one
// partial row each, and column_finish adds them in order.  Two rows at a time share the barrier of their reductions.
// Wider rows are read several times (from L2, mostly); their column sums take a pass of their own.
// Rows off the 16-byte grid are read entry by entry, lanes side by side; the layout is the same otherwise.
#include <math.h>

#include <algorithm>

#include "tsr_layers.cuh"

namespace tsr {

__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// Sum over the CTA; `slot` (32 floats) must not be in use by an earlier sum that a thread may still read.
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
    float eps, inv_n;
};

// The k-th entry of a thread: vectors of eight side by side (VEC), or single entries `threads` apart.
template <bool VEC>
__device__ __forceinline__ int column_of(int k, int tid, int threads) { return VEC ? ((k >> 3) * threads + tid) * 8 + (k & 7) : k * threads + tid; }

template <typename T, bool VEC, int NE>
__device__ __forceinline__ void load_row(const T *row, int tid, int threads, int cols, float (&v)[NE])
{
    if (VEC) {
#pragma unroll
        for (int i = 0; i < NE / 8; ++i) {
            float t[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            const int c = (i * threads + tid) * 8;
            if (c < cols) load8(row + c, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[8 * i + j] = t[j];
        }
    } else {
#pragma unroll
        for (int k = 0; k < NE; ++k) v[k] = k * threads + tid < cols ? load_f(row + k * threads + tid) : 0.f;
    }
}
template <typename T, bool VEC, int NE>
__device__ __forceinline__ void store_row(T *row, int tid, int threads, int cols, const float (&v)[NE])
{
    if (VEC) {
#pragma unroll
        for (int i = 0; i < NE / 8; ++i) {
            const int c = (i * threads + tid) * 8;
            if (c < cols) {
                float t[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] = v[8 * i + j];
                store8(row + c, t);
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < NE; ++k) if (k * threads + tid < cols) store_f(row + k * threads + tid, v[k]);
    }
}
__device__ __forceinline__ float param(const void *p, int c, bool is_bf16, float none) { return p ? load_as(p, c, is_bf16) : none; }

// CTA false: a warp per row; true: a CTA per row.
template <typename T, bool VEC, int NE, bool CTA>
__global__ void __launch_bounds__(CTA ? 1024 : 256)
norm_forward_kernel(const NormArgs a)
{
    __shared__ float slots[CTA ? 2 : 1][32];
    pdl_trigger();
    pdl_wait();
    const int tid = CTA ? threadIdx.x : (threadIdx.x & 31), threads = CTA ? blockDim.x : 32;
    const int64_t per = CTA ? 1 : blockDim.x >> 5, first = CTA ? 0 : threadIdx.x >> 5;
    for (int64_t r = blockIdx.x * per + first; r < a.rows; r += gridDim.x * per) {
        float v[NE];
        load_row<T, VEC, NE>((const T *)a.x + r * a.ldx, tid, threads, a.cols, v);
        float x0 = 0.f, m0 = 0.f;
        if (a.center) {
            x0 = load_f((const T *)a.x + r * a.ldx);
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < NE; ++k) {
                v[k] = column_of<VEC>(k, tid, threads) < a.cols ? v[k] - x0 : 0.f;
                s += v[k];
            }
            m0 = (CTA ? cta_sum(s, slots[0]) : warp_sum(s)) * a.inv_n;
        }
        const float mu = x0 + m0;
        float q = 0.f;
#pragma unroll
        for (int k = 0; k < NE; ++k) {
            v[k] = column_of<VEC>(k, tid, threads) < a.cols ? v[k] - m0 : 0.f;
            q = fmaf(v[k], v[k], q);
        }
        q = (CTA ? cta_sum(q, slots[CTA ? 1 : 0]) : warp_sum(q)) * a.inv_n;
        const float rstd = 1.f / sqrtf(q + a.eps);
        if (a.stats && tid == 0) { a.stats[2 * r] = mu; a.stats[2 * r + 1] = rstd; }
#pragma unroll
        for (int k = 0; k < NE; ++k) {
            const int c = column_of<VEC>(k, tid, threads);
            if (c < a.cols) v[k] = fmaf(v[k] * rstd, param(a.weight, c, a.p_bf16, 1.f), param(a.bias, c, a.p_bf16, 0.f));
        }
        store_row<T, VEC, NE>((T *)a.y + r * a.ldy, tid, threads, a.cols, v);
        if (CTA && !a.center) __syncthreads();     // the slot of the only sum is free again
    }
}

// Any width: three passes over the row.
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
            for (int c = threadIdx.x; c < a.cols; c += 1024) m0 += load_f(x + c) - x0;
            m0 = cta_sum(m0, slots[0]) * a.inv_n;
        }
        const float mu = x0 + m0;
        for (int c = threadIdx.x; c < a.cols; c += 1024) { const float d = load_f(x + c) - x0 - m0; q = fmaf(d, d, q); }
        const float rstd = 1.f / sqrtf(cta_sum(q, slots[1]) * a.inv_n + a.eps);
        if (a.stats && threadIdx.x == 0) { a.stats[2 * r] = mu; a.stats[2 * r + 1] = rstd; }
        T *y = (T *)a.y + r * a.ldy;
        for (int c = threadIdx.x; c < a.cols; c += 1024)
            store_f(y + c, fmaf((load_f(x + c) - x0 - m0) * rstd, param(a.weight, c, a.p_bf16, 1.f), param(a.bias, c, a.p_bf16, 0.f)));
        __syncthreads();
    }
}

constexpr int NB_ROWS = 2;     // rows that share a barrier

// NE columns per thread (8 or 16).  CTA false (up to 256 columns): a warp per pair of rows, the CTA's warps side by side, their column sums
// joined at the end; true: the whole CTA on a pair of rows.
template <typename T, bool VEC, int NE, bool CTA>
__global__ void __launch_bounds__(CTA ? 1024 : 256)
norm_backward_kernel(const NormArgs a)
{
    __shared__ float2 slots[2][NB_ROWS][32];
    __shared__ float joined[CTA ? 1 : 8][CTA ? 1 : 256];
    pdl_trigger();
    pdl_wait();
    const int tid = CTA ? threadIdx.x : (threadIdx.x & 31), threads = CTA ? blockDim.x : 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const int64_t per = CTA ? NB_ROWS : NB_ROWS * warps, first = CTA ? 0 : NB_ROWS * warp;
    float w[NE], dw[NE], db[NE];
#pragma unroll
    for (int k = 0; k < NE; ++k) {
        const int c = column_of<VEC>(k, tid, threads);
        w[k] = c < a.cols ? param(a.weight, c, a.p_bf16, 1.f) : 0.f;
        dw[k] = db[k] = 0.f;
    }
    int turn = 0;
    for (int64_t r0 = blockIdx.x * per + first; r0 < a.rows; r0 += gridDim.x * per, turn ^= 1) {
        float x[NB_ROWS][NE], g[NB_ROWS][NE], rs[NB_ROWS], mu[NB_ROWS];
        float2 s[NB_ROWS];
#pragma unroll
        for (int i = 0; i < NB_ROWS; ++i) {
            const int64_t r = min(r0 + i, a.rows - 1);       // (a row past the end is read again and left out below)
            load_row<T, VEC, NE>((const T *)a.x + r * a.ldx, tid, threads, a.cols, x[i]);
            load_row<T, VEC, NE>((const T *)a.dy + r * a.lddy, tid, threads, a.cols, g[i]);
            mu[i] = a.stats_in[2 * r];
            rs[i] = a.stats_in[2 * r + 1];
        }
#pragma unroll
        for (int i = 0; i < NB_ROWS; ++i) {
            const bool live = r0 + i < a.rows;
            s[i] = make_float2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < NE; ++k) {
                const bool in = column_of<VEC>(k, tid, threads) < a.cols;
                x[i][k] = in ? (x[i][k] - mu[i]) * rs[i] : 0.f;           // h
                if (live) {
                    dw[k] = fmaf(g[i][k], x[i][k], dw[k]);
                    db[k] += g[i][k];
                }
                g[i][k] *= w[k];
                s[i].x += g[i][k];
                s[i].y = fmaf(g[i][k], x[i][k], s[i].y);
            }
            s[i].x = warp_sum(s[i].x);
            s[i].y = warp_sum(s[i].y);
        }
        if (CTA) {
            if (lane < NB_ROWS) slots[turn][lane][warp] = lane == 0 ? s[0] : s[NB_ROWS - 1];
            __syncthreads();      // one per turn: the slots of the turn before last are written again only after the last one's barrier
#pragma unroll
            for (int i = 0; i < NB_ROWS; ++i) {
                const float2 t = lane < warps ? slots[turn][i][lane] : make_float2(0.f, 0.f);
                s[i].x = warp_sum(t.x);
                s[i].y = warp_sum(t.y);
            }
        }
#pragma unroll
        for (int i = 0; i < NB_ROWS; ++i) {
            if (!a.y || r0 + i >= a.rows) continue;
            const float c1 = a.center ? s[i].x * a.inv_n : 0.f, c2 = s[i].y * a.inv_n;
#pragma unroll
            for (int k = 0; k < NE; ++k) g[i][k] = rs[i] * (g[i][k] - fmaf(x[i][k], c2, c1));
            store_row<T, VEC, NE>((T *)a.y + (r0 + i) * a.ldy, tid, threads, a.cols, g[i]);
        }
    }
    // column sums of this CTA
#pragma unroll
    for (int set = 0; set < 2; ++set) {
        if (!(set ? a.want_db : a.want_dw)) continue;
        float *out = a.partial + ((int64_t)(set && a.want_dw ? gridDim.x : 0) + blockIdx.x) * a.cols;
        if (CTA) {
#pragma unroll
            for (int k = 0; k < NE; ++k) {
                const int c = column_of<VEC>(k, tid, threads);
                if (c < a.cols) out[c] = set ? db[k] : dw[k];
            }
        } else {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < NE; ++k) {
                const int c = column_of<VEC>(k, tid, threads);
                if (c < a.cols) joined[warp][c] = set ? db[k] : dw[k];
            }
            __syncthreads();
            for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
                float t = 0.f;
                for (int i = 0; i < warps; ++i) t += joined[i][c];
                out[c] = t;
            }
        }
    }
}

// Any width: dx alone, two passes over the row, ...
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
        for (int c = threadIdx.x; c < a.cols; c += 1024) {
            const float g = load_f(dy + c) * param(a.weight, c, a.p_bf16, 1.f);
            c1 += g;
            c2 = fmaf(g, (load_f(x + c) - mu) * rs, c2);
        }
        c1 = cta_sum(c1, slots[0]);
        c2 = cta_sum(c2, slots[1]) * a.inv_n;
        c1 = a.center ? c1 * a.inv_n : 0.f;
        T *dx = (T *)a.y + r * a.ldy;
        for (int c = threadIdx.x; c < a.cols; c += 1024) {
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

template <typename T, bool VEC>
cudaError_t forward_as(const NormArgs &a, int sms, cudaStream_t s)
{
    if (a.cols <= 2048) {
        const dim3 grid((unsigned)std::min<int64_t>((a.rows + 7) / 8, (int64_t)sms * 64));
        if (a.cols <= 256) return launch_dependent(norm_forward_kernel<T, VEC, 8, false>, grid, dim3(256), 0, s, 1, a);
        if (a.cols <= 512) return launch_dependent(norm_forward_kernel<T, VEC, 16, false>, grid, dim3(256), 0, s, 1, a);
        if (a.cols <= 1024) return launch_dependent(norm_forward_kernel<T, VEC, 32, false>, grid, dim3(256), 0, s, 1, a);
        return launch_dependent(norm_forward_kernel<T, VEC, 64, false>, grid, dim3(256), 0, s, 1, a);
    }
    const dim3 grid((unsigned)std::min<int64_t>(a.rows, (int64_t)sms * 64));
    if (a.cols <= 16384) return launch_dependent(norm_forward_kernel<T, VEC, 16, true>, grid, dim3((a.cols + 511) / 512 * 32), 0, s, 1, a);
    return launch_dependent(norm_forward_wide_kernel<T>, grid, dim3(1024), 0, s, 1, a);
}

// CTAs of the backward pass, each of which leaves a partial row: a few per SM, and no more than there are pairs of rows.
int backward_parts(int64_t rows, int64_t cols, int sms)
{
    const int threads = cols <= 256 ? 256 : (int)std::min<int64_t>(1024, (cols + 255) / 256 * 32);
    const int64_t pairs = (rows + NB_ROWS - 1) / NB_ROWS, warps_worth = cols <= 256 ? (pairs + 7) / 8 : pairs;
    if (cols > 16384) return (int)std::max<int64_t>(1, std::min<int64_t>((rows + 31) / 32, 64));
    return (int)std::max<int64_t>(1, std::min<int64_t>(warps_worth, (int64_t)sms * std::max(1, 1024 / threads)));
}

template <typename T, bool VEC>
cudaError_t backward_as(const NormArgs &a, int parts, cudaStream_t s)
{
    const dim3 grid(parts);
    if (a.cols <= 256) return launch_dependent(norm_backward_kernel<T, VEC, 8, false>, grid, dim3(256), 0, s, 1, a);
    if (a.cols <= 8192) return launch_dependent(norm_backward_kernel<T, VEC, 8, true>, grid, dim3((a.cols + 255) / 256 * 32), 0, s, 1, a);
    return launch_dependent(norm_backward_kernel<T, VEC, 16, true>, grid, dim3((a.cols + 511) / 512 * 32), 0, s, 1, a);
}

template <typename T>
cudaError_t backward_wide(const NormArgs &a, int parts, int sms, cudaStream_t s)
{
    if (a.y) {
        const cudaError_t e = launch_dependent(norm_backward_wide_kernel<T>, dim3((unsigned)std::min<int64_t>(a.rows, (int64_t)sms * 2)), dim3(1024), 0, s, 1, a);
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
bool whole_vectors(const tsr_matrix &m, const tsr_norm_desc &d)
{
    return !m.data || (aligned_to(m.data, 16) && (d.rows <= 1 || m.ld * type_bytes(d.dtype) % 16 == 0));
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
    const bool vec = d.cols % 8 == 0 && whole_vectors(x, d) && whole_vectors(y, d);
    cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e;
    if (d.dtype == TSR_BF16) e = vec ? forward_as<bf16, true>(a, sms, s) : forward_as<bf16, false>(a, sms, s);
    else e = vec ? forward_as<float, true>(a, sms, s) : forward_as<float, false>(a, sms, s);
    return e == cudaSuccess ? TSR_OK : TSR_ERR_CUDA;
}

extern "C" tsr_status tsr_norm_workspace_bytes(const tsr_norm_desc *desc, size_t *bytes)
{
    const tsr_status st = check_norm(desc);
    if (st != TSR_OK) return st;
    if (!bytes) return TSR_ERR_INVALID_ARG;
    const int sms = device_sms();
    *bytes = (size_t)2 * 4 * (size_t)desc->cols * (size_t)backward_parts(desc->rows, desc->cols, sms ? sms : 148);
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
    const int parts = backward_parts(d.rows, d.cols, sms);
    if (dweight || dbias) {
        const size_t need = (size_t)2 * 4 * (size_t)d.cols * (size_t)parts;
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
    if (d.rows > 0) {
        cudaError_t e;
        if (d.cols > 16384) e = d.dtype == TSR_BF16 ? backward_wide<bf16>(a, parts, sms, s) : backward_wide<float>(a, parts, sms, s);
        else {
            const bool vec = d.cols % 8 == 0 && whole_vectors(x, d) && whole_vectors(dy, d) && whole_vectors(dx, d);
            if (d.dtype == TSR_BF16) e = vec ? backward_as<bf16, true>(a, parts, s) : backward_as<bf16, false>(a, parts, s);
            else e = vec ? backward_as<float, true>(a, parts, s) : backward_as<float, false>(a, parts, s);
        }
        if (e != cudaSuccess) return TSR_ERR_CUDA;
    }
    const bool gb = d.g_dtype == TSR_BF16;
    void *one = dweight ? dweight : dbias, *two = dweight ? dbias : nullptr;
    if (one && column_finish((const float *)workspace, d.rows ? parts : 0, d.cols, d.cols, one, gb, two, gb, d.accumulate != 0, s) != cudaSuccess) return TSR_ERR_CUDA;
    return TSR_OK;
}
