// Linear layer: host side of its products (operand preparation, choice of tiles, split of K) and the kernels around them.
// Formulas in tsr.h; the products themselves are in tsr_linear_gemm.cu.
//
//   linear_pack_kernel     BF16 operand whose pitch or address TMA does not take -> workspace with a 128-byte pitch (one pass over it)
//   linear_split_kernel    FP32 operand -> three BF16 planes whose sum it is
//   linear_few_kernel      the whole layer for few rows
//   linear_dz_kernel       dz = dropout(dy) o act'(pre) and the column sums of dz (the bias's gradient), one pass over dy and pre
//   linear_finish_kernel   split K: slabs added in order, then the epilogue
//   column_finish_kernel   partial column sums added in order (bias, and the norm's weight and bias)
#include <math.h>

#include <algorithm>

#include "tsr_linear.cuh"

namespace tsr {

// ---- kernels ----------------------------------------------------------------------------------------------------------

// Operands that are copied, both of a product in one launch.  dst has a pitch of whole 16-byte units; a thread writes one unit of eight entries.
struct CopyJob {
    const void *src;
    bf16 *dst;
    int64_t lds, ldd, plane, rows;      // plane: entries between the three planes of an FP32 matrix
    int32_t cols, units;                // units per row
};
struct CopyJobs { CopyJob job[2]; int32_t n; };
// Which unit of which job, and its row and column.
__device__ __forceinline__ const CopyJob &job_at(const CopyJobs &a, int64_t u, int64_t first, int64_t &r, int &c)
{
    const bool second = u >= first;
    const CopyJob &j = a.job[second];
    if (second) u -= first;
    r = u < ((int64_t)1 << 32) ? (int64_t)((uint32_t)u / (uint32_t)j.units) : u / j.units;
    c = (int)(u - r * j.units) * 8;
    return j;
}
__global__ void __launch_bounds__(256)
linear_pack_kernel(const __grid_constant__ CopyJobs a)
{
    pdl_trigger();
    pdl_wait();
    const int64_t first = a.job[0].rows * a.job[0].units, total = first + (a.n > 1 ? a.job[1].rows * a.job[1].units : 0);
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
        int64_t r;
        int c;
        const CopyJob &j = job_at(a, u, first, r, c);
        const bf16 *s = (const bf16 *)j.src + r * j.lds + c;
        bf16 *d = j.dst + r * j.ldd + c;
        if (c + 8 <= j.cols) *(uint4 *)d = load16_any(s);
        else {
            for (int i = 0; i < j.cols - c; ++i) d[i] = s[i];
        }
    }
}

// x = p1 + p2 + p3 in BF16: each the rounded remainder of those before, 24 bits together (an entry below 2^-110 loses the bits that fall
// below 2^-133).  A value that would round to infinity keeps its leading bits; an infinity or NaN has no remainder.
__device__ __forceinline__ void split3(float x, bf16 (&p)[3])
{
    const uint32_t b = __float_as_uint(x);
    const bool special = (b & 0x7f800000u) == 0x7f800000u;
    p[0] = __float2bfloat16_rn(x);
    if (!special && (__float_as_uint(__bfloat162float(p[0])) & 0x7f800000u) == 0x7f800000u) p[0] = __ushort_as_bfloat16((unsigned short)(b >> 16));
    const float r1 = special ? 0.f : x - __bfloat162float(p[0]);
    p[1] = __float2bfloat16_rn(r1);
    p[2] = __float2bfloat16_rn(r1 - __bfloat162float(p[1]));
}
__device__ __forceinline__ void store_planes(bf16 *dst, int64_t plane, const float (&v)[8])
{
    uint32_t w[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bf16 a[3], b[3];
        split3(v[2 * i], a);
        split3(v[2 * i + 1], b);
#pragma unroll
        for (int k = 0; k < 3; ++k) w[k][i] = (uint32_t)__bfloat16_as_ushort(a[k]) | ((uint32_t)__bfloat16_as_ushort(b[k]) << 16);
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) *(uint4 *)(dst + k * plane) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
}
// FP32 -> three planes of rows x ldd, `plane` entries apart.
__global__ void __launch_bounds__(256)
linear_split_kernel(const __grid_constant__ CopyJobs a)
{
    pdl_trigger();
    pdl_wait();
    const int64_t first = a.job[0].rows * a.job[0].units, total = first + (a.n > 1 ? a.job[1].rows * a.job[1].units : 0);
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
        int64_t r;
        int c;
        const CopyJob &j = job_at(a, u, first, r, c);
        const float *s = (const float *)j.src + r * j.lds + c;
        float v[8];
        if (c + 8 <= j.cols) load8_any(s, v);
        else load8_part(s, j.cols - c, v);
        store_planes(j.dst + r * j.ldd + c, j.plane, v);      // (the pitch is whole units: what is written past the last column is zero)
    }
}

// Split tiles: the slabs of a tile (tile_m x width, FP32, one behind the other) are added in order, then the epilogue runs.  With `slabs` NULL the
// sum is zero and the tiles cover the whole matrix (K = 0).  A thread takes eight neighbours of a row.
struct FinishArgs {
    LinearTiles g;
    const float *slabs;
    int32_t tile_m, tail, out_f32;     // tiles that were split; type of out, residual and pre
    int32_t vec;                       // eight neighbours of out, residual and pre can be moved at once
    LinearEpilogue e;
};
template <typename T>
__device__ __forceinline__ void store_some(T *p, const float (&v)[8], int n, bool vec)
{
    if (vec && n == 8) store8(p, v);
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j) if (j < n) store_f(p + j, v[j]);
    }
}
template <typename T>
__global__ void __launch_bounds__(256)
linear_finish_kernel(const __grid_constant__ FinishArgs a)
{
    pdl_trigger();
    pdl_wait();
    const LinearEpilogue &e = a.e;
    const uint32_t per_row = a.g.width / 8, per_tile = a.tile_m * per_row;
    const int64_t total = (int64_t)a.tail * per_tile;
    const uint32_t call_key = e.drop.threshold ? drop_call_key(e.drop) : 0u;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
        const int tail = (int)(u / per_tile);
        const uint32_t in = (uint32_t)(u - (int64_t)tail * per_tile), rr = in / per_row, cc = (in - rr * per_row) * 8;
        int m0, n0;
        linear_tile_at(a.g, a.g.whole + tail, a.tile_m, m0, n0);
        const int64_t r = m0 + (int64_t)rr;
        const int c = n0 + (int)cc, n = min(8, a.g.N - c);
        if (r >= a.g.M || n <= 0) continue;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, o[8];
        if (e.res) {
            const T *res = (const T *)e.res + r * e.ldr + c;
            if (a.vec && n == 8) load8(res, o);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = j < n ? load_f(res + j) : 0.f;
            }
        }
        if (a.slabs) {
            const float *s = a.slabs + (int64_t)tail * a.g.splits * a.tile_m * a.g.width + (int64_t)in * 8;
#pragma unroll 4
            for (int p = 0; p < a.g.splits; ++p) {
                float x[8];
                load8(s + (int64_t)p * a.tile_m * a.g.width, x);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += x[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= e.scale;
        }
        if (e.bias) {
#pragma unroll
            for (int j = 0; j < 8; ++j) if (j < n) v[j] += load_as(e.bias, c + j, e.bias_bf16);
        }
        if (e.pre) store_some((T *)e.pre + r * e.ldp + c, v, n, a.vec);
        if (e.act) {
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
                // (one copy of the activation's code: rotated through the first place)
                const float z = act_value<T>(e.act, v[0]);
#pragma unroll
                for (int i = 0; i < 7; ++i) v[i] = v[i + 1];
                v[7] = z;
            }
        }
        if (e.drop.threshold) {
            const DropRow key = drop_row_key(call_key, r);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const uint32_t w = drop_word(key, (uint32_t)(c + j) >> 1);
                v[j] = drop_lo(w, v[j], e.drop);
                v[j + 1] = drop_hi(w, v[j + 1], e.drop);
            }
        }
        if (e.res) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += o[j];
        }
        store_some((T *)e.out + r * e.ldo + c, v, n, a.vec);
    }
}

// Few rows (up to eight at a time): the layer is bound by reading the weight once.  A warp takes four output columns at a time (what it reads of x counts for all
// of them) and every n-th slice of 256 entries of K, eight per lane at any alignment, against the rows of x in shared memory (FP32, a chunk of K at a
// time); FP32 stays in FP32 here.  Lanes, then the warps that share columns, join their sums, then a lane per entry runs the epilogue.  One launch,
// nothing in the workspace.
struct FewArgs {
    const void *x, *w;
    int64_t ldx, ldw;
    int32_t M, N, K, along_k, chunk;      // along_k: warps of a CTA that share columns; chunk: entries of K in shared memory at a time
    LinearEpilogue e;
};
constexpr int FEW_ROWS = 8, FEW_COLS = 4, FEW_SHARED = 24576;      // entries of x in shared memory: two CTAs fit an SM
constexpr int64_t FEW_MOST_K = 1 << 24;                           // beyond that K has to be split further, and the kernel counts in 32 bits
// N values of each lane (a power of two), summed over the lanes: with each exchange a lane keeps half of them; lane 32 / N * i has the i-th at last.
template <int N>
__device__ __forceinline__ float sums_over_lanes(const float (&v)[N], int lane, int step = 16)
{
    if constexpr (N == 1) {
        float x = v[0];
        for (int o = step; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        return x;
    } else {
        const bool hi = lane & step;
        float half[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) half[i] = (hi ? v[N / 2 + i] : v[i]) + __shfl_xor_sync(0xffffffffu, hi ? v[i] : v[N / 2 + i], step);
        return sums_over_lanes<N / 2>(half, lane, step / 2);
    }
}
// Eight entries of each of C rows from entry k on, all loads before the first use.
template <bool ALIGNED, int C>
__device__ __forceinline__ void load8_of(const bf16 *const (&w)[C], int k, float (&v)[C][8])
{
    uint4 a[C], b[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const uintptr_t at = (uintptr_t)(w[c] + k);
        const uint4 *base = (const uint4 *)(at & ~(uintptr_t)15);
        a[c] = __ldg(base);
        if (!ALIGNED) b[c] = __ldg(base + (at % 16 ? 1 : 0));
    }
#pragma unroll
    for (int c = 0; c < C; ++c) unpack8(ALIGNED ? a[c] : shift16(a[c], b[c], (uint32_t)(uintptr_t)(w[c] + k) & 15u), v[c]);
}
template <bool ALIGNED, int C>
__device__ __forceinline__ void load8_of(const float *const (&w)[C], int k, float (&v)[C][8])
{
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (ALIGNED) {
            const float4 a = __ldg((const float4 *)(w[c] + k)), b = __ldg((const float4 *)(w[c] + k) + 1);
            v[c][0] = a.x; v[c][1] = a.y; v[c][2] = a.z; v[c][3] = a.w; v[c][4] = b.x; v[c][5] = b.y; v[c][6] = b.z; v[c][7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = __ldg(w[c] + k + i);
        }
    }
}
// ALIGNED: the rows of the weight start on 16 bytes.
template <typename T, int ROWS, bool ALIGNED>
__global__ void __launch_bounds__(256, ROWS > 2 ? 2 : 3)
linear_few_kernel(const __grid_constant__ FewArgs a)
{
    constexpr int C = FEW_COLS, VALUES = ROWS * C;
    extern __shared__ __align__(16) float xs[];      // ROWS x chunk
    __shared__ float parts[8][VALUES];
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, kw = warp % a.along_k, per_cta = 8 / a.along_k * C, tiles = (a.N + per_cta - 1) / per_cta;
    const int row0 = blockIdx.y * ROWS, rows = min(ROWS, a.M - row0);
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int col0 = tile * per_cta + warp / a.along_k * C;
        const T *w[C];
#pragma unroll
        for (int c = 0; c < C; ++c) w[c] = (const T *)a.w + (int64_t)min(col0 + c, a.N - 1) * a.ldw;
        float2 acc[ROWS][C];
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c) acc[r][c] = pair(0.f);
        for (int k0 = 0; k0 < a.K; k0 += a.chunk) {
            const int len = min(a.chunk, a.K - k0), padded = (len + 7) & ~7;
            if (tile == (int)blockIdx.x || a.K > a.chunk) {      // (rows of one chunk stay)
                __syncthreads();
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
#pragma unroll 4
                    for (int i = threadIdx.x; i < padded; i += 256) xs[r * a.chunk + i] = r < rows && i < len ? load_f((const T *)a.x + (row0 + r) * a.ldx + k0 + i) : 0.f;
                __syncthreads();
            }
#pragma unroll 2
            for (int i = (kw * 32 + lane) * 8; i < len; i += a.along_k * 256) {
                float v[C][8];
                if (i + 8 <= len) load8_of<ALIGNED>(w, k0 + i, v);
                else {
#pragma unroll
                    for (int c = 0; c < C; ++c) load8_part(w[c] + k0 + i, len - i, v[c]);
                }
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const float4 p = *(const float4 *)&xs[r * a.chunk + i], q = *(const float4 *)&xs[r * a.chunk + i + 4];
#pragma unroll
                    for (int c = 0; c < C; ++c) {
                        acc[r][c] = fma2(make_float2(v[c][0], v[c][1]), make_float2(p.x, p.y), acc[r][c]);
                        acc[r][c] = fma2(make_float2(v[c][2], v[c][3]), make_float2(p.z, p.w), acc[r][c]);
                        acc[r][c] = fma2(make_float2(v[c][4], v[c][5]), make_float2(q.x, q.y), acc[r][c]);
                        acc[r][c] = fma2(make_float2(v[c][6], v[c][7]), make_float2(q.z, q.w), acc[r][c]);
                    }
                }
            }
        }
        float sums[VALUES];
#pragma unroll
        for (int i = 0; i < VALUES; ++i) sums[i] = acc[i / C][i % C].x + acc[i / C][i % C].y;
        float z = sums_over_lanes<VALUES>(sums, lane);
        const int value = lane / (32 / VALUES), r = value / C, col = col0 + value % C;
        if (a.along_k > 1) {
            __syncthreads();      // (of the tile before, all have been read)
            if (lane % (32 / VALUES) == 0) parts[warp][value] = z;
            __syncthreads();
            if (kw) continue;
            z = 0.f;
            for (int k = 0; k < a.along_k; ++k) z += parts[warp + k][value];
        }
        if (lane % (32 / VALUES) || r >= rows || col >= a.N) continue;
        const LinearEpilogue &e = a.e;
        const int64_t row = row0 + r;
        if (e.bias) z += load_as(e.bias, col, e.bias_bf16);
        if (e.pre) store_f((T *)e.pre + row * e.ldp + col, z);
        z = act_value<T>(e.act, z);
        if (e.drop.threshold) z = drop_entry(drop_row_key(drop_call_key(e.drop), row), (uint32_t)col, z, e.drop);
        if (e.res) z += load_f((const T *)e.res + row * e.ldr + col);
        store_f((T *)e.out + row * e.ldo + col, z);
    }
}
// Rows of a matrix that start on 16 bytes.
static bool tma_takes(const void *p, int64_t rows, int64_t ld, int es) { return aligned_to(p, 16) && (rows <= 1 || (ld * es) % 16 == 0); }
template <typename T>
static cudaError_t few_launch(FewArgs a, int sms, cudaStream_t s)
{
    // as many CTAs as SMs at least, as long as there is K to share
    a.along_k = 1;
    const int groups = (a.M + FEW_ROWS - 1) / FEW_ROWS;
    while (a.along_k < 8 && a.along_k * 256 < a.K && (int64_t)a.N * a.along_k * groups < (int64_t)sms * 2 * 8 * FEW_COLS) a.along_k *= 2;
    const int per_cta = 8 / a.along_k * FEW_COLS;
    const dim3 grid((unsigned)std::min((a.N + per_cta - 1) / per_cta, sms * (a.M > 2 ? 2 : 3)), groups);
    const int rows = a.M <= 2 ? a.M : a.M <= 4 ? 4 : FEW_ROWS;
    a.chunk = (int)std::min<int64_t>(FEW_SHARED / rows, round_up(a.K, 8));
    const size_t smem = (size_t)rows * a.chunk * 4;
    const auto launch = [&](auto kernel) {
        // (the same limit in every call: it belongs to the kernel, and other threads may be between here and their launch)
        const cudaError_t e = smem > 40 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SHARED * 4) : cudaSuccess;
        return e == cudaSuccess ? launch_dependent(kernel, grid, dim3(256), smem, s, 1, a) : e;
    };
    if (tma_takes(a.w, a.N, a.ldw, sizeof(T))) {
        if (a.M <= 1) return launch(linear_few_kernel<T, 1, true>);
        if (a.M <= 2) return launch(linear_few_kernel<T, 2, true>);
        if (a.M <= 4) return launch(linear_few_kernel<T, 4, true>);
        return launch(linear_few_kernel<T, FEW_ROWS, true>);
    }
    if (a.M <= 1) return launch(linear_few_kernel<T, 1, false>);
    if (a.M <= 2) return launch(linear_few_kernel<T, 2, false>);
    if (a.M <= 4) return launch(linear_few_kernel<T, 4, false>);
    return launch(linear_few_kernel<T, FEW_ROWS, false>);
}

// dz and its column sums.  BF16 layers round dz, as an operand of both products (error of dx and dweight 0.0017 -> 0.0023 of the result, three quarters of
// which their own rounding brings anyway; two parts would double the products).  Without an activation dz is a selection from dy, rounded by nothing: the factor
// of dropout is left to the products' epilogue.  A CTA takes 256 columns and a range of rows; a lane eight columns side by side, a warp every eighth row.  dy and pre
// may lie at any alignment, dz has a pitch of whole 16-byte units.  dz NULL: the sums alone.
// The grid is what is resident at once (a third more left SMs idle for 40 % of the time), and what hides the loads is the number of warps: unrolled
// loops were slower, the more so the further (8192 x 5461 with SiLU off the 16-byte grid: 58 us; at an earlier stage 72, unrolled twice 95, four times 131 at three CTAs).
constexpr int DZ_CTAS = 4;     // on an SM
struct DzArgs {
    const void *dy, *pre;
    void *dz;                  // BF16, or (FP32) three BF16 planes `plane` entries apart
    float *partial;            // [gridDim.y][cols], NULL: no sums, or they go to `sums`
    void *sums;                // with a single range of rows: the sums themselves
    int32_t sums_bf16, accumulate;
    int64_t lddy, ldpre, lddz, plane, rows;
    int32_t cols, rows_per;
    DropArgs drop;             // with a factor of 1 where ACT is TSR_ACT_NONE
    float sum_scale;           // of the sums: the factor there, otherwise 1
};
template <typename T, int ACT>
__global__ void __launch_bounds__(256, DZ_CTAS)
linear_dz_kernel(const DzArgs a)
{
    __shared__ float sums[8][256];
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = blockIdx.x * 256 + lane * 8, n = a.cols - c0;
    const int64_t r0 = (int64_t)blockIdx.y * a.rows_per + warp, r1 = min(a.rows, (int64_t)(blockIdx.y + 1) * a.rows_per);
    const uint32_t call_key = a.drop.threshold ? drop_call_key(a.drop) : 0u;
    float acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    if (n > 0) {
        const T *dy = (const T *)a.dy + r0 * a.lddy + c0, *pre = ACT ? (const T *)a.pre + r0 * a.ldpre + c0 : nullptr;
        bf16 *dz = a.dz ? (bf16 *)a.dz + r0 * a.lddz + c0 : nullptr;
#pragma unroll 1
        for (int64_t r = r0; r < r1; r += 8) {
            float g[8], z[8];
            if (n >= 8) {
                load8_any(dy, g);
                if (ACT) load8_any(pre, z);
            } else {
                load8_part(dy, n, g);
                if (ACT) load8_part(pre, n, z);
            }
            if (ACT) {
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const float2 d = slope_pair<T, ACT>(make_float2(z[j], z[j + 1]));
                    g[j] *= d.x;
                    g[j + 1] *= d.y;
                }
                pre += 8 * a.ldpre;
            }
            if (a.drop.threshold) {      // last, as a selection: what fell is zero whatever pre holds
                const DropRow key = drop_row_key(call_key, r);
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const uint32_t w = drop_word(key, (uint32_t)(c0 + j) >> 1);
                    g[j] = drop_lo(w, g[j], a.drop);
                    g[j + 1] = drop_hi(w, g[j + 1], a.drop);
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += g[j];
            if (dz) {
                // (past the last column: zeros, into the padding)
                if constexpr (sizeof(T) == 2) store8(dz, g);
                else store_planes(dz, a.plane, g);
                dz += 8 * a.lddz;
            }
            dy += 8 * a.lddy;
        }
    }
    if (!a.partial && !a.sums) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[warp][lane * 8 + j] = acc[j];
    __syncthreads();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < a.cols) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += sums[w][threadIdx.x];
        s *= a.sum_scale;
        if (a.partial) a.partial[(int64_t)blockIdx.y * a.cols + c] = s;
        else store_as(a.sums, c, a.sums_bf16, a.accumulate ? s + load_as(a.sums, c, a.sums_bf16) : s);
    }
}

template <typename T>
static cudaError_t dz_launch(const DzArgs &a, int act, dim3 grid, cudaStream_t s)
{
    switch (act) {
    case TSR_ACT_RELU: return launch_dependent(linear_dz_kernel<T, TSR_ACT_RELU>, grid, dim3(256), 0, s, 1, a);
    case TSR_ACT_GELU: return launch_dependent(linear_dz_kernel<T, TSR_ACT_GELU>, grid, dim3(256), 0, s, 1, a);
    case TSR_ACT_GELU_TANH: return launch_dependent(linear_dz_kernel<T, TSR_ACT_GELU_TANH>, grid, dim3(256), 0, s, 1, a);
    case TSR_ACT_SILU: return launch_dependent(linear_dz_kernel<T, TSR_ACT_SILU>, grid, dim3(256), 0, s, 1, a);
    default: return launch_dependent(linear_dz_kernel<T, TSR_ACT_NONE>, grid, dim3(256), 0, s, 1, a);
    }
}

// CW columns per CTA of 1024 threads: 32, or 8 where 32 would leave half of the SMs without work.  Threads of a column add every (1024 / CW)-th row, their sums are
// added over the lanes of a warp and then over the warps: the order depends on sizes alone.  (586 rows of 512 columns: 7.5 us with 32, 4.8 with 8.)
template <int CW>
__global__ void __launch_bounds__(1024)
column_finish_kernel(const float *__restrict__ partial, int parts, int64_t ldp, int64_t cols, void *out, int out_bf16, void *out2, int out2_bf16, int accumulate)
{
    __shared__ float sums[32][CW + 1];
    pdl_trigger();
    pdl_wait();
    if (blockIdx.y) { partial += parts * ldp; out = out2; out_bf16 = out2_bf16; }
    const int x = threadIdx.x % CW, y = threadIdx.x / CW, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * CW + x;
    float s = 0.f;
    if (c < cols) {
#pragma unroll 16
        for (int p = y; p < parts; p += 1024 / CW) s += partial[p * ldp + c];
    }
#pragma unroll
    for (int o = CW; o < 32; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) < CW) sums[warp][x] = s;
    __syncthreads();
    if (y == 0 && c < cols) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) s += sums[i][x];
        if (accumulate) s += load_as(out, c, out_bf16);
        store_as(out, c, out_bf16, s);
    }
}

// ---- shared host helpers ----------------------------------------------------------------------------------------------

int device_sms()
{
    static int known[64] = {};
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return 0; }
    if (dev < 64 && known[dev]) return known[dev];
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) { cudaGetLastError(); return 0; }
    if (dev < 64) known[dev] = n;
    return n;
}

bool drop_args(const tsr_dropout_desc &d, DropArgs *out)
{
    if (!(d.p >= 0.f && d.p <= 1.f)) return false;
    out->threshold = (uint32_t)floor((double)d.p * 65536.0 + 0.5);
    out->scale = out->threshold == 65536u ? 0.f : (float)(65536.0 / (65536 - (int)out->threshold));
    if (!aligned_to(d.step, 8)) return false;
    out->seed_key = mix32((uint32_t)d.seed ^ mix32((uint32_t)(d.seed >> 32) + 0x9e3779b9u));
    out->offset = d.offset;
    out->step = d.step;
    return true;
}

cudaError_t column_finish(const float *partial, int parts, int64_t ldp, int64_t cols, void *out, bool out_bf16, void *out2, bool out2_bf16,
                          bool accumulate, cudaStream_t stream)
{
    if (cols <= 0) return cudaSuccess;
    const int sets = out2 ? 2 : 1;
    const bool narrow = (cols + 31) / 32 * sets <= device_sms() / 2;
    const auto launch = [&](auto kernel, int cw) {
        return launch_dependent(kernel, dim3((unsigned)((cols + cw - 1) / cw), sets), dim3(1024), 0, stream, 1, partial, parts, ldp, cols, out, (int)out_bf16, out2, (int)out2_bf16, (int)accumulate);
    };
    return narrow ? launch(column_finish_kernel<8>, 8) : launch(column_finish_kernel<32>, 32);
}

// ---- one product ------------------------------------------------------------------------------------------------------

namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                  const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encoder()
{
    static EncodeTiledFn fn = nullptr;
    if (!fn) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        fn = (EncodeTiledFn)p;
    }
    return fn;
}

// Row-major matrix, boxes of `inner` bytes (128 or 64, with the swizzle of that width) x box_rows; planes > 1: that many of them, `plane` entries
// apart, in one box.
bool encode(CUtensorMap *out, const void *base, int64_t rows, int64_t cols, int64_t ld, bool f32, int box_rows, int inner = 128, int planes = 1, int64_t plane = 0)
{
    EncodeTiledFn fn = encoder();
    if (!fn) return false;
    const int es = f32 ? 4 : 2;
    if (rows <= 1) ld = round_up(cols, 16 / es);         // a single row has no pitch
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes}, strides[2] = {(cuuint64_t)ld * es, (cuuint64_t)plane * es};
    const cuuint32_t box[3] = {(cuuint32_t)(inner / es), (cuuint32_t)box_rows, (cuuint32_t)planes}, step[3] = {1, 1, 1};
    return fn(out, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, planes > 1 ? 3 : 2, const_cast<void *>(base), dims, strides, box, step,
              CU_TENSOR_MAP_INTERLEAVE_NONE, inner == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}


// [rows x K], or (mn) stored as [K x rows].  FP32 operands come as three BF16 planes, `plane` entries apart (see three_planes).
struct Operand { const void *p; int64_t ld; bool mn; int64_t plane; };

struct Product {
    int64_t M, N, K;
    bool f32;            // operands
    Operand A, B;
    bool out_f32;
    LinearEpilogue e;    // out, res, pre, bias with their pitches
};

struct Shape { int cg, width, splits, kb, kb_per; int64_t m_tiles, n_tiles, whole, tail; };   // tail: tiles that are split

// Tile shape and split of K by a model in SM clocks.  A K block of 64 entries costs the MMAs 2 width clocks (32 of FP32: 6 width) and the SM's
// intake of 64 bytes a clock its share of the operands; a wave of tiles costs the larger one times its blocks.  The tiles of the last wave
// (and, where that is nearly full, of the one before) may be split, so that the last wave is short: for that their slabs are
// written (32 bytes a clock and SM) and read again (3000 bytes a clock in all) by another launch.
Shape search(const Product &p, int sms)
{
    Shape best = {};
    double best_cost = 1e300;
    const int bk = p.f32 ? 32 : 64, kb = (int)((p.K + bk - 1) / bk);
    static const struct { int cg, width; } kinds[] = {{2, 256}, {2, 192}, {2, 128}, {2, 64}, {1, 128}, {1, 64}};
    for (const auto &k : kinds) {
        const int64_t mt = (p.M + 128 * k.cg - 1) / (128 * k.cg), nt = (p.N + k.width - 1) / k.width, tiles = mt * nt;
        const int slots = sms / k.cg;
        const double mma = (p.f32 ? 6.0 : 2.0) * k.width, intake = (p.f32 ? 3.0 : 2.0) * (128 + k.width / k.cg);
        const int stage = (p.f32 ? 3 * 64 : 128) * (128 + k.width / k.cg), stages = linear_stages(stage, p.e.pre != nullptr);
        // (with a single stage loads and MMAs take turns)
        const double per_kb = stages > 1 ? std::max(mma, intake) : mma + intake + 1000.0, tile = kb * per_kb + 300.0, last = 3000.0 + 800.0 * (k.cg - 1) + 12.0 * k.width;
        const int64_t full = tiles / slots, rem = tiles % slots;
        auto offer = [&](double cost, int64_t tail, int s, int per) {
            if (cost < best_cost) { best_cost = cost; best = {k.cg, k.width, s, kb, per, mt, nt, tiles - tail, tail}; }
        };
        offer(last + (double)(full + (rem ? 1 : 0)) * tile, 0, 1, kb);
        for (int extra = 0; extra < 2; ++extra) {
            const int64_t tail = rem + (extra ? slots : 0);
            if (tail == 0 || tail > tiles) continue;
            const int most = (int)std::min<int64_t>(kb / 2, 2 * slots / tail + 1);
            for (int want = 2; want <= most; ++want) {
                const int per = (kb + want - 1) / want, s = (kb + per - 1) / per;
                if (s != want) continue;
                const double waves = (double)((tail * s + slots - 1) / slots), slab = 128.0 * k.width * 4;
                offer(last + (double)((tiles - tail) / slots) * tile + waves * (per * per_kb + 300.0 + slab / 32.0) + 4000.0 + (double)tail * s * slab * k.cg / 3000.0, tail, s, per);
            }
        }
    }
    return best;
}

// The search takes a few microseconds and a call needs its result several times: the last results of the host thread are kept, by sizes.
Shape choose(const Product &p, int sms)
{
    struct Known { int64_t M, N, K; int f32, pre, sms; Shape shape; };
    static thread_local Known known[8] = {};
    static thread_local int next = 0;
    const int f32 = p.f32, pre = p.e.pre != nullptr;
    for (const Known &k : known)
        if (k.M == p.M && k.N == p.N && k.K == p.K && k.f32 == f32 && k.pre == pre && k.sms == sms) return k.shape;
    Known &k = known[next++ & 7];
    k = {p.M, p.N, p.K, f32, pre, sms, search(p, sms)};
    return k.shape;
}

// Whether the kernel for few rows takes the product.  us, it / the tensor cores (which copy a weight that is not aligned, and split FP32 in three):
//   BF16 aligned      2048 -> 2048, 1 row 4.8 / 7.9, 4 rows 7.1 / 7.9, 8 rows 10.4 / 8.0;  2048 -> 32768, 1 row 28.3 / 25.2
//   BF16 not aligned  2047 -> 2047, 1 row 5.4 / 12.1, 8 rows 11.7 / 14.2;  5461 -> 2048, 4 rows 15.4 / 19.8, 8 rows (x does not fit) 40.9 / 19.7
//   FP32              2048 -> 2048, 1 row 4.8 / 19.7, 8 rows 10.7 / 20.0;  5461 -> 2048, 4 rows 23.8 / 40.9, 8 rows (does not fit) 47.0 / 41.0
// Without aligned BF16, more rows go through it in groups of eight while the product is small: one launch instead of two or three (64 x 512 -> 512 FP32
// 8.2 / 11.2, 64 x 700 -> 700 19.4 / 13.5; BF16 not aligned 64 x 511 -> 512 8.7 / 7.2).
bool few_rows(const Product &p)
{
    if (p.M <= 0 || p.M > 8 * FEW_ROWS || p.N <= 0 || p.K <= 0 || p.K > FEW_MOST_K) return false;
    const bool fits = (p.M <= 2 ? p.M : p.M <= 4 ? 4 : FEW_ROWS) * p.K <= FEW_SHARED;
    const double size = (double)p.M * p.N * p.K;
    if (!p.f32 && tma_takes(p.B.p, p.N, p.B.ld, 2)) return fits && p.M <= 4 && size <= 33554432.0;
    if (p.M > FEW_ROWS) return fits && size <= (p.f32 ? 16777216.0 : 8388608.0);
    return fits || (p.f32 && p.M <= 4);
}

struct Room {      // walks the workspace; with base NULL it only counts
    char *base;
    size_t at;
    void *take(size_t bytes)
    {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return base ? base + here : nullptr;
    }
};

template <typename Kern>
cudaError_t copy_operands(Kern kernel, const CopyJobs &jobs, int sms, cudaStream_t stream)
{
    int64_t units = 0;
    for (int i = 0; i < jobs.n; ++i) units += jobs.job[i].rows * jobs.job[i].units;
    if (!units) return cudaSuccess;
    return launch_dependent(kernel, dim3((unsigned)std::min<int64_t>((units + 255) / 256, (int64_t)sms * 32)), dim3(256), 0, stream, 1, jobs);
}

// The product's scratch, and (run) its launches.
tsr_status product(const Product &p, Room &room, bool run, int sms, cudaStream_t stream)
{
    if (p.M == 0 || p.N == 0) return TSR_OK;
    const int os = p.out_f32 ? 4 : 2;
    const bool out_tma = tma_takes(p.e.out, p.M, p.e.ldo, os), res_tma = p.e.res && tma_takes(p.e.res, p.M, p.e.ldr, os), pre_tma = p.e.pre && tma_takes(p.e.pre, p.M, p.e.ldp, os);
    FinishArgs f = {};
    f.out_f32 = p.out_f32;
    f.e = p.e;
    f.vec = out_tma && (!p.e.pre || pre_tma) && (!p.e.res || res_tma);
    auto finish = [&]() -> tsr_status {
        const int64_t units = (int64_t)f.tail * f.tile_m * (f.g.width / 8);
        const dim3 grid((unsigned)std::min<int64_t>((units + 255) / 256, (int64_t)sms * 16));
        const cudaError_t rc = f.out_f32 ? launch_dependent(linear_finish_kernel<float>, grid, dim3(256), 0, stream, 1, f) : launch_dependent(linear_finish_kernel<bf16>, grid, dim3(256), 0, stream, 1, f);
        return rc == cudaSuccess ? TSR_OK : TSR_ERR_CUDA;
    };
    if (p.K == 0) {
        f.tile_m = 128;
        f.g.M = (int)p.M; f.g.N = (int)p.N; f.g.width = 64;
        const int64_t mt = (p.M + 127) / 128, nt = (p.N + 63) / 64;
        if (mt * nt > (int64_t)1 << 30) return TSR_ERR_SHAPE;
        f.g.m_tiles = (int)mt; f.g.n_tiles = (int)nt; f.tail = (int)(mt * nt);
        return run ? finish() : TSR_OK;
    }

    Shape s = choose(p, sms);
    if (p.f32 && !p.out_f32 && s.whole) {
        // FP32 operands, BF16 weight gradient: the kernel has FP32 boxes alone there, so all tiles go through slabs, as single parts where K needs no split
        s.tail = s.m_tiles * s.n_tiles;
        s.whole = 0;
        s.splits = 1;
        s.kb_per = s.kb;
    }
    if (s.m_tiles * s.n_tiles > (int64_t)1 << 28) return TSR_ERR_SHAPE;
    LinearGemm g = {};
    g.M = (int)p.M; g.N = (int)p.N;
    g.width = s.width; g.m_tiles = (int)s.m_tiles; g.n_tiles = (int)s.n_tiles;
    g.whole = (int)s.whole; g.splits = s.splits; g.items = (int)(s.whole + s.tail * s.splits);
    g.kb_total = s.kb; g.kb_per = s.kb_per;

    // A product with few rows fetches no more of A than exists (the MMAs then read what shared memory happens to hold: rows that nobody stores)
    const int a_rows = s.cg == 1 && s.m_tiles == 1 ? (int)round_up(std::min<int64_t>(p.M, 128), 16) : 128;
    // operands
    const int planes = p.f32 ? 3 : 1, inner = p.f32 ? 64 : 128;
    const Operand *op[2] = {&p.A, &p.B};
    CopyJobs jobs = {};
    const int64_t extent[2] = {p.M, p.N};
    for (int i = 0; i < 2; ++i) {
        const Operand &o = *op[i];
        const int64_t rows = o.mn ? p.K : extent[i], cols = o.mn ? extent[i] : p.K;    // as stored
        const void *at = o.p;
        int64_t ld = o.ld;
        // A K-major operand whose rows do not start on 128 bytes costs two lines per row and K block, a fifth of the product's time; copying
        // it first pays where the other extent is long enough.  us, as it lies / copied: 8192 x 5464 -> 2048 (the weight) 150 / 134, 8192 x 2056 -> 8192 (both) 220 / 195,
        // 16384 x 1032 -> 1032 52 / 46, 1500 x 8200 -> 5464 (x) 126 / 108; 4096 x 520 -> 512 13 / 15, 2048 x 5464 -> 2048 (neither by the rule) 48 / 57.
        const bool straddles = !o.mn && rows > 1 && (o.ld % 64 || !aligned_to(o.p, 128)) && p.K >= 512 && extent[1 - i] >= 3200;
        if (!p.f32 && (straddles || !tma_takes(o.p, rows, o.ld, 2))) {
            ld = round_up(cols, 64);
            bf16 *copy = (bf16 *)room.take((size_t)rows * ld * 2);
            jobs.job[jobs.n++] = {o.p, copy, o.ld, ld, 0, rows, (int)cols, (int)((cols + 7) / 8)};
            at = copy;
        }
        // an MN-major box: 64 entries side by side (128 bytes) x the K block; a K-major one: the K block x the rows of a CTA
        const bool ok = !run || (o.mn ? encode(i ? &g.tmB : &g.tmA, at, rows, cols, ld, false, inner / 2, 128, planes, o.plane)
                                      : encode(i ? &g.tmB : &g.tmA, at, rows, cols, ld, false, i ? s.width / s.cg : a_rows, inner, planes, o.plane));
        if (!ok) return TSR_ERR_CUDA;
        (i ? g.b_mn : g.a_mn) = o.mn;
    }
    if (run && copy_operands(linear_pack_kernel, jobs, sms, stream) != cudaSuccess) return TSR_ERR_CUDA;
    g.a_rows = a_rows;
    g.a_boxes = (a_rows + 63) / 64;
    g.b_boxes = (s.width / s.cg + 63) / 64;
    const int a_bytes = planes * 128 * inner, a_copied = planes * (g.a_mn ? g.a_boxes * 64 * inner : a_rows * inner), b_bytes = planes * (g.b_mn ? g.b_boxes * 64 * inner : s.width / s.cg * inner);
    g.b_offset = a_bytes;
    g.stage_bytes = a_bytes + b_bytes;
    g.stage_tx = (uint32_t)(s.cg * (a_copied + b_bytes));
    g.stages = linear_stages(g.stage_bytes, p.e.pre != nullptr);

    float *slabs = s.tail ? (float *)room.take((size_t)s.tail * s.splits * 128 * s.cg * s.width * 4) : nullptr;
    if (!run) return TSR_OK;
    if (s.tail && !encode(&g.tmSlab, slabs, s.tail * s.splits * 128 * s.cg, s.width, s.width, true, 32)) return TSR_ERR_CUDA;
    g.e = p.e;
    g.whole_edge = p.N * os % 16 == 0;
    for (int i = 0; i < 2 && p.f32; ++i) g.parts[i] = {(const bf16 *)op[i]->p, op[i]->ld, op[i]->plane};
    g.K = (int)p.K;
    if (s.whole) {
        g.e.out_tma = out_tma;
        g.e.res_tma = res_tma;
        g.e.pre_tma = pre_tma;
        if (out_tma && !encode(&g.tmOut, p.e.out, p.M, p.N, p.e.ldo, p.out_f32, 32)) return TSR_ERR_CUDA;
        if (res_tma && !encode(&g.tmRes, p.e.res, p.M, p.N, p.e.ldr, p.out_f32, 32)) return TSR_ERR_CUDA;
        if (pre_tma && !encode(&g.tmPre, p.e.pre, p.M, p.N, p.e.ldp, p.out_f32, 32)) return TSR_ERR_CUDA;
    }
    if (linear_gemm_launch(g, s.cg, p.f32, p.out_f32, sms, stream) != cudaSuccess) return TSR_ERR_CUDA;
    if (!s.tail) return TSR_OK;
    f.g = g;
    f.slabs = slabs;
    f.tile_m = 128 * s.cg;
    f.tail = (int)s.tail;
    return finish();
}

// Three BF16 planes of an FP32 matrix (rows x cols) in the workspace, as an operand; the copy is left to `jobs`.
void three_planes(const tsr_matrix &m, int64_t rows, int64_t cols, bool mn, Operand *o, Room &room, CopyJobs *jobs)
{
    o->ld = round_up(std::max<int64_t>(cols, 1), 64);
    o->plane = std::max<int64_t>(rows, 1) * o->ld;
    o->mn = mn;
    bf16 *copy = (bf16 *)room.take((size_t)3 * o->plane * 2);
    o->p = copy;
    if (rows && cols) jobs->job[jobs->n++] = {m.data, copy, m.ld, o->ld, o->plane, rows, (int)cols, (int)((cols + 7) / 8)};
}

constexpr int64_t MOST = 0x7fffffff - 1023;

tsr_status check_desc(const tsr_linear_desc &d, DropArgs *drop)
{
    if (!type_ok(d.dtype) || !type_ok(d.b_dtype) || !type_ok(d.gw_dtype) || !type_ok(d.gb_dtype)) return TSR_ERR_UNSUPPORTED;
    if (d.activation < TSR_ACT_NONE || d.activation > TSR_ACT_SILU) return TSR_ERR_UNSUPPORTED;
    if (d.rows < 0 || d.ins < 0 || d.outs < 0 || d.rows > MOST || d.ins > MOST || d.outs > MOST) return TSR_ERR_SHAPE;
    if (!drop_args(d.dropout, drop)) return TSR_ERR_INVALID_ARG;
    return TSR_OK;
}
// A matrix that the call needs, or (want false) may do without.
tsr_status check_matrix(const tsr_matrix &m, int64_t rows, int64_t cols, int32_t dtype, bool want)
{
    if (!m.data) return want && rows > 0 && cols > 0 ? TSR_ERR_INVALID_ARG : TSR_OK;
    if (!extent_ok(rows, cols, m.ld)) return TSR_ERR_SHAPE;
    return aligned_to(m.data, type_bytes(dtype)) ? TSR_OK : TSR_ERR_ALIGNMENT;
}

#define CHECK_MATRIX(m, rows, cols, dtype, want) \
    do { const tsr_status st_ = check_matrix(m, rows, cols, dtype, want); if (st_ != TSR_OK) return st_; } while (0)

tsr_status forward(const tsr_linear_desc *d, const tsr_linear_io *io, void *workspace, size_t bytes, size_t *need, cudaStream_t stream)
{
    if (!d || !io) return TSR_ERR_INVALID_ARG;
    Product p = {};
    tsr_status st = check_desc(*d, &p.e.drop);
    if (st != TSR_OK) return st;
    CHECK_MATRIX(io->x, d->rows, d->ins, d->dtype, true);
    CHECK_MATRIX(io->weight, d->outs, d->ins, d->dtype, true);
    CHECK_MATRIX(io->residual, d->rows, d->outs, d->dtype, false);
    CHECK_MATRIX(io->pre, d->rows, d->outs, d->dtype, false);
    CHECK_MATRIX(io->y, d->rows, d->outs, d->dtype, true);
    if (!aligned_to(io->bias, type_bytes(d->b_dtype))) return TSR_ERR_ALIGNMENT;
    p.M = d->rows; p.N = d->outs; p.K = d->ins;
    p.f32 = p.out_f32 = d->dtype == TSR_F32;
    p.A = {io->x.data, io->x.ld, false, 0};
    p.B = {io->weight.data, io->weight.ld, false, 0};
    p.e.out = io->y.data; p.e.ldo = io->y.ld;
    p.e.res = io->residual.data; p.e.ldr = io->residual.ld;
    p.e.pre = io->pre.data; p.e.ldp = io->pre.ld;
    p.e.bias = io->bias; p.e.bias_bf16 = d->b_dtype == TSR_BF16;
    p.e.act = d->activation;
    p.e.scale = 1.f;
    const int sms = device_sms();
    const auto all = [&](Room &room, bool run, int n) -> tsr_status {
        if (few_rows(p)) {
            if (!run) return TSR_OK;
            FewArgs a = {};
            a.x = io->x.data; a.ldx = io->x.ld; a.w = io->weight.data; a.ldw = io->weight.ld;
            a.M = (int)p.M; a.N = (int)p.N; a.K = (int)p.K;
            a.e = p.e;
            return (p.f32 ? few_launch<float>(a, n, stream) : few_launch<bf16>(a, n, stream)) == cudaSuccess ? TSR_OK : TSR_ERR_CUDA;
        }
        if (p.f32 && p.M > 0 && p.N > 0 && p.K > 0) {
            CopyJobs jobs = {};
            three_planes(io->x, d->rows, d->ins, false, &p.A, room, &jobs);
            three_planes(io->weight, d->outs, d->ins, false, &p.B, room, &jobs);
            if (run && copy_operands(linear_split_kernel, jobs, n, stream) != cudaSuccess) return TSR_ERR_CUDA;
        }
        return product(p, room, run, n, stream);
    };
    Room count = {nullptr, 0};
    st = all(count, false, sms ? sms : 148);
    if (st != TSR_OK) return st;
    if (need) { *need = count.at; return TSR_OK; }
    if (count.at && (!workspace || bytes < count.at)) return TSR_ERR_WORKSPACE;
    if (count.at && !aligned_to(workspace, 256)) return TSR_ERR_ALIGNMENT;
    if (p.M == 0 || p.N == 0) return TSR_OK;
    if (!sms) return TSR_ERR_CUDA;
    Room room = {(char *)workspace, 0};
    return all(room, true, sms);
}

constexpr int DZ_COLS = 256;

tsr_status backward(const tsr_linear_desc *d, const tsr_linear_grads *io, void *workspace, size_t bytes, size_t *need, cudaStream_t stream)
{
    if (!d || !io) return TSR_ERR_INVALID_ARG;
    DropArgs drop;
    tsr_status st = check_desc(*d, &drop);
    if (st != TSR_OK) return st;
    const bool dx = io->dx.data, dw = io->dweight.data, db = io->dbias;
    CHECK_MATRIX(io->dy, d->rows, d->outs, d->dtype, dx || dw || db);
    CHECK_MATRIX(io->pre, d->rows, d->outs, d->dtype, d->activation != TSR_ACT_NONE && (dx || dw || db));
    CHECK_MATRIX(io->weight, d->outs, d->ins, d->dtype, dx);
    CHECK_MATRIX(io->x, d->rows, d->ins, d->dtype, dw);
    CHECK_MATRIX(io->dx, d->rows, d->ins, d->dtype, false);
    CHECK_MATRIX(io->dweight, d->outs, d->ins, d->gw_dtype, false);
    if (!aligned_to(io->dbias, type_bytes(d->gb_dtype))) return TSR_ERR_ALIGNMENT;
    const bool f32 = d->dtype == TSR_F32;
    const int64_t T = d->rows, I = d->ins, O = d->outs;
    const int known = device_sms(), sms = known ? known : 148;

    // dz, and the partial sums of its columns (see the kernel): what is resident at once, 32 rows each at least
    const bool make_dz = (d->activation != TSR_ACT_NONE || drop.threshold || f32) && (dx || dw) && T > 0 && O > 0;      // (FP32: dz in planes)
    const int64_t col_blocks = (O + DZ_COLS - 1) / DZ_COLS;
    const int64_t most = col_blocks ? std::max<int64_t>(1, T <= 64 ? 1 : std::min<int64_t>((T + 31) / 32, DZ_CTAS * sms / col_blocks)) : 1;
    const int64_t rows_per = T ? round_up((T + most - 1) / most, 8) : 8;
    const int64_t parts = std::max<int64_t>(1, (T + rows_per - 1) / rows_per);

    const float scale = d->activation == TSR_ACT_NONE && drop.threshold ? drop.scale : 1.f;      // applied behind the products and the sums
    tsr_matrix dz = io->dy;
    Product px = {}, pw = {};
    size_t total = 0;
    for (int pass = 0; pass < 2; ++pass) {
        const bool run = pass == 1;
        if (run) {
            if (need) { *need = total; return TSR_OK; }
            if (total && (!workspace || bytes < total)) return TSR_ERR_WORKSPACE;
            if (total && !aligned_to(workspace, 256)) return TSR_ERR_ALIGNMENT;
            if (!known) return TSR_ERR_CUDA;
        }
        Room room = {run ? (char *)workspace : nullptr, 0};
        if (make_dz) {
            dz.ld = round_up(O, 64);
            dz.data = room.take((size_t)T * dz.ld * (f32 ? 6 : 2));
        }
        const bool direct = parts == 1 && T > 0;      // a single range of rows: its sums are the result
        float *partial = db && !direct ? (float *)room.take((size_t)parts * O * 4) : nullptr;
        if (run && T > 0 && (make_dz || db)) {
            DzArgs a = {};
            a.dy = io->dy.data; a.lddy = io->dy.ld;
            a.pre = io->pre.data; a.ldpre = io->pre.ld;
            a.dz = make_dz ? dz.data : nullptr; a.lddz = dz.ld; a.plane = T * dz.ld;
            a.partial = partial;
            if (direct) { a.sums = io->dbias; a.sums_bf16 = d->gb_dtype == TSR_BF16; a.accumulate = d->accumulate; }
            a.rows = T; a.cols = (int)O; a.rows_per = (int)rows_per;
            a.drop = drop;
            if (d->activation == TSR_ACT_NONE) a.drop.scale = 1.f;
            a.sum_scale = scale;
            const dim3 grid((unsigned)col_blocks, (unsigned)parts);
            const cudaError_t rc = f32 ? dz_launch<float>(a, d->activation, grid, stream) : dz_launch<bf16>(a, d->activation, grid, stream);
            if (rc != cudaSuccess) return TSR_ERR_CUDA;
        }
        if (run && db && !direct && column_finish(partial, T ? (int)parts : 0, O, O, io->dbias, d->gb_dtype == TSR_BF16, nullptr, false, d->accumulate != 0, stream) != cudaSuccess) return TSR_ERR_CUDA;
        // FP32: planes of the other operands
        Operand dz_op = {dz.data, dz.ld, false, T * dz.ld}, w_op = {io->weight.data, io->weight.ld, true, 0}, x_op = {io->x.data, io->x.ld, true, 0};
        if (f32 && T > 0 && O > 0 && I > 0) {
            CopyJobs jobs = {};
            if (dx) three_planes(io->weight, O, I, true, &w_op, room, &jobs);
            if (dw) three_planes(io->x, T, I, true, &x_op, room, &jobs);
            if (run && copy_operands(linear_split_kernel, jobs, sms, stream) != cudaSuccess) return TSR_ERR_CUDA;
        }
        // the two products run one after the other: they share what is left of the workspace
        size_t after = room.at;
        if (dx) {
            px = {};
            px.M = T; px.N = I; px.K = O;
            px.f32 = px.out_f32 = f32;
            px.A = dz_op;
            px.B = w_op;
            px.e.scale = scale;
            px.e.out = io->dx.data; px.e.ldo = io->dx.ld;
            Room own = room;
            st = product(px, own, run, sms, stream);
            if (st != TSR_OK) return st;
            after = std::max(after, own.at);
        }
        if (dw) {
            pw = {};
            pw.M = O; pw.N = I; pw.K = T;
            pw.f32 = f32;
            pw.out_f32 = d->gw_dtype == TSR_F32;
            pw.A = dz_op;
            pw.A.mn = true;
            pw.B = x_op;
            pw.e.scale = scale;
            pw.e.out = io->dweight.data; pw.e.ldo = io->dweight.ld;
            if (d->accumulate) { pw.e.res = pw.e.out; pw.e.ldr = pw.e.ldo; }
            Room own = room;
            st = product(pw, own, run, sms, stream);
            if (st != TSR_OK) return st;
            after = std::max(after, own.at);
        }
        total = after;
    }
    return TSR_OK;
}

}  // namespace
}  // namespace tsr

using namespace tsr;

extern "C" tsr_status tsr_linear_forward_bytes(const tsr_linear_desc *desc, const tsr_linear_io *io, size_t *bytes)
{
    return bytes ? forward(desc, io, nullptr, 0, bytes, nullptr) : TSR_ERR_INVALID_ARG;
}
extern "C" tsr_status tsr_linear_forward(const tsr_linear_desc *desc, const tsr_linear_io *io, void *workspace, size_t workspace_bytes, void *stream)
{
    return forward(desc, io, workspace, workspace_bytes, nullptr, (cudaStream_t)stream);
}
extern "C" tsr_status tsr_linear_backward_bytes(const tsr_linear_desc *desc, const tsr_linear_grads *io, size_t *bytes)
{
    return bytes ? backward(desc, io, nullptr, 0, bytes, nullptr) : TSR_ERR_INVALID_ARG;
}
extern "C" tsr_status tsr_linear_backward(const tsr_linear_desc *desc, const tsr_linear_grads *io, void *workspace, size_t workspace_bytes, void *stream)
{
    return backward(desc, io, workspace, workspace_bytes, nullptr, (cudaStream_t)stream);
}
extern "C" tsr_status tsr_layer_poll_status(int32_t *status, void *stream)
{
    if (!status) return TSR_ERR_INVALID_ARG;
    int32_t linear = 0, norm = 0;
    if (linear_status_read(&linear, (cudaStream_t)stream) != cudaSuccess || norm_status_read(&norm, (cudaStream_t)stream) != cudaSuccess) return TSR_ERR_CUDA;
    *status = linear ? linear : norm;
    return TSR_OK;
}
