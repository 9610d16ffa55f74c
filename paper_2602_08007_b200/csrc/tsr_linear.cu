// Linear layer: host side of its products (operand preparation, choice of tiles, split of K) and the kernels around them.
// Formulas in tsr.h; the products themselves are in tsr_linear_gemm.cu.
//
//   linear_pack_kernel     BF16 operand whose pitch or address TMA does not take -> workspace with a 16-byte pitch (one pass over it)
//   linear_split_kernel    FP32 operand -> high and low TF32 planes, K-major (transposed where the product contracts over rows)
//   linear_dz_kernel       dz = dropout(dy) o act'(pre) and the column sums of dz (the bias's gradient), one pass over dy and pre
//   linear_finish_kernel   split K: slabs added in order, then the epilogue
//   column_finish_kernel   partial column sums added in order (bias, and the norm's weight and bias)
#include <math.h>

#include <algorithm>

#include "tsr_linear.cuh"

namespace tsr {

// ---- kernels ----------------------------------------------------------------------------------------------------------

// dst[r][0 .. cols) = src[r][..]; dst has a pitch of whole 16-byte units.  A thread writes one unit of eight entries.
__global__ void __launch_bounds__(256)
linear_pack_kernel(const bf16 *__restrict__ src, int64_t lds, bf16 *__restrict__ dst, int64_t ldd, int64_t rows, int cols, int units)
{
    pdl_trigger();
    pdl_wait();
    const int64_t total = rows * units;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
        const int64_t r = u / units;
        const int c = (int)(u - r * units) * 8;
        const bf16 *s = src + r * lds + c;
        uint32_t w[4];
        if (c + 8 <= cols) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (uint32_t)__bfloat16_as_ushort(s[2 * i]) | ((uint32_t)__bfloat16_as_ushort(s[2 * i + 1]) << 16);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = c + 2 * i < cols ? (uint32_t)__bfloat16_as_ushort(s[2 * i]) : 0u;
                if (c + 2 * i + 1 < cols) w[i] |= (uint32_t)__bfloat16_as_ushort(s[2 * i + 1]) << 16;
            }
        }
        *(uint4 *)(dst + r * ldd + c) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// x = high + low: high is x rounded to TF32 (10 stored mantissa bits, to nearest with ties away from zero), low the remainder, rounded
// the same way: together 2^-22 of x.  Values that would round to infinity keep their leading bits; an infinity or NaN has no remainder.
__device__ __forceinline__ float tf32_round(float x)
{
    const uint32_t b = __float_as_uint(x);
    const uint32_t r = (b + 0x1000u) & 0xffffe000u;
    const bool keep = (b & 0x7f800000u) == 0x7f800000u;               // infinity or NaN
    const bool over = (r & 0x7f800000u) == 0x7f800000u;
    return keep ? x : __uint_as_float(over ? (b & 0xffffe000u) : r);
}
__device__ __forceinline__ void tf32_split(float x, float &hi, float &lo)
{
    hi = tf32_round(x);
    lo = (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? 0.f : tf32_round(x - hi);
}

// src: rows x cols of a row-major FP32 matrix; dst: planes (high, then low) of `prow` rows each, pitch ldd.  TRANS: plane[c][r] = src[r][c].
template <bool TRANS>
__global__ void __launch_bounds__(256)
linear_split_kernel(const float *__restrict__ src, int64_t lds, float *__restrict__ dst, int64_t ldd, int64_t prow, int rows, int cols)
{
    __shared__ float tile[32][33];
    pdl_trigger();
    pdl_wait();
    const int tc = (cols + 31) / 32;
    const int64_t tiles = (int64_t)((rows + 31) / 32) * tc;
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int r0 = (int)(t / tc) * 32, c0 = (int)(t % tc) * 32;
#pragma unroll
        for (int i = y; i < 32; i += 8) {
            const int r = r0 + i, c = c0 + x;
            const float v = r < rows && c < cols ? src[(int64_t)r * lds + c] : 0.f;
            if (TRANS) tile[i][x] = v;
            else if (r < rows && c < cols) {
                float hi, lo;
                tf32_split(v, hi, lo);
                dst[(int64_t)r * ldd + c] = hi;
                dst[(prow + r) * ldd + c] = lo;
            }
        }
        if (TRANS) {
            __syncthreads();
#pragma unroll
            for (int i = y; i < 32; i += 8) {
                const int r = c0 + i, c = r0 + x;      // row and column of the planes
                if (r < cols && c < rows) {
                    float hi, lo;
                    tf32_split(tile[x][i], hi, lo);
                    dst[(int64_t)r * ldd + c] = hi;
                    dst[(prow + r) * ldd + c] = lo;
                }
            }
            __syncthreads();
        }
    }
}

// Slabs (rows x ld, FP32) of a split product, added in order, then the epilogue.  splits = 0: the sum is zero (K = 0).
struct FinishArgs {
    const float *slabs;
    int64_t slab_rows, ld;
    int32_t splits, M, N, out_f32;     // out_f32: type of out, residual and pre
    LinearEpilogue e;
};
__global__ void __launch_bounds__(256)
linear_finish_kernel(const FinishArgs a)
{
    pdl_trigger();
    pdl_wait();
    const LinearEpilogue &e = a.e;
    const bool b16 = !a.out_f32;
    const int units = (a.N + 3) / 4;
    const int64_t total = (int64_t)a.M * units;
    const uint32_t call_key = e.drop.threshold ? drop_call_key(e.drop) : 0u;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
        const int64_t r = u / units;
        const int c = (int)(u - r * units) * 4;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        const float *s = a.slabs + r * a.ld + c;
#pragma unroll 4
        for (int p = 0; p < a.splits; ++p) {
            const float4 x = *(const float4 *)(s + p * a.slab_rows * a.ld);
            v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
        }
        const DropRow key = e.drop.threshold ? drop_row_key(call_key, r) : DropRow{0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (c + j >= a.N) break;
            float z = v[j];
            if (e.bias) z += load_as(e.bias, c + j, e.bias_bf16);
            if (e.pre) store_as(e.pre, r * e.ldp + c + j, b16, z);
            z = act_value(e.act, z);
            if (e.drop.threshold) z = drop_entry(key, (uint32_t)(c + j), z, e.drop);
            if (e.res) z += load_as(e.res, r * e.ldr + c + j, b16);
            store_as(e.out, r * e.ldo + c + j, b16, z);
        }
    }
}

// dz and its column sums.  A CTA takes 256 columns and a range of rows; a lane eight columns (side by side where VEC: everything
// is in whole, aligned vectors; 32 apart otherwise), a warp every eighth row.  dz NULL: the sums alone.
struct DzArgs {
    const void *dy, *pre;
    void *dz;
    float *partial;            // [gridDim.y][ldp], NULL: no sums
    int64_t lddy, ldpre, lddz, ldp, rows;
    int32_t cols, rows_per, act;
    DropArgs drop;
};
template <typename T, bool VEC>
__global__ void __launch_bounds__(256)
linear_dz_kernel(const DzArgs a)
{
    __shared__ float sums[8][256];
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = blockIdx.x * 256 + (VEC ? lane * 8 : lane);
    const int64_t r0 = (int64_t)blockIdx.y * a.rows_per, r1 = min(a.rows, r0 + a.rows_per);
    const uint32_t call_key = a.drop.threshold ? drop_call_key(a.drop) : 0u;
    float acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    if (c0 < a.cols) {
#pragma unroll 2
        for (int64_t r = r0 + warp; r < r1; r += 8) {
            const T *dy = (const T *)a.dy + r * a.lddy + c0;
            const T *pre = (const T *)a.pre + r * a.ldpre + c0;
            float g[8], z[8];
            if (VEC) {
                load8(dy, g);
                if (a.act) load8(pre, z);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = c0 + 32 * j < a.cols ? load_f(dy + 32 * j) : 0.f;
                if (a.act) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) z[j] = c0 + 32 * j < a.cols ? load_f(pre + 32 * j) : 0.f;
                }
            }
            if (a.act) {
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] *= act_slope(a.act, z[j]);
            }
            if (a.drop.threshold) {      // last, as a selection: what fell is zero whatever pre holds
                const DropRow key = drop_row_key(call_key, r);
                if (VEC) {
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const uint32_t w = drop_word(key, (uint32_t)(c0 + j) >> 1);
                        g[j] = drop_lo(w, g[j], a.drop);
                        g[j + 1] = drop_hi(w, g[j + 1], a.drop);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] = drop_entry(key, (uint32_t)(c0 + 32 * j), g[j], a.drop);
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += g[j];
            if (a.dz) {
                T *dz = (T *)a.dz + r * a.lddz + c0;
                if (VEC) store8(dz, g);
                else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) if (c0 + 32 * j < a.cols) store_f(dz + 32 * j, g[j]);
                }
            }
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[warp][VEC ? lane * 8 + j : lane + 32 * j] = acc[j];
    __syncthreads();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < a.cols) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += sums[w][threadIdx.x];
        a.partial[blockIdx.y * a.ldp + c] = s;
    }
}

// 32 columns per CTA; warp w adds rows w, w + 32, ..., then one warp adds the 32 sums: the order depends on `parts` alone.
__global__ void __launch_bounds__(1024)
column_finish_kernel(const float *__restrict__ partial, int parts, int64_t ldp, int64_t cols, void *out, int out_bf16, void *out2, int out2_bf16, int accumulate)
{
    __shared__ float sums[32][33];
    pdl_trigger();
    pdl_wait();
    if (blockIdx.y) { partial += parts * ldp; out = out2; out_bf16 = out2_bf16; }
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + x;
    float s = 0.f;
    if (c < cols) {
#pragma unroll 4
        for (int p = y; p < parts; p += 32) s += partial[p * ldp + c];
    }
    sums[y][x] = s;
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
    out->seed_key = mix32((uint32_t)d.seed ^ mix32((uint32_t)(d.seed >> 32) + 0x9e3779b9u));
    out->offset = d.offset;
    out->step = d.step;
    return true;
}

cudaError_t column_finish(const float *partial, int parts, int64_t ldp, int64_t cols, void *out, bool out_bf16, void *out2, bool out2_bf16,
                          bool accumulate, cudaStream_t stream)
{
    if (cols <= 0) return cudaSuccess;
    const dim3 grid((unsigned)((cols + 31) / 32), out2 ? 2 : 1);
    return launch_dependent(column_finish_kernel, grid, dim3(1024), 0, stream, 1, partial, parts, ldp, cols, out, (int)out_bf16, out2, (int)out2_bf16, (int)accumulate);
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

// Row-major matrix, boxes of 128 bytes x box_rows with the 128-byte swizzle.
bool encode(CUtensorMap *out, const void *base, int64_t rows, int64_t cols, int64_t ld, bool f32, int box_rows)
{
    EncodeTiledFn fn = encoder();
    if (!fn) return false;
    const int es = f32 ? 4 : 2;
    if (rows <= 1) ld = round_up(cols, 16 / es);         // a single row has no pitch
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * es};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / es), (cuuint32_t)box_rows}, step[2] = {1, 1};
    return fn(out, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides, box, step,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool tma_takes(const void *p, int64_t rows, int64_t ld, int es) { return aligned_to(p, 16) && (rows <= 1 || (ld * es) % 16 == 0); }

struct Operand { const void *p; int64_t ld; bool mn; };   // [rows x K], or (mn) stored as [K x rows]

struct Product {
    int64_t M, N, K;
    bool f32;            // operands
    Operand A, B;
    bool out_f32;
    LinearEpilogue e;    // out, res, pre, bias with their pitches
};

struct Shape { int cg, width, splits, kb_per, kb_total; int64_t m_tiles, n_tiles; };

// Tile shape and split of K by a model in SM clocks.  A K block of 128 bytes costs the MMAs 2 width clocks (6 x as much
// for the three FP32 products), and the SM's intake of 64 bytes a clock its share of the operands; a wave of tiles costs that
// times the blocks of a split; a split pays for its slabs (about 3000 bytes a clock over all SMs) and for another launch.
Shape choose(const Product &p, int sms)
{
    Shape best = {};
    double best_cost = 1e300;
    const int bk = p.f32 ? 32 : 64;
    const int kb = (int)((p.K + bk - 1) / bk);
    static const struct { int cg, width; } kinds[] = {{2, 256}, {2, 192}, {2, 128}, {2, 64}, {1, 128}, {1, 64}};
    for (const auto &k : kinds) {
        const int64_t mt = (p.M + 128 * k.cg - 1) / (128 * k.cg), nt = (p.N + k.width - 1) / k.width;
        const int slots = sms / k.cg;
        const double mma = (p.f32 ? 6.0 : 2.0) * k.width, intake = (p.f32 ? 2.0 : 1.0) * 2.0 * (128 + k.width / k.cg);
        const double per_kb = std::max(mma, intake);
        const int most = (int)std::min<int64_t>(std::max(1, kb / 2), std::max<int64_t>(1, 2 * slots / std::max<int64_t>(1, mt * nt)));
        for (int want = 1; want <= most; ++want) {
            const int per = (kb + want - 1) / want, s = (kb + per - 1) / per;
            if (s != want) continue;
            const double waves = (double)((mt * nt * s + slots - 1) / slots);
            double cost = 3000.0 + waves * (per * per_kb + 300.0) + 12.0 * k.width;
            if (s > 1) cost += 5000.0 + (double)s * (double)p.M * (double)p.N * 8.0 / 3000.0;
            if (cost < best_cost) { best_cost = cost; best = {k.cg, k.width, s, per, kb, mt, nt}; }
        }
    }
    return best;
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

// The product's scratch, and (run) its launches.  Slabs come last, so that two products after one another can share `room` from there on.
tsr_status product(const Product &p, Room &room, bool run, int sms, cudaStream_t stream)
{
    if (p.M == 0 || p.N == 0) return TSR_OK;
    FinishArgs f = {};
    f.M = (int)p.M; f.N = (int)p.N; f.out_f32 = p.out_f32;
    f.e = p.e;
    auto finish = [&]() -> tsr_status {
        const int64_t units = p.M * ((p.N + 3) / 4);
        const unsigned blocks = (unsigned)std::min<int64_t>((units + 255) / 256, (int64_t)sms * 16);
        return launch_dependent(linear_finish_kernel, dim3(blocks), dim3(256), 0, stream, 1, f) == cudaSuccess ? TSR_OK : TSR_ERR_CUDA;
    };
    if (p.K == 0) return run ? finish() : TSR_OK;

    const Shape s = choose(p, sms);
    if (s.m_tiles * s.n_tiles * s.splits > (int64_t)1 << 30) return TSR_ERR_SHAPE;
    const int es = p.f32 ? 4 : 2;
    LinearGemm g = {};
    g.M = (int)p.M; g.N = (int)p.N;
    g.kb_total = s.kb_total; g.kb_per = s.kb_per;
    g.width = s.width; g.m_tiles = (int)s.m_tiles; g.n_tiles = (int)s.n_tiles; g.tiles = (int)(s.m_tiles * s.n_tiles * s.splits);

    // operands
    const Operand *op[2] = {&p.A, &p.B};
    const int64_t extent[2] = {p.M, p.N};
    const int kbox[2] = {128, s.width / s.cg};            // rows of a K-major box
    for (int i = 0; i < 2; ++i) {
        const Operand &o = *op[i];
        const int64_t rows = o.mn ? p.K : extent[i], cols = o.mn ? extent[i] : p.K;    // as stored
        CUtensorMap *map = i ? &g.tmB : &g.tmA;
        if (p.f32) {
            const int64_t ld = round_up(p.K, 4);
            float *planes = (float *)room.take((size_t)2 * extent[i] * ld * 4);
            if (run) {
                const int64_t tiles = ((rows + 31) / 32) * ((cols + 31) / 32);
                const dim3 grid((unsigned)std::min<int64_t>(tiles, (int64_t)sms * 32));
                const cudaError_t rc = o.mn ? launch_dependent(linear_split_kernel<true>, grid, dim3(256), 0, stream, 1, (const float *)o.p, o.ld, planes, ld, extent[i], (int)rows, (int)cols)
                                            : launch_dependent(linear_split_kernel<false>, grid, dim3(256), 0, stream, 1, (const float *)o.p, o.ld, planes, ld, extent[i], (int)rows, (int)cols);
                if (rc != cudaSuccess) return TSR_ERR_CUDA;
                if (!encode(map, planes, 2 * extent[i], p.K, ld, true, kbox[i])) return TSR_ERR_CUDA;
            }
            (i ? g.b_plane_rows : g.a_plane_rows) = (int)extent[i];
            continue;
        }
        const void *at = o.p;
        int64_t ld = o.ld;
        if (!tma_takes(o.p, rows, o.ld, es)) {
            ld = round_up(cols, 8);
            bf16 *packed = (bf16 *)room.take((size_t)rows * ld * 2);
            if (run) {
                const int units = (int)(ld / 8);
                const dim3 grid((unsigned)std::min<int64_t>((rows * units + 255) / 256, (int64_t)sms * 32));
                if (launch_dependent(linear_pack_kernel, grid, dim3(256), 0, stream, 1, (const bf16 *)o.p, o.ld, packed, ld, rows, (int)cols, units) != cudaSuccess) return TSR_ERR_CUDA;
            }
            at = packed;
        }
        if (run && !encode(map, at, rows, cols, ld, false, o.mn ? 64 : kbox[i])) return TSR_ERR_CUDA;
        (i ? g.b_mn : g.a_mn) = o.mn;
    }
    const int planes = p.f32 ? 2 : 1;
    g.b_boxes = (s.width / s.cg + 63) / 64;
    g.stage_tx = (uint32_t)(s.cg * planes * 128 * 128 + (g.b_mn ? s.cg * g.b_boxes * 8192 : planes * s.width * 128));

    if (s.splits > 1) {
        f.slab_rows = round_up(p.M, 32);
        f.ld = round_up(p.N, 4);
        f.splits = s.splits;
        float *slabs = (float *)room.take((size_t)s.splits * f.slab_rows * f.ld * 4);
        if (!run) return TSR_OK;
        f.slabs = slabs;
        g.slab_rows = (int)f.slab_rows;
        g.whole_edge = 1;
        g.e.out = slabs; g.e.ldo = f.ld; g.e.out_tma = 1;
        if (!encode(&g.tmOut, slabs, s.splits * f.slab_rows, p.N, f.ld, true, 32)) return TSR_ERR_CUDA;
        if (linear_gemm_launch(g, s.cg, p.f32, true, sms, stream) != cudaSuccess) return TSR_ERR_CUDA;
        return finish();
    }
    if (!run) return TSR_OK;
    g.e = p.e;
    const int os = p.out_f32 ? 4 : 2;
    g.whole_edge = p.N * os % 16 == 0;
    g.e.out_tma = tma_takes(p.e.out, p.M, p.e.ldo, os);
    if (g.e.out_tma && !encode(&g.tmOut, p.e.out, p.M, p.N, p.e.ldo, p.out_f32, 32)) return TSR_ERR_CUDA;
    g.e.res_tma = p.e.res && tma_takes(p.e.res, p.M, p.e.ldr, os);
    if (g.e.res_tma && !encode(&g.tmRes, p.e.res, p.M, p.N, p.e.ldr, p.out_f32, 32)) return TSR_ERR_CUDA;
    g.e.pre_tma = p.e.pre && tma_takes(p.e.pre, p.M, p.e.ldp, os);
    if (g.e.pre_tma && !encode(&g.tmPre, p.e.pre, p.M, p.N, p.e.ldp, p.out_f32, 32)) return TSR_ERR_CUDA;
    return linear_gemm_launch(g, s.cg, p.f32, p.out_f32, sms, stream) == cudaSuccess ? TSR_OK : TSR_ERR_CUDA;
}

constexpr int64_t MOST = 0x7fffffff - 1023;

tsr_status check_desc(const tsr_linear_desc &d, DropArgs *drop)
{
    if (!type_ok(d.dtype) || !type_ok(d.b_dtype) || !type_ok(d.gw_dtype) || !type_ok(d.gb_dtype)) return TSR_ERR_UNSUPPORTED;
    if (d.activation < TSR_ACT_NONE || d.activation > TSR_ACT_SILU) return TSR_ERR_UNSUPPORTED;
    if (d.rows < 0 || d.ins < 0 || d.outs < 0 || d.rows > MOST || d.ins > MOST || d.outs > MOST) return TSR_ERR_SHAPE;
    // two FP32 planes of an operand, or the slabs of a split, are addressed by 32-bit row numbers
    if (d.dtype == TSR_F32 && (d.rows > MOST / 2 || d.ins > MOST / 2 || d.outs > MOST / 2)) return TSR_ERR_SHAPE;
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
    p.A = {io->x.data, io->x.ld, false};
    p.B = {io->weight.data, io->weight.ld, false};
    p.e.out = io->y.data; p.e.ldo = io->y.ld;
    p.e.res = io->residual.data; p.e.ldr = io->residual.ld;
    p.e.pre = io->pre.data; p.e.ldp = io->pre.ld;
    p.e.bias = io->bias; p.e.bias_bf16 = d->b_dtype == TSR_BF16;
    p.e.act = d->activation;
    const int sms = device_sms();
    Room count = {nullptr, 0};
    st = product(p, count, false, sms ? sms : 148, stream);
    if (st != TSR_OK) return st;
    if (need) { *need = count.at; return TSR_OK; }
    if (count.at && (!workspace || bytes < count.at)) return TSR_ERR_WORKSPACE;
    if (count.at && !aligned_to(workspace, 256)) return TSR_ERR_ALIGNMENT;
    if (p.M == 0 || p.N == 0) return TSR_OK;
    if (!sms) return TSR_ERR_CUDA;
    Room room = {(char *)workspace, 0};
    return product(p, room, true, sms, stream);
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

    // dz, and the partial sums of its columns: enough CTAs to fill the GPU four times, 32 rows each at least
    const bool make_dz = (d->activation != TSR_ACT_NONE || drop.threshold) && (dx || dw) && T > 0 && O > 0;
    const int64_t col_blocks = (O + DZ_COLS - 1) / DZ_COLS;
    int64_t parts = col_blocks ? std::max<int64_t>(1, std::min<int64_t>((T + 31) / 32, (4 * sms + col_blocks - 1) / col_blocks)) : 1;
    const int64_t rows_per = T ? round_up((T + parts - 1) / parts, 8) : 8;
    parts = std::max<int64_t>(1, (T + rows_per - 1) / rows_per);

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
            dz.ld = round_up(O, 16 / (f32 ? 4 : 2));
            dz.data = room.take((size_t)T * dz.ld * (f32 ? 4 : 2));
        }
        float *partial = db ? (float *)room.take((size_t)parts * O * 4) : nullptr;
        if (run && T > 0 && (make_dz || db)) {
            DzArgs a = {};
            a.dy = io->dy.data; a.lddy = io->dy.ld;
            a.pre = io->pre.data; a.ldpre = io->pre.ld;
            a.dz = make_dz ? dz.data : nullptr; a.lddz = dz.ld;
            a.partial = partial; a.ldp = O;
            a.rows = T; a.cols = (int)O; a.rows_per = (int)rows_per; a.act = d->activation;
            a.drop = drop;
            const int es = f32 ? 4 : 2;
            bool vec = O % 8 == 0 && aligned_to(a.dy, 16) && (a.lddy * es) % 16 == 0;
            if (d->activation) vec = vec && aligned_to(a.pre, 16) && (a.ldpre * es) % 16 == 0;
            const dim3 grid((unsigned)col_blocks, (unsigned)parts);
            cudaError_t rc;
            if (f32) rc = vec ? launch_dependent(linear_dz_kernel<float, true>, grid, dim3(256), 0, stream, 1, a) : launch_dependent(linear_dz_kernel<float, false>, grid, dim3(256), 0, stream, 1, a);
            else rc = vec ? launch_dependent(linear_dz_kernel<bf16, true>, grid, dim3(256), 0, stream, 1, a) : launch_dependent(linear_dz_kernel<bf16, false>, grid, dim3(256), 0, stream, 1, a);
            if (rc != cudaSuccess) return TSR_ERR_CUDA;
        }
        if (run && db && column_finish(partial, T ? (int)parts : 0, O, O, io->dbias, d->gb_dtype == TSR_BF16, nullptr, false, d->accumulate != 0, stream) != cudaSuccess) return TSR_ERR_CUDA;
        // the two products run one after the other: they share what is left of the workspace
        size_t after = room.at;
        if (dx) {
            px = {};
            px.M = T; px.N = I; px.K = O;
            px.f32 = px.out_f32 = f32;
            px.A = {dz.data, dz.ld, false};
            px.B = {io->weight.data, io->weight.ld, true};
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
            pw.A = {dz.data, dz.ld, true};
            pw.B = {io->x.data, io->x.ld, true};
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
    return layer_status_read(status, (cudaStream_t)stream) == cudaSuccess ? TSR_OK : TSR_ERR_CUDA;
}
