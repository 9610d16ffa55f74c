// Dense parameters through a kept plan: AdamW over many tensors with FP32 or 8-bit states, the global gradient norm with
// its clipping factor, and the conversion of states (Section 3.4, "in dense form"; formulas in tsr.h).
//
// Everything here streams: a step reads parameter, gradient and moments once and writes parameter and moments once, so
// HBM bounds it (bytes per element: FP32 state 16, 8-bit state 4 + 16/256, plus the parameter twice and the gradient).
// Work is laid out in UNITS of 256 consecutive elements of one tensor, one warp each -- the block of the 8-bit state, so
// that a block's maximum is one warp reduction -- and CHUNKS of units, one CTA each, listed in a table.
#include <cuda_fp8.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <stdarg.h>
#include <stdio.h>

#include "tsr_device.cuh"
#include "tsr_internal.h"
#include "tsr_pdl.cuh"

namespace tsr {

constexpr int UNIT = TSR_DENSE_BLOCK;      // elements of a warp's piece of work
static_assert(UNIT == 32 * 8, "a lane holds eight elements of a unit");
constexpr int WARPS = 8;                   // per CTA
constexpr int UNITS_PER_WARP = 2;
constexpr int CHUNK = UNIT * WARPS * UNITS_PER_WARP;
constexpr int NORM_CTAS = 1184;            // most CTAs of a norm launch (8 on each of 148 SMs)

enum DenseRecFlags : uint32_t {
    REC_VEC = 1,         // all that a step touches can be read in vectors of eight elements
    REC_VEC_STATE = 2,   // the moments can
    REC_VEC_GRAD = 4,    // the gradient can
    REC_PITCHED = 8,     // rows that do not follow one another directly
    REC_Q8 = 16,
    REC_G_BF16 = 32,
};

struct alignas(16) DenseRec {   // one tensor on the device
    void *p;
    const void *g;
    void *m, *v;
    float2 *scale;
    bf16 *image;
    int64_t n, cols, ldp, ldg, ldi;
    float lr_mult, wd_mult;
    uint32_t flags;
    int32_t index;              // position in the plan
};

struct DenseChunk { int32_t rec, at; };   // elements [at * CHUNK, (at + 1) * CHUNK) of a tensor

struct DenseStep {
    StepScalars sc;
    float lr, wd;
    float sqrt_inv_bc2;
    const float *grad_scale;
    uint32_t seed_key, step_lo;
};

// ---- vectors of eight elements ------------------------------------------------------------------------------------

struct Vec32 { uint32_t w[8]; };   // 32 bytes

__device__ __forceinline__ Vec32 load32(const void *p)
{
    Vec32 r;
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7])
                 : "l"(p) : "memory");
    return r;
}
__device__ __forceinline__ void store32(void *p, const Vec32 &r)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 :: "l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]), "r"(r.w[7]) : "memory");
}
__device__ __forceinline__ uint4 load16(const void *p)
{
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
    return r;
}
__device__ __forceinline__ uint2 load8(const void *p)
{
    uint2 r;
    asm volatile("ld.global.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p) : "memory");
    return r;
}

// Eight elements of type T as they lie in memory, and as FP32.
template <typename T> struct Eight;
template <> struct Eight<float> {
    Vec32 r;
    __device__ __forceinline__ void load(const float *p) { r = load32(p); }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(r.w[j]);
    }
    static __device__ __forceinline__ void put(float *p, const float (&x)[8])
    {
        Vec32 r;
#pragma unroll
        for (int j = 0; j < 8; ++j) r.w[j] = __float_as_uint(x[j]);
        store32(p, r);
    }
};
template <> struct Eight<bf16> {
    uint4 r;
    __device__ __forceinline__ void load(const bf16 *p) { r = load16(p); }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = __uint_as_float(w[j] << 16);
            x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void put(bf16 *p, const float (&x)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
            w[j] = *(const uint32_t *)&b;
        }
        *(uint4 *)p = make_uint4(w[0], w[1], w[2], w[3]);
    }
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float &d, float x) { d = x; }
__device__ __forceinline__ void from_f32(bf16 &d, float x) { d = __float2bfloat16_rn(x); }

// ---- 8-bit values ---------------------------------------------------------------------------------------------------

__device__ __forceinline__ void e4m3_unpack(uint2 c, float (&x)[8])
{
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[j >> 1] >> (16 * (j & 1))), __NV_E4M3);
        const float2 f = __half22float2(__half2(h));
        x[2 * j] = f.x;
        x[2 * j + 1] = f.y;
    }
}

__device__ __forceinline__ uint2 e4m3_pack(const float (&x)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = __nv_cvt_float2_to_fp8x2(make_float2(x[2 * j], x[2 * j + 1]), __NV_SATFINITE, __NV_E4M3);
    return make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
}

// The smallest power of two S >= 2^-126 with absmax <= 448 S = 1.75 * 2^8 S, and 1 / S, from the bits of absmax: adding
// 0x1fffff carries into the exponent exactly where the mantissa is above 1.75.  NaN where absmax is not finite.
__device__ __forceinline__ void block_scale(uint32_t absmax_bits, float &scale, float &inv)
{
    if (absmax_bits >= 0x7f800000u) {
        scale = inv = __uint_as_float(0x7fc00000u);
        return;
    }
    const int e = max((int)((absmax_bits + 0x1fffffu) >> 23) - 135, -126);
    scale = __uint_as_float((uint32_t)(e + 127) << 23);
    inv = __uint_as_float((uint32_t)(127 - e) << 23);
}

// Random words: 32-bit multiply-xorshift mixing of (element + key1), with a second key between the two multiplications
// so that the words of two tensors or steps are not shifted copies of one sequence.  The multipliers are those of the
// 32-bit finaliser of MurmurHash3 (A. Appleby, public domain).
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x)
{
    x ^= x >> 16; x *= 0x85ebca6bu; x ^= x >> 13; x *= 0xc2b2ae35u; return x ^ (x >> 16);
}
__device__ __forceinline__ uint32_t random_word(uint32_t counter, uint32_t key1, uint32_t key2)
{
    uint32_t x = counter + key1;
    x ^= x >> 16;
    x *= 0x85ebca6bu;
    x = x ^ (x >> 13) ^ key2;
    x *= 0xc2b2ae35u;
    return x ^ (x >> 16);
}

// |y| <= 448 rounded to an E4M3 value, away from zero with probability (remainder / spacing): 16 random bits are added
// below the three mantissa bits and the rest is cut off.  Below 2^-6 the spacing is 2^-9 throughout; adding 2^-6 first
// puts such values where FP32 numbers with three mantissa bits have that spacing.
__device__ __forceinline__ float e4m3_stochastic(float y, uint32_t bits16)
{
    const float a = fabsf(y);
    const float c = a < 0x1p-6f ? 0x1p-6f : 0.f;
    const uint32_t z = __float_as_uint(__fadd_rn(a, c)) + (bits16 << 4);
    return copysignf(__fsub_rn(__uint_as_float(z & 0xfff00000u), c), y);
}

__device__ __forceinline__ float bf16_stochastic(float x, uint32_t bits16)
{
    uint32_t b = __float_as_uint(x);
    if ((b & 0x7f800000u) != 0x7f800000u) b += bits16;   // Inf and NaN stay what they are
    return __uint_as_float(b & 0xffff0000u);
}

// ---- one unit's arithmetic ------------------------------------------------------------------------------------------

struct UnitKeys { uint32_t k1, k2; };

// The update of one lane's eight elements.  On entry m, v are the held moments (8-bit state: m and r = sqrt(v)), on exit
// the new ones in FP32.  Every rounding of the 8-bit form is one IEEE operation, so its stored bits are well defined; the
// update itself takes the approximate quotient.
template <bool Q8>
__device__ __forceinline__ void update_eight(float (&p)[8], const float (&g)[8], float (&m)[8], float (&v)[8], const DenseStep &a, float lr, float decay)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float d;
        if constexpr (Q8) {
            m[j] = __fadd_rn(__fmul_rn(a.sc.beta1, m[j]), __fmul_rn(a.sc.omb1, g[j]));
            v[j] = __fsqrt_rn(__fadd_rn(__fmul_rn(a.sc.beta2, __fmul_rn(v[j], v[j])), __fmul_rn(a.sc.omb2, __fmul_rn(g[j], g[j]))));
            d = __fdividef(__fmul_rn(m[j], a.sc.inv_bc1), __fmaf_rn(v[j], a.sqrt_inv_bc2, a.sc.eps));
        } else {
            d = core_update_elem(g[j], m[j], v[j], a.sc);
        }
        p[j] = __fmaf_rn(-lr, d, __fmul_rn(decay, p[j]));
    }
}

// New scales of the warp's block, and its values scaled and (stochastic) rounded to E4M3 values; element(j) is the
// position of x[j] in the tensor.
template <bool SR, typename Elem>
__device__ __forceinline__ float2 quantise_eight(float (&m)[8], float (&r)[8], UnitKeys k, Elem element)
{
    uint32_t bm = 0, br = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        bm = max(bm, __float_as_uint(m[j]) & 0x7fffffffu);
        br = max(br, __float_as_uint(r[j]) & 0x7fffffffu);
    }
    bm = __reduce_max_sync(0xffffffffu, bm);
    br = __reduce_max_sync(0xffffffffu, br);
    float2 scale, inv;
    block_scale(bm, scale.x, inv.x);
    block_scale(br, scale.y, inv.y);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const bool some = r[j] > 0.f;
        m[j] = __fmul_rn(m[j], inv.x);
        r[j] = __fmul_rn(r[j], inv.y);
        if constexpr (SR) {
            const uint32_t w = random_word((uint32_t)element(j), k.k1, k.k2);
            m[j] = e4m3_stochastic(m[j], w & 0xffffu);
            r[j] = e4m3_stochastic(r[j], w >> 16);
        }
        if (some) r[j] = fmaxf(r[j], 0x1p-9f);
    }
    return scale;
}

// BF16 parameters, stochastic: one random word serves elements 2i and 2i + 1.
template <typename Elem>
__device__ __forceinline__ void round_params(float (&p)[8], UnitKeys k, Elem element)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int64_t e = element(j);
        const uint32_t w = random_word((uint32_t)(e >> 1), k.k1 ^ 0x5bd1e995u, k.k2);
        p[j] = bf16_stochastic(p[j], (e & 1) ? w >> 16 : w & 0xffffu);
    }
}

// Where elements base + lane + 32 j of a tensor lie: row and column of the first by one division, the others by steps.
struct Walk {
    int64_t row, col;
    const DenseRec &t;
    __device__ __forceinline__ Walk(const DenseRec &rec, int64_t e) : row(0), col(e), t(rec)
    {
        if (t.flags & REC_PITCHED) split(e);
    }
    __device__ __forceinline__ void split(int64_t e)
    {
        if ((uint64_t)e < 0x100000000ull && (uint64_t)t.cols < 0x100000000ull) {
            row = (uint32_t)e / (uint32_t)t.cols;
            col = (uint32_t)e - (uint32_t)row * (uint32_t)t.cols;
        } else {
            row = e / t.cols;
            col = e - row * t.cols;
        }
    }
    __device__ __forceinline__ void next()   // 32 elements on
    {
        col += 32;
        if ((t.flags & REC_PITCHED) && col >= t.cols) {
            if (t.cols >= 32) { col -= t.cols; ++row; } else split(row * t.cols + col);
        }
    }
    __device__ __forceinline__ int64_t at(int64_t ld) const { return row * ld + col; }
};

template <typename PT, typename GT, bool Q8, bool SR>
__global__ void __launch_bounds__(WARPS * 32)
dense_step_kernel(const DenseRec *__restrict__ recs, const DenseChunk *__restrict__ chunks, const DenseStep a)
{
    pdl_trigger();
    const DenseChunk ch = chunks[blockIdx.x];
    const DenseRec t = recs[ch.rec];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float lr = __fmul_rn(a.lr, t.lr_mult);
    const float decay = __fsub_rn(1.f, __fmul_rn(lr, __fmul_rn(a.wd, t.wd_mult)));
    UnitKeys key = {0, 0};
    if constexpr (SR) {
        key.k1 = mix32(a.seed_key ^ mix32(a.step_lo + 0x7f4a7c15u * (uint32_t)(t.index + 1)));
        key.k2 = mix32(key.k1 ^ 0xa511e9b3u);
    }
    pdl_wait();
    float gs = 1.f;
    if (a.grad_scale) {
        gs = *(const volatile float *)a.grad_scale;
        if (!isfinite(gs)) return;
    }
    PT *P = (PT *)t.p;
    const GT *G = (const GT *)t.g;
#pragma unroll 1
    for (int u = 0; u < UNITS_PER_WARP; ++u) {
        const int64_t base = (int64_t)ch.at * CHUNK + (u * WARPS + warp) * UNIT;
        if (base >= t.n) return;
        float p[8], g[8], m[8], v[8];
        float2 scale = make_float2(0.f, 0.f);
        if constexpr (Q8) scale = t.scale[base / UNIT];
        if ((t.flags & REC_VEC) && base + UNIT <= t.n) {
            const int64_t e = base + lane * 8;
            Walk w(t, e);
            Eight<PT> rp; rp.load(P + w.at(t.ldp));
            Eight<GT> rg; rg.load(G + w.at(t.ldg));
            if constexpr (Q8) {
                const uint2 cm = load8((const uint8_t *)t.m + e), cv = load8((const uint8_t *)t.v + e);
                e4m3_unpack(cm, m);
                e4m3_unpack(cv, v);
            } else {
                Eight<float> rm, rv;
                rm.load((const float *)t.m + e);
                rv.load((const float *)t.v + e);
                rm.get(m);
                rv.get(v);
            }
            rp.get(p);
            rg.get(g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                g[j] = __fmul_rn(g[j], gs);
                if constexpr (Q8) { m[j] *= scale.x; v[j] *= scale.y; }
            }
            update_eight<Q8>(p, g, m, v, a, lr, decay);
            auto element = [&](int j) { return e + j; };
            if constexpr (SR && sizeof(PT) == 2) round_params(p, key, element);
            Eight<PT>::put(P + w.at(t.ldp), p);
            if (sizeof(PT) == 4 && t.image) Eight<bf16>::put(t.image + w.at(t.ldi), p);
            if constexpr (Q8) {
                const float2 s = quantise_eight<SR>(m, v, key, element);
                *(uint2 *)((uint8_t *)t.m + e) = e4m3_pack(m);
                *(uint2 *)((uint8_t *)t.v + e) = e4m3_pack(v);
                if (lane == 0) t.scale[base / UNIT] = s;
            } else {
                Eight<float>::put((float *)t.m + e, m);
                Eight<float>::put((float *)t.v + e, v);
            }
        } else {
            // any alignment, any pitch, and the last unit of a tensor: element by element, 32 neighbours at a time
            auto element = [&](int j) { return base + lane + 32 * j; };
            Walk w(t, element(0));
            int64_t at_p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t e = element(j);
                p[j] = g[j] = m[j] = v[j] = 0.f;
                at_p[j] = 0;
                if (e < t.n) {
                    at_p[j] = w.at(t.ldp);
                    p[j] = to_f32(P[at_p[j]]);
                    g[j] = __fmul_rn(to_f32(G[w.at(t.ldg)]), gs);
                    if constexpr (Q8) {
                        m[j] = scale.x * __half2float(__half(__nv_cvt_fp8_to_halfraw(((const uint8_t *)t.m)[e], __NV_E4M3)));
                        v[j] = scale.y * __half2float(__half(__nv_cvt_fp8_to_halfraw(((const uint8_t *)t.v)[e], __NV_E4M3)));
                    } else {
                        m[j] = ((const float *)t.m)[e];
                        v[j] = ((const float *)t.v)[e];
                    }
                }
                w.next();
            }
            update_eight<Q8>(p, g, m, v, a, lr, decay);
            if constexpr (SR && sizeof(PT) == 2) round_params(p, key, element);
            float2 s = make_float2(0.f, 0.f);
            if constexpr (Q8) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (element(j) >= t.n) m[j] = v[j] = 0.f;   // (0 * NaN of a poisoned block)
                s = quantise_eight<SR>(m, v, key, element);
            }
            Walk wi(t, element(0));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t e = element(j);
                if (e < t.n) {
                    from_f32(P[at_p[j]], p[j]);
                    if (sizeof(PT) == 4 && t.image) from_f32(t.image[wi.at(t.ldi)], p[j]);
                    if constexpr (Q8) {
                        ((uint8_t *)t.m)[e] = __nv_cvt_float_to_fp8(m[j], __NV_SATFINITE, __NV_E4M3);
                        ((uint8_t *)t.v)[e] = __nv_cvt_float_to_fp8(v[j], __NV_SATFINITE, __NV_E4M3);
                    } else {
                        ((float *)t.m)[e] = m[j];
                        ((float *)t.v)[e] = v[j];
                    }
                }
                wi.next();
            }
            if (Q8 && lane == 0) t.scale[base / UNIT] = s;
        }
    }
}

// ---- norm -----------------------------------------------------------------------------------------------------------

// Sum of eight squares.  FP32 squares overflow above 1.8e19 and lose bits below 1e-19: where the FP32 sum is outside a
// range that rules both out, it is taken again in FP64 (the values are still in registers).
__device__ __forceinline__ double square_sum(const float (&g)[8])
{
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = __fmaf_rn(g[j], g[j], s);
    if (s >= 1e-25f && s <= 1e37f) return (double)s;
    double d = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) d += (double)g[j] * (double)g[j];
    return d;
}

__device__ __forceinline__ double cta_sum(double x, double *sh)   // valid in thread 0
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_down_sync(0xffffffffu, x, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
    __syncthreads();
    if (threadIdx.x == 0) {
        x = sh[0];
        for (int w = 1; w < WARPS; ++w) x += sh[w];
    }
    return x;
}

__global__ void __launch_bounds__(WARPS * 32)
dense_norm_kernel(const DenseRec *__restrict__ recs, const DenseChunk *__restrict__ chunks, int count, float max_norm,
                  double *partial, uint32_t *ticket, float *out)
{
    __shared__ double sh[WARPS];
    __shared__ bool last;
    pdl_trigger();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    double sum = 0.0;
    for (int c = blockIdx.x; c < count; c += gridDim.x) {
        const DenseChunk ch = chunks[c];
        const DenseRec &t = recs[ch.rec];
#pragma unroll 1
        for (int u = 0; u < UNITS_PER_WARP; ++u) {
            const int64_t base = (int64_t)ch.at * CHUNK + (u * WARPS + warp) * UNIT;
            if (base >= t.n) break;
            float g[8];
            if ((t.flags & REC_VEC_GRAD) && base + UNIT <= t.n) {
                const Walk w(t, base + lane * 8);
                if (t.flags & REC_G_BF16) {
                    Eight<bf16> r; r.load((const bf16 *)t.g + w.at(t.ldg)); r.get(g);
                } else {
                    Eight<float> r; r.load((const float *)t.g + w.at(t.ldg)); r.get(g);
                }
            } else {
                Walk w(t, base + lane);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    g[j] = 0.f;
                    if (base + lane + 32 * j < t.n)
                        g[j] = (t.flags & REC_G_BF16) ? to_f32(((const bf16 *)t.g)[w.at(t.ldg)]) : ((const float *)t.g)[w.at(t.ldg)];
                    w.next();
                }
            }
            sum += square_sum(g);
        }
    }
    sum = cta_sum(sum, sh);
    if (threadIdx.x == 0) {
        partial[blockIdx.x] = sum;
        __threadfence();
        last = atomicInc(ticket, gridDim.x - 1) == gridDim.x - 1;   // wraps to 0: ready for the next launch
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum = 0.0;
    for (int c = threadIdx.x; c < (int)gridDim.x; c += WARPS * 32) sum += *(volatile double *)(partial + c);
    __syncthreads();
    sum = cta_sum(sum, sh);
    if (threadIdx.x == 0) {
        const float norm = (float)sqrt(sum);
        out[0] = norm;
        out[1] = isfinite(norm) ? (float)fmin(1.0, (double)max_norm / ((double)norm + 1e-6)) : __uint_as_float(0x7fc00000u);
    }
}

// ---- conversion -----------------------------------------------------------------------------------------------------

__global__ void __launch_bounds__(WARPS * 32)
dense_copy_state_kernel(const DenseRec *__restrict__ drecs, const DenseRec *__restrict__ srecs, const DenseChunk *__restrict__ chunks)
{
    pdl_trigger();
    const DenseChunk ch = chunks[blockIdx.x];
    const DenseRec &d = drecs[ch.rec];
    const DenseRec &s = srecs[ch.rec];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();
    const bool dq = d.flags & REC_Q8, sq = s.flags & REC_Q8;
#pragma unroll 1
    for (int u = 0; u < UNITS_PER_WARP; ++u) {
        const int64_t base = (int64_t)ch.at * CHUNK + (u * WARPS + warp) * UNIT;
        if (base >= d.n) return;
        const bool vec = (d.flags & s.flags & REC_VEC_STATE) && base + UNIT <= d.n;
        float m[8], v[8];
        auto element = [&](int j) { return vec ? base + lane * 8 + j : base + lane + 32 * j; };
        float2 scale = make_float2(1.f, 1.f);
        if (sq) scale = s.scale[base / UNIT];
        if (vec && sq) {
            e4m3_unpack(load8((const uint8_t *)s.m + element(0)), m);
            e4m3_unpack(load8((const uint8_t *)s.v + element(0)), v);
        } else if (vec) {
            Eight<float> r;
            r.load((const float *)s.m + element(0)); r.get(m);
            r.load((const float *)s.v + element(0)); r.get(v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t e = element(j);
                m[j] = v[j] = 0.f;
                if (e < d.n) {
                    m[j] = sq ? __half2float(__half(__nv_cvt_fp8_to_halfraw(((const uint8_t *)s.m)[e], __NV_E4M3))) : ((const float *)s.m)[e];
                    v[j] = sq ? __half2float(__half(__nv_cvt_fp8_to_halfraw(((const uint8_t *)s.v)[e], __NV_E4M3))) : ((const float *)s.v)[e];
                }
            }
        }
        float2 out_scale = scale;
        if (!dq && sq) {
#pragma unroll
            for (int j = 0; j < 8; ++j) { m[j] *= scale.x; v[j] *= scale.y; v[j] = __fmul_rn(v[j], v[j]); }
        } else if (dq && !sq) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __fsqrt_rn(v[j]);
            out_scale = quantise_eight<false>(m, v, UnitKeys{0, 0}, element);
        }
        if (vec && dq) {
            *(uint2 *)((uint8_t *)d.m + element(0)) = e4m3_pack(m);
            *(uint2 *)((uint8_t *)d.v + element(0)) = e4m3_pack(v);
        } else if (vec) {
            Eight<float>::put((float *)d.m + element(0), m);
            Eight<float>::put((float *)d.v + element(0), v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t e = element(j);
                if (e >= d.n) continue;
                if (dq) {
                    ((uint8_t *)d.m)[e] = __nv_cvt_float_to_fp8(m[j], __NV_SATFINITE, __NV_E4M3);
                    ((uint8_t *)d.v)[e] = __nv_cvt_float_to_fp8(v[j], __NV_SATFINITE, __NV_E4M3);
                } else {
                    ((float *)d.m)[e] = m[j];
                    ((float *)d.v)[e] = v[j];
                }
            }
        }
        if (dq && lane == 0) d.scale[base / UNIT] = out_scale;
    }
}

}  // namespace tsr

using namespace tsr;

// ---- host side ------------------------------------------------------------------------------------------------------

struct tsr_dense_plan {
    std::vector<tsr_dense_desc> descs;
    std::vector<DenseRec> recs;
    std::vector<DenseChunk> chunks;         // state-only tensors, then the stepped ones group by group, then norm-only ones
    struct Group { int key, first, count; };
    std::vector<Group> groups;              // chunks of tensors that share types: one launch each
    int step_first = 0, step_end = 0;
    size_t workspace_bytes = 0;
    bool bound = false;
    int device = -1, norm_ctas = 0;
    DenseRec *d_recs = nullptr;
    DenseChunk *d_chunks = nullptr;
    double *d_partial = nullptr;
    uint32_t *d_ticket = nullptr;
    mutable std::string err;
};

namespace {

tsr_status dense_fail(const tsr_dense_plan *plan, tsr_status s, const char *fmt, ...)
{
    if (plan) {
        char buf[256];
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(buf, sizeof buf, fmt, ap);
        va_end(ap);
        try { plan->err = buf; } catch (...) {}
    }
    return s;
}

#define DENSE_CUDA(plan, call)                                                                                  \
    do {                                                                                                        \
        cudaError_t e__ = (call);                                                                               \
        if (e__ != cudaSuccess) return dense_fail(plan, TSR_ERR_CUDA, "%s failed: %s", #call, cudaGetErrorString(e__)); \
    } while (0)

constexpr int64_t DENSE_MOST = (int64_t)1 << 40;   // elements of a tensor with its pitch; keeps products in 64 bits

enum { KEY_P_BF16 = 1, KEY_G_BF16 = 2, KEY_Q8 = 4, KEY_COUNT = 8 };

int key_of(const tsr_dense_desc &d)
{
    return (d.p_dtype == TSR_BF16 ? KEY_P_BF16 : 0) | (d.g_dtype == TSR_BF16 ? KEY_G_BF16 : 0) | (d.state == TSR_STATE_Q8 ? KEY_Q8 : 0);
}

template <bool SR>
cudaError_t step_launch(int key, const DenseRec *recs, const DenseChunk *chunks, int count, const DenseStep &a, cudaStream_t s)
{
    const dim3 grid(count), block(WARPS * 32);
    switch (key) {
    case 0: return launch_dependent(dense_step_kernel<float, float, false, SR>, grid, block, 0, s, 1, recs, chunks, a);
    case KEY_P_BF16: return launch_dependent(dense_step_kernel<bf16, float, false, SR>, grid, block, 0, s, 1, recs, chunks, a);
    case KEY_G_BF16: return launch_dependent(dense_step_kernel<float, bf16, false, SR>, grid, block, 0, s, 1, recs, chunks, a);
    case KEY_P_BF16 | KEY_G_BF16: return launch_dependent(dense_step_kernel<bf16, bf16, false, SR>, grid, block, 0, s, 1, recs, chunks, a);
    case KEY_Q8: return launch_dependent(dense_step_kernel<float, float, true, SR>, grid, block, 0, s, 1, recs, chunks, a);
    case KEY_Q8 | KEY_P_BF16: return launch_dependent(dense_step_kernel<bf16, float, true, SR>, grid, block, 0, s, 1, recs, chunks, a);
    case KEY_Q8 | KEY_G_BF16: return launch_dependent(dense_step_kernel<float, bf16, true, SR>, grid, block, 0, s, 1, recs, chunks, a);
    default: return launch_dependent(dense_step_kernel<bf16, bf16, true, SR>, grid, block, 0, s, 1, recs, chunks, a);
    }
}

tsr_status dense_ready(const tsr_dense_plan *plan)
{
    if (!plan->bound) return dense_fail(plan, TSR_ERR_NOT_BOUND, "tsr_dense_plan_bind has not been called");
    int dev = -1;
    DENSE_CUDA(plan, cudaGetDevice(&dev));
    if (dev != plan->device) return dense_fail(plan, TSR_ERR_INVALID_ARG, "the plan is bound on device %d, the current device is %d", plan->device, dev);
    return TSR_OK;
}

bool aligned(const void *p, int64_t bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }
int64_t size_of(int32_t dtype) { return dtype == TSR_BF16 ? 2 : 4; }

// A matrix whose lanes' vectors of eight elements each lie in one row, aligned to their size.
bool vector_rows(const void *p, int64_t es, int64_t rows, int64_t cols, int64_t ld)
{
    if (!aligned(p, 8 * es)) return false;
    return ld == cols || rows == 1 || (cols % 8 == 0 && ld % 8 == 0);
}

tsr_status dense_bind(tsr_dense_plan *plan, const tsr_dense_ptrs *ptrs, void *workspace)
{
    std::vector<DenseRec> recs(plan->descs.size());
    for (size_t i = 0; i < recs.size(); ++i) {
        const tsr_dense_desc &d = plan->descs[i];
        const tsr_dense_ptrs &p = ptrs[i];
        DenseRec &r = recs[i];
        memset(&r, 0, sizeof r);
        r.n = d.rows * d.cols;
        if (r.n == 0) continue;
        const bool grad = d.flags != TSR_DENSE_STATE_ONLY, state = d.flags != TSR_DENSE_NORM_ONLY, step = d.flags == 0;
        const int64_t ps = size_of(d.p_dtype), gs = size_of(d.g_dtype);
        const bool q8 = d.state == TSR_STATE_Q8;
        if ((grad && !p.grad) || (state && (!p.m || !p.v || (q8 && !p.scale))) || (step && !p.param))
            return dense_fail(plan, TSR_ERR_INVALID_ARG, "tensor %zu: NULL pointer", i);
        if ((grad && !aligned(p.grad, gs)) || (state && !q8 && (!aligned(p.m, 4) || !aligned(p.v, 4))) ||
            (state && q8 && !aligned(p.scale, 8)) || (step && (!aligned(p.param, ps) || !aligned(p.image, 2))))
            return dense_fail(plan, TSR_ERR_ALIGNMENT, "tensor %zu: a buffer is not aligned to its element type", i);
        if (step && p.image && d.p_dtype != TSR_F32)
            return dense_fail(plan, TSR_ERR_INVALID_ARG, "tensor %zu: an image needs an FP32 parameter", i);
        if (step && p.image && (d.ldi < d.cols || d.ldi > DENSE_MOST / d.rows)) return dense_fail(plan, TSR_ERR_SHAPE, "tensor %zu: bad ldi", i);
        r.cols = d.cols; r.ldp = d.ldp; r.ldg = d.ldg; r.ldi = d.ldi;
        r.lr_mult = d.lr_mult; r.wd_mult = d.wd_mult;
        r.index = (int32_t)i;
        if (q8) r.flags |= REC_Q8;
        if (d.g_dtype == TSR_BF16) r.flags |= REC_G_BF16;
        bool dense = true;
        if (grad) {
            r.g = p.grad;
            dense = dense && d.ldg == d.cols;
            if (vector_rows(p.grad, gs, d.rows, d.cols, d.ldg)) r.flags |= REC_VEC_GRAD;
        }
        if (state) {
            r.m = p.m; r.v = p.v;
            if (q8) r.scale = (float2 *)p.scale;
            if (aligned(p.m, q8 ? 8 : 32) && aligned(p.v, q8 ? 8 : 32)) r.flags |= REC_VEC_STATE;
        }
        if (step) {
            r.p = p.param;
            r.image = (bf16 *)p.image;
            dense = dense && d.ldp == d.cols && (!p.image || d.ldi == d.cols);
            if ((r.flags & REC_VEC_GRAD) && (r.flags & REC_VEC_STATE) && vector_rows(p.param, ps, d.rows, d.cols, d.ldp) &&
                (!p.image || vector_rows(p.image, 2, d.rows, d.cols, d.ldi)))
                r.flags |= REC_VEC;
        }
        if (!dense && d.rows > 1) {
            r.flags |= REC_PITCHED;
            // one pitched matrix among dense ones: vectors of the dense ones would cross its rows
            if (d.cols % 8 != 0) r.flags &= ~(uint32_t)(REC_VEC | REC_VEC_GRAD);
        }
    }
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return dense_fail(plan, TSR_ERR_CUDA, "no CUDA device available");
    DENSE_CUDA(plan, cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    plan->bound = false;
    DENSE_CUDA(plan, cudaDeviceSynchronize());   // nothing that still runs may see the tables change
    char *at = (char *)workspace;
    plan->d_recs = (DenseRec *)at;
    at += round_up((int64_t)(recs.size() * sizeof(DenseRec)), 256);
    plan->d_chunks = (DenseChunk *)at;
    at += round_up((int64_t)(plan->chunks.size() * sizeof(DenseChunk)), 256);
    plan->d_partial = (double *)at;
    at += NORM_CTAS * sizeof(double);
    plan->d_ticket = (uint32_t *)at;
    if (!recs.empty()) DENSE_CUDA(plan, cudaMemcpy(plan->d_recs, recs.data(), recs.size() * sizeof(DenseRec), cudaMemcpyHostToDevice));
    if (!plan->chunks.empty())
        DENSE_CUDA(plan, cudaMemcpy(plan->d_chunks, plan->chunks.data(), plan->chunks.size() * sizeof(DenseChunk), cudaMemcpyHostToDevice));
    DENSE_CUDA(plan, cudaMemset(plan->d_ticket, 0, sizeof(uint32_t)));
    DENSE_CUDA(plan, cudaDeviceSynchronize());
    plan->recs.swap(recs);
    plan->device = dev;
    plan->norm_ctas = std::min(NORM_CTAS, 8 * sms);
    plan->bound = true;
    return TSR_OK;
}

void dense_layout(tsr_dense_plan *plan, const tsr_dense_desc *descs, int32_t count)
{
    if (count > 0) plan->descs.assign(descs, descs + count);
    auto add = [&](int i) {
        const int64_t n = plan->descs[i].rows * plan->descs[i].cols;
        for (int64_t k = 0; k * CHUNK < n; ++k) plan->chunks.push_back({i, (int32_t)k});
    };
    for (int i = 0; i < count; ++i)
        if (plan->descs[i].flags == TSR_DENSE_STATE_ONLY) add(i);
    plan->step_first = (int)plan->chunks.size();
    for (int key = 0; key < KEY_COUNT; ++key) {
        const int first = (int)plan->chunks.size();
        for (int i = 0; i < count; ++i)
            if (plan->descs[i].flags == 0 && key_of(plan->descs[i]) == key) add(i);
        const int got = (int)plan->chunks.size() - first;
        if (got) plan->groups.push_back({key, first, got});
    }
    plan->step_end = (int)plan->chunks.size();
    for (int i = 0; i < count; ++i)
        if (plan->descs[i].flags == TSR_DENSE_NORM_ONLY) add(i);
    plan->workspace_bytes = (size_t)(round_up((int64_t)(plan->descs.size() * sizeof(DenseRec)), 256) +
                                     round_up((int64_t)(plan->chunks.size() * sizeof(DenseChunk)), 256) +
                                     NORM_CTAS * (int64_t)sizeof(double) + 256);
}

}  // namespace

extern "C" {

tsr_status tsr_dense_plan_create(tsr_dense_plan **out, const tsr_dense_desc *descs, int32_t count)
{
    if (!out) return TSR_ERR_INVALID_ARG;
    *out = nullptr;
    if (count < 0 || (count > 0 && !descs)) return TSR_ERR_INVALID_ARG;
    int64_t total = 0;   // chunks: the table's indices are 32-bit
    for (int i = 0; i < count; ++i) {
        const tsr_dense_desc &d = descs[i];
        if (d.rows < 0 || d.cols < 0) return TSR_ERR_SHAPE;
        if (d.flags != 0 && d.flags != TSR_DENSE_NORM_ONLY && d.flags != TSR_DENSE_STATE_ONLY) return TSR_ERR_INVALID_ARG;
        const bool grad = d.flags != TSR_DENSE_STATE_ONLY, state = d.flags != TSR_DENSE_NORM_ONLY, step = d.flags == 0;
        if ((grad && d.ldg < d.cols) || (step && d.ldp < d.cols)) return TSR_ERR_SHAPE;
        if (grad && d.g_dtype != TSR_F32 && d.g_dtype != TSR_BF16) return TSR_ERR_UNSUPPORTED;
        if (step && d.p_dtype != TSR_F32 && d.p_dtype != TSR_BF16) return TSR_ERR_UNSUPPORTED;
        if (state && d.state != TSR_STATE_F32 && d.state != TSR_STATE_Q8) return TSR_ERR_UNSUPPORTED;
        if (!isfinite(d.lr_mult) || !isfinite(d.wd_mult)) return TSR_ERR_INVALID_ARG;
        const int64_t most = DENSE_MOST;
        if (d.rows > 0 && d.cols > most / d.rows) return TSR_ERR_SHAPE;
        if (d.rows > 0 && ((grad && d.ldg > most / d.rows) || (step && d.ldp > most / d.rows))) return TSR_ERR_SHAPE;
        total += (d.rows * d.cols + CHUNK - 1) / CHUNK;
        if (total > 0x7fffffff) return TSR_ERR_SHAPE;
    }
    tsr_dense_plan *plan = new (std::nothrow) tsr_dense_plan;
    if (!plan) return TSR_ERR_INVALID_ARG;
    try {
        dense_layout(plan, descs, count);
    } catch (...) {   // the host is out of memory
        delete plan;
        return TSR_ERR_INVALID_ARG;
    }
    *out = plan;
    return TSR_OK;
}

tsr_status tsr_dense_plan_destroy(tsr_dense_plan *plan)
{
    if (!plan) return TSR_ERR_INVALID_ARG;
    delete plan;
    return TSR_OK;
}

const char *tsr_dense_plan_last_error(const tsr_dense_plan *plan) { return plan ? plan->err.c_str() : ""; }

tsr_status tsr_dense_plan_workspace_bytes(const tsr_dense_plan *plan, size_t *bytes)
{
    if (!plan || !bytes) return TSR_ERR_INVALID_ARG;
    *bytes = plan->workspace_bytes;
    return TSR_OK;
}

tsr_status tsr_dense_plan_bind(tsr_dense_plan *plan, const tsr_dense_ptrs *ptrs, int32_t count, void *workspace, size_t workspace_bytes)
{
    if (!plan) return TSR_ERR_INVALID_ARG;
    if (count != (int32_t)plan->descs.size() || (count > 0 && !ptrs)) return dense_fail(plan, TSR_ERR_INVALID_ARG, "ptrs/count mismatch");
    if (!workspace || workspace_bytes < plan->workspace_bytes)
        return dense_fail(plan, TSR_ERR_WORKSPACE, "workspace needs %zu bytes", plan->workspace_bytes);
    if (!aligned(workspace, 256)) return dense_fail(plan, TSR_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
    try {
        return dense_bind(plan, ptrs, workspace);
    } catch (...) {
        return dense_fail(plan, TSR_ERR_INVALID_ARG, "out of host memory");
    }
}

tsr_status tsr_dense_plan_step(tsr_dense_plan *plan, const tsr_hyper *h, const float *grad_scale, int32_t rounding, uint64_t seed, void *stream)
{
    if (!plan) return TSR_ERR_INVALID_ARG;
    if (!h) return dense_fail(plan, TSR_ERR_INVALID_ARG, "hyper is NULL");
    if (h->step < 1) return dense_fail(plan, TSR_ERR_INVALID_ARG, "hyper.step must be >= 1");
    if (h->rule != TSR_RULE_ADAM) return dense_fail(plan, TSR_ERR_INVALID_ARG, "dense parameters are stepped by TSR_RULE_ADAM only");
    if (!(h->beta1 >= 0.f && h->beta1 < 1.f) || !(h->beta2 >= 0.f && h->beta2 < 1.f))
        return dense_fail(plan, TSR_ERR_INVALID_ARG, "betas must lie in [0, 1)");
    if (rounding != TSR_ROUND_NEAREST && rounding != TSR_ROUND_STOCHASTIC) return dense_fail(plan, TSR_ERR_INVALID_ARG, "unknown rounding");
    if (!aligned(grad_scale, 4)) return dense_fail(plan, TSR_ERR_ALIGNMENT, "grad_scale is not aligned to a float");
    tsr_status st = dense_ready(plan);
    if (st != TSR_OK) return st;
    DenseStep a;
    memset(&a, 0, sizeof a);
    a.sc.beta1 = h->beta1; a.sc.beta2 = h->beta2; a.sc.eps = h->eps;
    a.sc.omb1 = (float)(1.0 - (double)h->beta1);
    a.sc.omb2 = (float)(1.0 - (double)h->beta2);
    const double ibc2 = 1.0 / (1.0 - pow((double)h->beta2, (double)h->step));
    a.sc.inv_bc1 = (float)(1.0 / (1.0 - pow((double)h->beta1, (double)h->step)));
    a.sc.inv_bc2 = (float)ibc2;
    a.sc.rule = TSR_RULE_ADAM;
    a.sqrt_inv_bc2 = (float)sqrt(ibc2);
    a.lr = h->lr;
    a.wd = h->weight_decay;
    a.grad_scale = grad_scale;
    a.seed_key = mix32((uint32_t)seed ^ mix32((uint32_t)(seed >> 32) + 0x9e3779b9u));
    a.step_lo = (uint32_t)h->step;
    for (const tsr_dense_plan::Group &g : plan->groups) {
        const DenseChunk *chunks = plan->d_chunks + g.first;
        const bool sr = rounding == TSR_ROUND_STOCHASTIC && (g.key & (KEY_Q8 | KEY_P_BF16));   // else nothing is rounded
        DENSE_CUDA(plan, sr ? step_launch<true>(g.key, plan->d_recs, chunks, g.count, a, (cudaStream_t)stream)
                            : step_launch<false>(g.key, plan->d_recs, chunks, g.count, a, (cudaStream_t)stream));
    }
    return TSR_OK;
}

tsr_status tsr_dense_plan_grad_norm(tsr_dense_plan *plan, float max_norm, float *out, void *stream)
{
    if (!plan) return TSR_ERR_INVALID_ARG;
    if (!out) return dense_fail(plan, TSR_ERR_INVALID_ARG, "out is NULL");
    if (!(max_norm > 0.f)) return dense_fail(plan, TSR_ERR_INVALID_ARG, "max_norm must be positive");
    if (!aligned(out, 4)) return dense_fail(plan, TSR_ERR_ALIGNMENT, "out is not aligned to a float");
    tsr_status st = dense_ready(plan);
    if (st != TSR_OK) return st;
    const int count = (int)plan->chunks.size() - plan->step_first;
    const int ctas = std::max(1, std::min(plan->norm_ctas, count));
    DENSE_CUDA(plan, launch_dependent(dense_norm_kernel, dim3(ctas), dim3(WARPS * 32), 0, (cudaStream_t)stream, 1,
                                      (const DenseRec *)plan->d_recs, (const DenseChunk *)plan->d_chunks + plan->step_first, count, max_norm,
                                      plan->d_partial, plan->d_ticket, out));
    return TSR_OK;
}

tsr_status tsr_dense_plan_copy_state(tsr_dense_plan *dst, const tsr_dense_plan *src, void *stream)
{
    if (!dst) return TSR_ERR_INVALID_ARG;
    if (!src) return dense_fail(dst, TSR_ERR_INVALID_ARG, "src is NULL");
    if (dst->descs.size() != src->descs.size()) return dense_fail(dst, TSR_ERR_SHAPE, "the plans list different numbers of tensors");
    for (size_t i = 0; i < dst->descs.size(); ++i) {
        const tsr_dense_desc &d = dst->descs[i], &s = src->descs[i];
        if (d.rows * d.cols != s.rows * s.cols || (d.flags == TSR_DENSE_NORM_ONLY) != (s.flags == TSR_DENSE_NORM_ONLY))
            return dense_fail(dst, TSR_ERR_SHAPE, "tensor %zu differs between the plans", i);
    }
    tsr_status st = dense_ready(dst);
    if (st != TSR_OK) return st;
    if (!src->bound) return dense_fail(dst, TSR_ERR_NOT_BOUND, "the source plan is not bound");
    if (src->device != dst->device) return dense_fail(dst, TSR_ERR_INVALID_ARG, "the plans are bound on different devices");
    if (dst == src || dst->step_end == 0) return TSR_OK;
    DENSE_CUDA(dst, launch_dependent(dense_copy_state_kernel, dim3(dst->step_end), dim3(WARPS * 32), 0, (cudaStream_t)stream, 1,
                                     (const DenseRec *)dst->d_recs, (const DenseRec *)src->d_recs, (const DenseChunk *)dst->d_chunks));
    return TSR_OK;
}

}  // extern "C"
