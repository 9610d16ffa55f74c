// Dense parameters through a kept plan: AdamW over many tensors with FP32 or 8-bit states, the global gradient norm with
// its clipping factor, and the conversion of states (Section 3.4, "in dense form"; formulas in tsr.h).
//
// Everything here streams: a step reads parameter, gradient and moments once and writes parameter and moments once, so
// HBM bounds it (bytes per element: FP32 state 16, 8-bit state 4 + 16/256, plus the parameter twice and the gradient).
// Work is laid out in UNITS of 256 consecutive elements of one tensor, one warp each -- the block of the 8-bit state, so
// that a block's maximum is one warp reduction -- and CHUNKS of up to 16 units per warp, one CTA each, listed in a table.
//
// Measured (B200, copy rate 6.53 TB/s; LLaMA-shaped sets, clipping factor on the device): FP32 state, 1B set with FP32 masters
// and BF16 gradients 4.81 ms (6.9 TB/s); 8-bit state, 130M set in BF16 0.169 to 0.182 ms (6.1 to 6.5 TB/s); stochastic, 1B set in
// BF16 2.55 to 2.66 ms (4.8 to 5.0 TB/s, bound by instruction issue); gradient norm of the 1B set 0.37 to 0.39 ms; state conversion
// of the 350M set 0.50 to 0.51 ms.  64 Mi elements, 8-bit state, BF16: 104 us to nearest, 131 stochastic; one element off the 16-byte
// grid 134 and 174.  Small calls take 2.1 us on the device.
#include <cuda_fp8.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <stdarg.h>
#include <stdio.h>

#include "tsr_dense_table.h"
#include "tsr_device.cuh"
#include "tsr_internal.h"
#include "tsr_pdl.cuh"

namespace tsr {

// CTAs on an SM of the kernels, whose registers are bounded for it.
constexpr int STEP_F32_CTAS = 4, STEP_Q8_CTAS = 3, COPY_CTAS = 5, NORM_CTAS = 4;
constexpr int SMS = 148;

enum DenseRecFlags : uint32_t {
    REC_VEC_STATE = 1,   // the moments can be read in vectors of eight elements
    REC_PAIR_STATE = 2,  // ... in pairs
    REC_PITCHED = 4,     // rows that do not follow one another directly
    REC_Q8 = 8,
    REC_G_BF16 = 16,
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

// Eight elements of type T as they lie in memory, and as FP32 pairs.
template <typename T> struct Eight;
template <> struct Eight<float> {
    Vec32 r;
    __device__ __forceinline__ void load(const float *p) { r = load32(p); }
    __device__ __forceinline__ void get(float2 (&x)[4]) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = make_float2(__uint_as_float(r.w[2 * j]), __uint_as_float(r.w[2 * j + 1]));
    }
    static __device__ __forceinline__ void put(float *p, const float2 (&x)[4])
    {
        Vec32 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) { r.w[2 * j] = __float_as_uint(x[j].x); r.w[2 * j + 1] = __float_as_uint(x[j].y); }
        store32(p, r);
    }
};
__device__ __forceinline__ uint4 bf16_pack(const float2 (&x)[4])
{
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(x[j].x, x[j].y);
        w[j] = *(const uint32_t *)&b;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <> struct Eight<bf16> {
    uint4 r;
    __device__ __forceinline__ void load(const bf16 *p) { r = load16(p); }
    __device__ __forceinline__ void get(float2 (&x)[4]) const
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
    }
    static __device__ __forceinline__ void put(bf16 *p, const float2 (&x)[4]) { *(uint4 *)p = bf16_pack(x); }
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float &d, float x) { d = x; }
__device__ __forceinline__ void from_f32(bf16 &d, float x) { d = __float2bfloat16_rn(x); }
__device__ __forceinline__ float &at(float2 (&x)[4], int j) { return (j & 1) ? x[j >> 1].y : x[j >> 1].x; }

// ---- 8-bit values ---------------------------------------------------------------------------------------------------

__device__ __forceinline__ void e4m3_unpack(uint2 c, float2 (&x)[4])
{
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        x[j] = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[j >> 1] >> (16 * (j & 1))), __NV_E4M3)));
}

__device__ __forceinline__ uint2 e4m3_pack(const float2 (&x)[4])
{
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = __nv_cvt_float2_to_fp8x2(x[j], __NV_SATFINITE, __NV_E4M3);
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
// The word before its last step x ^ (x >> 16): the upper half is final, the lower one is still to be combined with it.
// (Sharing x >> 16 among the lane's neighbours, which differ in it only across a carry, was measured: 3 % slower.)
__device__ __forceinline__ uint32_t random_word(uint32_t counter, uint32_t key1, uint32_t key2)
{
    uint32_t x = counter + key1;
    x ^= x >> 16;
    x *= 0x85ebca6bu;
    x = x ^ (x >> 13) ^ key2;
    return x * 0xc2b2ae35u;
}

// Which elements of its tensor a lane holds: pairs of neighbours that follow one another, or that are 64 apart; half: half of
// the first one's position.  Counters are taken modulo 2^32.
struct EightFrom { uint32_t half; static constexpr int STEP = 2; };
struct PairsFrom { uint32_t half; static constexpr int STEP = 64; };

// ---- one unit's arithmetic ------------------------------------------------------------------------------------------
//
// A lane's eight elements are four pairs, because sm_100 multiplies and adds FP32 pairs in one instruction (each half
// rounded as the scalar operation).  The 8-bit form is bound by instruction issue before it is by HBM, so the pairs and
// the three-operand maximum matter.

struct UnitKeys { uint32_t k1, k2; };

__device__ __forceinline__ float2 pair(float x) { return make_float2(x, x); }
__device__ __forceinline__ unsigned long long bits_of(float2 a) { return *(const unsigned long long *)&a; }
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    unsigned long long d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits_of(a)), "l"(bits_of(b)));
    return *(const float2 *)&d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(bits_of(a)), "l"(bits_of(b)), "l"(bits_of(c)));
    return *(const float2 *)&d;
}
// a + b; results and operands below 2^-126 count as zero.  The flush is there for the roots, and it keeps a product and its
// sum two operations: without it the assembler joins a pair's mul.rn and add.rn into one multiply-add (seen as other
// stored bits where the rounded product lies halfway between two 8-bit values).
__device__ __forceinline__ float2 add_flush(float2 a, float2 b)
{
    unsigned long long d;
    asm("add.rn.ftz.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits_of(a)), "l"(bits_of(b)));
    return *(const float2 *)&d;
}
__device__ __forceinline__ float max_abs3(float a, float b, float c)   // NaN if any is NaN
{
    float d;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float max_abs8(const float2 (&x)[4])
{
    return max_abs3(max_abs3(x[0].x, x[0].y, x[1].x), max_abs3(x[1].y, x[2].x, x[2].y), max_abs3(x[3].x, x[3].y, 0.f));
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float max8(const float2 (&x)[4])
{
    return max3(max3(x[0].x, x[0].y, x[1].x), max3(x[1].y, x[2].x, x[2].y), fmaxf(x[3].x, x[3].y));
}
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}
__device__ __forceinline__ float warp_max_abs(float x)
{
    float d;
    asm("redux.sync.max.abs.NaN.f32 %0, %1, 0xffffffff;" : "=f"(d) : "f"(x));
    return d;
}
__device__ __forceinline__ float rcp_approx(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Minus the correctly rounded root of x = -nx, for x = 0 or 2^-102 <= x < infinity, without a branch: with y ~ 1 / sqrt(x)
// from the hardware's approximation, s = x y is the root to about 2^-22, and s + (x - s^2) y / 2 is one Newton step whose residual
// the fused multiply-add forms exactly (Markstein's square root, IBM J. Res. Dev. 34, 1990).  Between 2^-126 and 2^-102 the root may
// be off by its last bit (a tenth are, at 2^-126): the residual then needs bits under 2^-149, the last that FP32 has.  Infinity
// gives NaN; its block reads as NaN either way.  Everything has its sign turned because a pair's sign costs two instructions,
// and the users of the root can turn a constant instead.
__device__ __forceinline__ float2 minus_sqrt_pair(float2 nx)
{
    float2 y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(fmaxf(-nx.x, 0x1p-126f)));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(fmaxf(-nx.y, 0x1p-126f)));
    const float2 s = mul2(nx, y);                 // -s
    const float2 d = fma2(s, s, nx);              // s^2 - x
    return fma2(d, mul2(pair(0.5f), y), s);
}

// The same from 2^-126 on: small ones from 2^48 x.  Compared with __fsqrt_rn on all these numbers: equal.
__device__ __forceinline__ float2 minus_sqrt_pair_any(float2 nx)
{
    const bool x = nx.x > -0x1p-98f, y = nx.y > -0x1p-98f;
    return mul2(minus_sqrt_pair(mul2(nx, make_float2(x ? 0x1p48f : 1.f, y ? 0x1p48f : 1.f))), make_float2(x ? 0x1p-24f : 1.f, y ? 0x1p-24f : 1.f));
}

// FP32 state: moments in, moments out (the arithmetic of tsr_dense_adamw).
__device__ __forceinline__ void update_f32(float2 (&p)[4], const float2 (&g)[4], float2 (&m)[4], float2 (&v)[4], const DenseStep &a, float lr, float decay)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float2 d;
        d.x = core_update_elem(g[j].x, m[j].x, v[j].x, a.sc);
        d.y = core_update_elem(g[j].y, m[j].y, v[j].y, a.sc);
        p[j] = fma2(pair(-lr), d, mul2(pair(decay), p[j]));
    }
}

// 8-bit state: m and r = sqrt(v) in, as E4M3 values and their scales; new m, -v and -r in FP32 out (r as minus_sqrt_pair gives it).  Every rounding on the way
// to the stored bits is one IEEE operation, so that they are well defined; the update itself takes the approximate
// quotient.  (beta1 scale) code is exactly beta1 (scale code), scale being a power of two.
__device__ __forceinline__ void update_q8(float2 (&p)[4], const float2 (&g)[4], float2 (&m)[4], float2 (&r)[4], float2 (&nv)[4], float2 scale, const DenseStep &a,
                                          float lr, float decay)
{
    const float b1s = __fmul_rn(a.sc.beta1, scale.x), rate = -__fmul_rn(lr, a.sc.inv_bc1);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        m[j] = add_flush(mul2(pair(b1s), m[j]), mul2(pair(a.sc.omb1), g[j]));
        r[j] = mul2(pair(scale.y), r[j]);
        nv[j] = add_flush(mul2(pair(-a.sc.beta2), mul2(r[j], r[j])), mul2(pair(-a.sc.omb2), mul2(g[j], g[j])));
        r[j] = minus_sqrt_pair(nv[j]);
        const float2 den = fma2(r[j], pair(-a.sqrt_inv_bc2), pair(a.sc.eps));
        p[j] = fma2(pair(rate), mul2(m[j], make_float2(rcp_approx(den.x), rcp_approx(den.y))), mul2(pair(decay), p[j]));
    }
}

// New scales of the warp's block, and the codes of m / scale and r / scale for the lane's eight (nr = -r; unless ROUNDED, as
// minus_sqrt_pair gives it for nv = -r^2).
//
// To nearest, the conversion instruction does it.  Stochastic: 2^-120 x / scale has the E4M3 code of x / scale in its bits 20
// to 26, FP32's exponent field running as E4M3's does and its denormal numbers being E4M3's (both have a spacing of one unit
// below exponent 1), so 16 random bits are added below bit 20 and the rest is cut off: one multiply-add on the bits, which
// also moves the code to the top byte.
//
// A root above zero has code 1 at least.  That takes two instructions an element, and only a block that spans a factor of
// 2^17 needs it: a warp without a root below 2^-9 scale skips them.
// It asks for roots below 2^-51 as well, where minus_sqrt_pair may err: with a scale of 2^-42 or more these have code 1 whatever
// their last bit, with a smaller one the roots are taken again.  v stays in registers for that (1B set stochastic: 1 % slower than
// without; 3 % if squares are looked at, by a vote of its own, before any root is taken).
template <bool SR, bool ROUNDED, typename Where>
__device__ __forceinline__ float2 quantise(float2 (&m)[4], float2 (&nr)[4], const float2 (&nv)[4], UnitKeys k, Where where, uint2 &cm, uint2 &cr)
{
    float2 scale, inv;
    block_scale(__float_as_uint(warp_max_abs(max_abs8(m))), scale.x, inv.x);
    block_scale(__float_as_uint(warp_max_abs(max_abs8(nr))), scale.y, inv.y);
    // (NaN, which compares false, needs no floor either)
    const bool floor = __any_sync(0xffffffffu, max8(nr) > __fmaf_rn(-0x1p-9f, scale.y, -0x1p-51f));
    if (!ROUNDED && floor && scale.y < 0x1p-42f && scale.y > 0x1p-126f) {   // (2^-126: all roots are zero)
#pragma unroll
        for (int j = 0; j < 4; ++j) nr[j] = minus_sqrt_pair_any(nv[j]);
        block_scale(__float_as_uint(warp_max_abs(max_abs8(nr))), scale.y, inv.y);
    }
    if constexpr (SR) {
        uint32_t um[8], ur[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 ym = mul2(mul2(m[j], pair(inv.x)), pair(0x1p-120f));
            const float2 yr = mul2(mul2(nr[j], pair(-inv.y)), pair(0x1p-120f));
            um[2 * j] = __float_as_uint(ym.x);
            um[2 * j + 1] = __float_as_uint(ym.y);
            ur[2 * j] = __float_as_uint(yr.x);
            ur[2 * j + 1] = __float_as_uint(yr.y);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t w = random_word(2 * where.half + Where::STEP * (j >> 1) + (j & 1), k.k1, k.k2);
            const uint32_t hi = __byte_perm(w, 0, 0x4324), lo = __byte_perm(w, 0, 0x4104) ^ hi;   // halves of the word, eight bits up
            um[j] = (um[j] * 16u + lo) | (um[j] & 0x80000000u);
            ur[j] = ur[j] * 16u + hi;
        }
        if (floor) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (at(nr, j) < 0.f) ur[j] = max(ur[j], 1u << 24);
        }
        cm.x = top_bytes(um[0], um[1], um[2], um[3]);
        cm.y = top_bytes(um[4], um[5], um[6], um[7]);
        cr.x = top_bytes(ur[0], ur[1], ur[2], ur[3]);
        cr.y = top_bytes(ur[4], ur[5], ur[6], ur[7]);
    } else {
        float2 y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            m[j] = mul2(m[j], pair(inv.x));
            y[j] = mul2(nr[j], pair(-inv.y));
        }
        if (floor) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (at(nr, j) < 0.f) at(y, j) = fmaxf(at(y, j), 0x1p-9f);
        }
        cm = e4m3_pack(m);
        cr = e4m3_pack(y);
        cr.x &= 0x7f7f7f7fu;   // a zero root may be -0
        cr.y &= 0x7f7f7f7fu;
    }
    return scale;
}

// BF16 parameters, stochastic: 16 random bits are added below the seven mantissa bits and the rest is cut off; one random
// word serves elements 2i and 2i + 1 (a pair starts at an even position).  Infinity, with nothing below those bits, stays as it
// is; a NaN does once its lower bits, from which a carry could run into the sign, are cleared.  Returns the BF16 values.
template <typename Where>
__device__ __forceinline__ uint4 round_params(const float2 (&p)[4], UnitKeys k, Where where)
{
    uint32_t w[4], b[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        b[2 * j] = __float_as_uint(p[j].x);
        b[2 * j + 1] = __float_as_uint(p[j].y);
    }
    if (isnan(max_abs8(p))) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if ((b[j] & 0x7fffffffu) > 0x7f800000u) b[j] = 0x7fff0000u;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t x = random_word(where.half + Where::STEP / 2 * j, k.k1 ^ 0x5bd1e995u, k.k2), hi = x >> 16;
        w[j] = __byte_perm(b[2 * j] + ((x ^ hi) & 0xffffu), b[2 * j + 1] + hi, 0x7632);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Where nothing is known of the alignment, a lane has the pairs of neighbours at base + 2 lane + 64 j, so that the warp's
// accesses stay together.  Walk says where a pair lies in a matrix with row pitch: row and column of the first by one
// division, the others by steps of 64.
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
    __device__ __forceinline__ void next()   // 64 elements on
    {
        col += 64;
        if ((t.flags & REC_PITCHED) && col >= t.cols) {
            if (t.cols >= 64) { col -= t.cols; ++row; } else split(row * t.cols + col);
        }
    }
    // the pair's elements, in a matrix of pitch ld
    __device__ __forceinline__ int64_t one(int64_t ld) const { return row * ld + col; }
    __device__ __forceinline__ int64_t two(int64_t ld) const
    {
        return (t.flags & REC_PITCHED) && col + 1 == t.cols ? (row + 1) * ld : row * ld + col + 1;
    }
};
__device__ __forceinline__ int64_t pair_at(int64_t base, int lane, int j) { return base + 2 * lane + 64 * j; }

// Pairs of moments, as codes or FP32; elements from n on are zero, and not written (WHOLE: there are none).  Where there are,
// every load is issued and the value dropped (the tensor's first element stands in): a load under a condition would be waited
// for before the next, a memory latency each.
template <bool WHOLE>
__device__ __forceinline__ uint2 load_code_pairs(const void *src, bool both, int64_t base, int lane, int64_t n)
{
    const uint8_t *c = (const uint8_t *)src;
    uint32_t two[4];
    if (WHOLE && both) {
#pragma unroll
        for (int j = 0; j < 4; ++j) two[j] = *(const uint16_t *)(c + pair_at(base, lane, j));
    } else {
        uint32_t one[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t e = pair_at(base, lane, j >> 1) + (j & 1);
            one[j] = c[WHOLE || e < n ? e : 0];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!WHOLE && pair_at(base, lane, j >> 1) + (j & 1) >= n) one[j] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) two[j] = one[2 * j] | (one[2 * j + 1] << 8);
    }
    return make_uint2(two[0] | (two[1] << 16), two[2] | (two[3] << 16));
}
template <bool WHOLE>
__device__ __forceinline__ void load_pairs(const void *src, bool both, int64_t base, int lane, int64_t n, float2 (&x)[4])
{
    const float *f = (const float *)src;
    if (WHOLE && both) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = *(const float2 *)(f + pair_at(base, lane, j));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t e = pair_at(base, lane, j >> 1) + (j & 1);
            at(x, j) = f[WHOLE || e < n ? e : 0];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!WHOLE && pair_at(base, lane, j >> 1) + (j & 1) >= n) at(x, j) = 0.f;
    }
}
template <bool WHOLE>
__device__ __forceinline__ void store_code_pairs(void *dst, bool both, int64_t base, int lane, int64_t n, uint2 codes)
{
    const uint32_t w[2] = {codes.x, codes.y};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t e = pair_at(base, lane, j);
        uint8_t *c = (uint8_t *)dst + e;
        const uint32_t two = w[j >> 1] >> (16 * (j & 1));
        if (both && (WHOLE || e + 1 < n)) *(uint16_t *)c = (uint16_t)two;
        else {
            if (WHOLE || e < n) c[0] = (uint8_t)two;
            if (WHOLE || e + 1 < n) c[1] = (uint8_t)(two >> 8);
        }
    }
}
template <bool WHOLE>
__device__ __forceinline__ void store_pairs(void *dst, bool both, int64_t base, int lane, int64_t n, const float2 (&x)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t e = pair_at(base, lane, j);
        float *f = (float *)dst + e;
        if (both && (WHOLE || e + 1 < n)) *(float2 *)f = x[j];
        else {
            if (WHOLE || e < n) f[0] = x[j].x;
            if (WHOLE || e + 1 < n) f[1] = x[j].y;
        }
    }
}

__device__ __forceinline__ float2 load_two(const float *x) { return *(const float2 *)x; }
__device__ __forceinline__ float2 load_two(const bf16 *x)
{
    const uint32_t w = *(const uint32_t *)x;
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

// The lane's pairs of a unit that lies at u, its elements from number `left` on `gap` places further.  TWO: whole pairs where u
// is aligned to them and nothing moves (the norm of a pitched gradient is 4 % faster with it, the FP32 step 2.5 % slower).
template <bool TWO, typename T>
__device__ __forceinline__ void load_run(const T *u, int left, int gap, int lane, float2 (&out)[4])
{
    if (TWO && left == UNIT && ((uintptr_t)u & (2 * sizeof(T) - 1)) == 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] = load_two(u + 2 * lane + 64 * j);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = 2 * lane + 64 * (j >> 1) + (j & 1);
            at(out, j) = to_f32(u[i < left ? i : i + gap]);
        }
    }
}
template <typename T>
__device__ __forceinline__ void store_run(T *u, int left, int gap, int lane, const float2 (&in)[4])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int i = 2 * lane + 64 * (j >> 1) + (j & 1);
        from_f32(u[i < left ? i : i + gap], (j & 1) ? in[j >> 1].y : in[j >> 1].x);
    }
}

// Pairs of a parameter, gradient or image (pitch ld).  row, col: where the unit starts (PLAIN, ROWS).
template <int PATH, bool TWO, typename T>
__device__ __forceinline__ void load_matrix(const T *x, const DenseRec &t, int64_t ld, int64_t base, int64_t row, int64_t col, int lane, float2 (&out)[4])
{
    if constexpr (PATH == PATH_ANY) {
        Walk w(t, pair_at(base, lane, 0));
        T raw[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t e = pair_at(base, lane, j);
            raw[2 * j] = x[e < t.n ? w.one(ld) : 0];
            raw[2 * j + 1] = x[e + 1 < t.n ? w.two(ld) : 0];
            w.next();
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) at(out, j) = pair_at(base, lane, j >> 1) + (j & 1) < t.n ? to_f32(raw[j]) : 0.f;
    } else {
        if constexpr (PATH == PATH_PLAIN) load_run<TWO>(x + base, UNIT, 0, lane, out);
        else load_run<TWO>(x + row * ld + col, (int)min(t.cols - col, (int64_t)UNIT), (int)(ld - t.cols), lane, out);
    }
}
template <int PATH, typename T>
__device__ __forceinline__ void store_matrix(T *x, const DenseRec &t, int64_t ld, int64_t base, int64_t row, int64_t col, int lane, const float2 (&in)[4])
{
    if constexpr (PATH == PATH_ANY) {
        Walk w(t, pair_at(base, lane, 0));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t e = pair_at(base, lane, j);
            if (e < t.n) from_f32(x[w.one(ld)], in[j].x);
            if (e + 1 < t.n) from_f32(x[w.two(ld)], in[j].y);
            w.next();
        }
    } else {
        if constexpr (PATH == PATH_PLAIN) store_run(x + base, UNIT, 0, lane, in);
        else store_run(x + row * ld + col, (int)min(t.cols - col, (int64_t)UNIT), (int)(ld - t.cols), lane, in);
    }
}

struct Values { float2 p[4], g[4], m[4], v[4], scale; };   // a lane's eight elements in FP32, and the block's scales

// The step of pairs from their values on; returns the block's new scales.
template <int PATH, typename PT, bool Q8, bool SR>
__device__ __forceinline__ float2 update_pairs(Values &x, const DenseRec &t, int64_t base, int64_t row, int64_t col, int lane, float gs, const DenseStep &a,
                                               float lr, float decay, UnitKeys key)
{
    constexpr bool WHOLE = PATH != PATH_ANY;
    const bool both = t.flags & REC_PAIR_STATE;
#pragma unroll
    for (int j = 0; j < 4; ++j) x.g[j] = mul2(x.g[j], pair(gs));
    float2 nv[4];
    if constexpr (Q8) update_q8(x.p, x.g, x.m, x.v, nv, x.scale, a, lr, decay);
    else update_f32(x.p, x.g, x.m, x.v, a, lr, decay);
    const PairsFrom where = {(uint32_t)(base >> 1) + lane};
    if constexpr (SR && sizeof(PT) == 2) {
        Eight<bf16> rounded;
        rounded.r = round_params(x.p, key, where);
        rounded.get(x.p);
    }
    store_matrix<PATH>((PT *)t.p, t, t.ldp, base, row, col, lane, x.p);
    if (sizeof(PT) == 4 && t.image) store_matrix<PATH>(t.image, t, t.ldi, base, row, col, lane, x.p);
    float2 scale = make_float2(0.f, 0.f);
    if constexpr (Q8) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!WHOLE && pair_at(base, lane, j >> 1) + (j & 1) >= t.n) at(x.m, j) = at(x.v, j) = at(nv, j) = 0.f;   // (0 * NaN of a poisoned block)
        uint2 cm, cr;
        scale = quantise<SR, false>(x.m, x.v, nv, key, where, cm, cr);
        store_code_pairs<WHOLE>(t.m, both, base, lane, t.n, cm);
        store_code_pairs<WHOLE>(t.v, both, base, lane, t.n, cr);
    } else {
        store_pairs<WHOLE>(t.m, both, base, lane, t.n, x.m);
        store_pairs<WHOLE>(t.v, both, base, lane, t.n, x.v);
    }
    return scale;
}

// The units of a warp on the paths without vectors, loaded straight from memory.
template <int PATH, typename PT, typename GT, bool Q8, bool SR>
__device__ __forceinline__ void step_pairs(const DenseRec &rec, int64_t base, int todo, int lane, float gs, const DenseStep &a, float lr, float decay, UnitKeys key)
{
    const DenseRec t = rec;
    constexpr int64_t STRIDE = WARPS * UNIT;
    constexpr bool WHOLE = PATH != PATH_ANY;
    const bool both = t.flags & REC_PAIR_STATE;
    if (WHOLE && !isfinite(gs)) return;   // (looking at it after the loads makes this path 3 % slower)
    int64_t row = 0, col = 0;
    if constexpr (PATH == PATH_ROWS) {
        row = base / t.cols;
        col = base - row * t.cols;
    }
#pragma unroll 1
    for (; todo > 0; --todo, base += STRIDE) {
        Values x;
        uint2 cm, cr;
        if constexpr (Q8) {
            x.scale = t.scale[base / UNIT];
            cm = load_code_pairs<WHOLE>(t.m, both, base, lane, t.n);
            cr = load_code_pairs<WHOLE>(t.v, both, base, lane, t.n);
        } else {
            load_pairs<WHOLE>(t.m, both, base, lane, t.n, x.m);
            load_pairs<WHOLE>(t.v, both, base, lane, t.n, x.v);
        }
        load_matrix<PATH, false>((const PT *)t.p, t, t.ldp, base, row, col, lane, x.p);
        load_matrix<PATH, false>((const GT *)t.g, t, t.ldg, base, row, col, lane, x.g);
        if (!WHOLE && !isfinite(gs)) return;
        if constexpr (Q8) {
            e4m3_unpack(cm, x.m);
            e4m3_unpack(cr, x.v);
        }
        const float2 s = update_pairs<PATH, PT, Q8, SR>(x, t, base, row, col, lane, gs, a, lr, decay, key);
        if (Q8 && lane == 0) t.scale[base / UNIT] = s;
        if constexpr (PATH == PATH_ROWS)
            for (col += STRIDE; col >= t.cols; col -= t.cols) ++row;
    }
}

// One whole unit of the vector path as it lies in memory: the lane's eight elements of everything.
template <typename PT, typename GT, bool Q8> struct RawUnit {
    Eight<PT> p;
    Eight<GT> g;
    uint2 cm, cr;
    Eight<float> m, v;
    float2 scale;
};

template <typename PT, typename GT, bool Q8> struct VectorUnit {   // pointers to the lane's elements of a unit
    PT *p;
    const GT *g;
    char *m, *v;
    float2 *scale;
    bf16 *image;
    static constexpr int MOMENT = Q8 ? 1 : 4;

    __device__ __forceinline__ VectorUnit(const DenseRec &t, int64_t base, int lane)
    {
        const int64_t e = base + lane * 8;
        p = (PT *)t.p + e;
        g = (const GT *)t.g + e;
        m = (char *)t.m + e * MOMENT;
        v = (char *)t.v + e * MOMENT;
        if constexpr (Q8) scale = t.scale + base / UNIT;
        image = sizeof(PT) == 4 && t.image ? t.image + e : nullptr;
    }
    __device__ __forceinline__ void load(RawUnit<PT, GT, Q8> &r, int off) const   // off: elements ahead, whole units
    {
        r.p.load(p + off);
        r.g.load(g + off);
        if constexpr (Q8) {
            r.cm = load8(m + off);
            r.cr = load8(v + off);
            r.scale = scale[off / UNIT];
        } else {
            r.m.load((const float *)m + off);
            r.v.load((const float *)v + off);
        }
    }
    __device__ __forceinline__ void advance(int64_t off)
    {
        p += off;
        g += off;
        m += off * MOMENT;
        v += off * MOMENT;
        if constexpr (Q8) scale += off / UNIT;
        if (sizeof(PT) == 4 && image) image += off;
    }
    static __device__ __forceinline__ void unpack(const RawUnit<PT, GT, Q8> &raw, Values &x)
    {
        raw.p.get(x.p);
        raw.g.get(x.g);
        if constexpr (Q8) {
            e4m3_unpack(raw.cm, x.m);
            e4m3_unpack(raw.cr, x.v);
            x.scale = raw.scale;
        } else {
            raw.m.get(x.m);
            raw.v.get(x.v);
        }
    }
    template <bool SR>
    __device__ __forceinline__ void step(Values &x, uint32_t half, int lane, float gs, const DenseStep &a, float lr, float decay, UnitKeys key) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) x.g[j] = mul2(x.g[j], pair(gs));
        float2 nv[4];
        if constexpr (Q8) update_q8(x.p, x.g, x.m, x.v, nv, x.scale, a, lr, decay);
        else update_f32(x.p, x.g, x.m, x.v, a, lr, decay);
        const EightFrom where = {half};
        if constexpr (SR && sizeof(PT) == 2) *(uint4 *)p = round_params(x.p, key, where);
        else Eight<PT>::put(p, x.p);
        if (sizeof(PT) == 4 && image) Eight<bf16>::put(image, x.p);
        if constexpr (Q8) {
            uint2 cm, cr;
            const float2 s = quantise<SR, false>(x.m, x.v, nv, key, where, cm, cr);
            *(uint2 *)m = cm;
            *(uint2 *)v = cr;
            if (lane == 0) *scale = s;
        } else {
            Eight<float>::put((float *)m, x.m);
            Eight<float>::put((float *)v, x.v);
        }
    }
};

// The 8-bit form reads so little per unit that a unit's loads in registers do not keep HBM busy.  So a warp's loads go to
// slots of shared memory that only its warp reads (asynchronous copies of 16 and 8 bytes, no barrier between warps): DEPTH
// slots, DEPTH - 1 of them on their way.
template <typename PT, typename GT, bool MIXED> struct Ring {
    static constexpr int P_VECS = sizeof(PT) / 2, G_VECS = sizeof(GT) / 2;   // 16-byte vectors of a lane
    static constexpr int THREADS = WARPS * 32;
    // a warp's parameters, gradients (MIXED: with room for two beginnings and ends off 16 bytes), codes of m and r, scales
    static constexpr int P_WARP = 512 * P_VECS + (MIXED ? 48 : 0), G_WARP = 512 * G_VECS + (MIXED ? 48 : 0);
    static constexpr int G_AT = WARPS * P_WARP, M_AT = G_AT + WARPS * G_WARP, V_AT = M_AT + THREADS * 8, S_AT = V_AT + THREADS * 8;
    static constexpr int SLOT = S_AT + WARPS * 8;
    static constexpr int DEPTH = P_VECS + G_VECS == 2 ? 5 : P_VECS + G_VECS == 3 ? 4 : 3;   // three CTAs on an SM
    static constexpr int BYTES = DEPTH * SLOT;

    static __device__ __forceinline__ void copy16(uint32_t to, const void *from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
    static __device__ __forceinline__ void copy8(uint32_t to, const void *from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory"); }
    static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    static __device__ __forceinline__ void drain() { asm volatile("cp.async.wait_all;" ::: "memory"); }
    static __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 2) : "memory"); }

    // Fills slot `to` (a shared-memory address) with the unit that is `units` units of this warp after u.
    static __device__ __forceinline__ void issue(uint32_t to, const VectorUnit<PT, GT, true> &u, int units, int warp, int lane)
    {
        const int off = units * WARPS * UNIT;
        put(to + warp * P_WARP, u.p + off, lane);
        put(to + G_AT + warp * G_WARP, u.g + off, lane);
        issue_state(to, u.m + off, u.v + off, u.scale + off / UNIT, warp, lane);
    }
    // m, v: the lane's eight codes
    static __device__ __forceinline__ void issue_state(uint32_t to, const void *m, const void *v, const float2 *scale, int warp, int lane)
    {
        copy8(to + M_AT + (warp * 32 + lane) * 8, m);
        copy8(to + V_AT + (warp * 32 + lane) * 8, v);
        if (lane == 0) copy8(to + S_AT + warp * 8, scale);
    }
    static __device__ __forceinline__ void fetch(const char *slot, int warp, int lane, RawUnit<PT, GT, true> &r)
    {
        get(slot + warp * P_WARP, lane, r.p);
        get(slot + G_AT + warp * G_WARP, lane, r.g);
        r.cm = *(const uint2 *)(slot + M_AT + (warp * 32 + lane) * 8);
        r.cr = *(const uint2 *)(slot + V_AT + (warp * 32 + lane) * 8);
        r.scale = *(const float2 *)(slot + S_AT + warp * 8);
    }
    // A warp's 256 BF16 elements: a vector of 16 bytes for each lane.
    static __device__ __forceinline__ void put(uint32_t to, const bf16 *x, int lane) { copy16(to + lane * 16, x); }
    static __device__ __forceinline__ void get(const char *s, int lane, Eight<bf16> &x) { x.r = *(const uint4 *)(s + lane * 16); }
    // 256 FP32 elements, 64 vectors: copied in order (lanes 16 bytes apart, so that whole sectors travel), read two by two.  Vector
    // c lies at place c ^ bit 3 of c, which keeps the reads, 32 bytes apart, free of bank conflicts.
    static __device__ __forceinline__ void put(uint32_t to, const float *x, int lane)
    {
        to += (lane ^ ((lane >> 3) & 1)) * 16;
        copy16(to, (const char *)x - lane * 16);
        copy16(to + 512, (const char *)x - lane * 16 + 512);
    }
    static __device__ __forceinline__ void get(const char *s, int lane, Eight<float> &x)
    {
        const int bit = (lane >> 2) & 1;
        const uint4 a = *(const uint4 *)(s + ((2 * lane) ^ bit) * 16), b = *(const uint4 *)(s + ((2 * lane + 1) ^ bit) * 16);
        x.r = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    }
};

// A unit of any alignment travels as the 16-byte vectors that hold it, the first and last with neighbouring bytes that are not
// looked at.  Every vector holds an element of the unit, so it lies in the same allocation granule.
// 2 N words of shared memory from s + off on, off < 16 a multiple of 2, s a multiple of 8 bytes: aligned words, moved by one if
// need be and, for an odd number of BF16 elements, by half a word.
template <int N>
__device__ __forceinline__ void read_shifted(const char *s, int off, uint32_t (&w)[2 * N])
{
    uint32_t x[2 * N + 2];
#pragma unroll
    for (int k = 0; k <= N; ++k) {
        const uint2 d = *(const uint2 *)(s + (off & 8) + 8 * k);
        x[2 * k] = d.x;
        x[2 * k + 1] = d.y;
    }
    if (off & 4) {
#pragma unroll
        for (int k = 0; k <= 2 * N; ++k) x[k] = x[k + 1];
    }
#pragma unroll
    for (int k = 0; k < 2 * N; ++k) w[k] = N == 2 ? __funnelshift_r(x[k], x[k + 1], (off & 2) * 8) : x[k];
}
__device__ __forceinline__ void shifted(const char *s, int off, int lane, Eight<bf16> &x)
{
    uint32_t w[4];
    read_shifted<2>(s + lane * 16, off, w);
    x.r = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void shifted(const char *s, int off, int lane, Eight<float> &x) { read_shifted<4>(s + lane * 32, off, x.r.w); }

// A warp's 256 elements, eight to a lane (words w), to an address of any alignment: through shared memory (the warp's own
// `room`, 48 bytes more than they take), so that all but the elements off the 16-byte grid leave in vectors.
template <typename T>
__device__ __forceinline__ void store_shifted(T *to, char *room, int lane, const uint32_t (&w)[2 * (int)sizeof(T)])
{
    constexpr int ES = sizeof(T), PER = 16 / ES;   // elements of a vector
    const int off = (int)((uintptr_t)to & 15);
    if (off == 0) {
#pragma unroll
        for (int k = 0; k < ES / 2; ++k) ((uint4 *)to)[lane * (ES / 2) + k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
        return;
    }
    __syncwarp();   // what was here has been read
#pragma unroll
    for (int k = 0; k < ES / 2; ++k) ((uint4 *)room)[lane * (ES / 2) + k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
    __syncwarp();
    uint32_t x[2 * ES];
    read_shifted<ES>(room + lane * 8 * ES, 16 - off, x);
    uint4 *v = (uint4 *)((char *)to - off) + 1 + lane * (ES / 2);
#pragma unroll
    for (int k = 0; k < ES / 2; ++k)
        if (lane < 31 || k < ES / 2 - 1) v[k] = make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
    if (lane < PER) {   // the first PER - off / ES elements and the last off / ES
        const int i = lane < PER - off / ES ? lane : UNIT - PER + lane;
        to[i] = ((const T *)room)[i];
    }
}

// What the ring's units without vectors share: from a filled slot to the stores.  to: the unit's parameters in memory (one run);
// g_off: bytes by which its gradients are off the 16-byte grid; m, v: the lane's eight codes.  `next` starts the next loads.
template <typename PT, typename GT, bool SR, typename Next>
__device__ __forceinline__ float2 step_shifted(char *slot, PT *to, bf16 *image, int g_off, char *m, char *v, uint32_t half, int warp, int lane, float gs,
                                               const DenseStep &a, float lr, float decay, UnitKeys key, Next next)
{
    typedef Ring<PT, GT, true> R;
    char *room = slot + warp * R::P_WARP;
    RawUnit<PT, GT, true> raw;
    shifted(room, (int)((uintptr_t)to & 15), lane, raw.p);
    shifted(slot + R::G_AT + warp * R::G_WARP, g_off, lane, raw.g);
    raw.cm = *(const uint2 *)(slot + R::M_AT + (warp * 32 + lane) * 8);
    raw.cr = *(const uint2 *)(slot + R::V_AT + (warp * 32 + lane) * 8);
    Values x;
    x.scale = *(const float2 *)(slot + R::S_AT + warp * 8);
    raw.p.get(x.p);
    raw.g.get(x.g);
    e4m3_unpack(raw.cm, x.m);
    e4m3_unpack(raw.cr, x.v);
    next();
#pragma unroll
    for (int j = 0; j < 4; ++j) x.g[j] = mul2(x.g[j], pair(gs));
    float2 nv[4];
    update_q8(x.p, x.g, x.m, x.v, nv, x.scale, a, lr, decay);
    const EightFrom where = {half};
    if constexpr (sizeof(PT) == 2) {
        uint4 w;
        if constexpr (SR) w = round_params(x.p, key, where);
        else w = bf16_pack(x.p);
        store_shifted(to, room, lane, {w.x, w.y, w.z, w.w});
    } else {
        store_shifted(to, room, lane, {__float_as_uint(x.p[0].x), __float_as_uint(x.p[0].y), __float_as_uint(x.p[1].x), __float_as_uint(x.p[1].y),
                                       __float_as_uint(x.p[2].x), __float_as_uint(x.p[2].y), __float_as_uint(x.p[3].x), __float_as_uint(x.p[3].y)});
        if (image) {
            const uint4 w = bf16_pack(x.p);
            store_shifted(image, room, lane, {w.x, w.y, w.z, w.w});
        }
    }
    uint2 cm, cr;
    const float2 scale = quantise<SR, false>(x.m, x.v, nv, key, where, cm, cr);
    *(uint2 *)m = cm;
    *(uint2 *)v = cr;
    return scale;
}

// The 8-bit step of a warp's units of a contiguous tensor off the 16-byte grid.
template <typename PT, typename GT, bool SR>
__device__ __forceinline__ void step_plain(const DenseRec &t, int64_t base, int todo, int warp, int lane, float gs, const DenseStep &a, float lr, float decay,
                                           UnitKeys key, char *slots)
{
    typedef Ring<PT, GT, true> R;
    constexpr int STRIDE = WARPS * UNIT;
    const int p_off = (int)((uintptr_t)((const PT *)t.p + base) & 15), g_off = (int)((uintptr_t)((const GT *)t.g + base) & 15);   // of every unit
    char *p = (char *)((PT *)t.p + base) - p_off + lane * 16;              // the lane's vector
    const char *g = (const char *)((const GT *)t.g + base) - g_off + lane * 16;
    char *m = (char *)t.m + base + lane * 8, *v = (char *)t.v + base + lane * 8;
    float2 *scale = t.scale + base / UNIT;
    bf16 *image = t.image ? t.image + base : nullptr;
    uint32_t half = (uint32_t)(base >> 1) + lane * 4;
    const uint32_t first = (uint32_t)__cvta_generic_to_shared(slots);
    auto issue = [&](uint32_t to, int units) {
        const int off = units * STRIDE;
        const uint32_t to_p = to + warp * R::P_WARP + lane * 16, to_g = to + R::G_AT + warp * R::G_WARP + lane * 16;
#pragma unroll
        for (int k = 0; k < R::P_VECS; ++k) R::copy16(to_p + 512 * k, p + off * (int)sizeof(PT) + 512 * k);
#pragma unroll
        for (int k = 0; k < R::G_VECS; ++k) R::copy16(to_g + 512 * k, g + off * (int)sizeof(GT) + 512 * k);
        if (lane == 0) {   // the vector of the last elements
            if (p_off) R::copy16(to_p + 512 * R::P_VECS, p + off * (int)sizeof(PT) + 512 * R::P_VECS);
            if (g_off) R::copy16(to_g + 512 * R::G_VECS, g + off * (int)sizeof(GT) + 512 * R::G_VECS);
        }
        R::issue_state(to, m + off, v + off, scale + off / UNIT, warp, lane);
    };
#pragma unroll
    for (int k = 0; k < R::DEPTH - 1; ++k) {
        if (k < todo) issue(first + k * R::SLOT, k);
        R::commit();
    }
    if (!isfinite(gs)) return R::drain();
    int in = (R::DEPTH - 1) * R::SLOT, out = 0;
#pragma unroll 1
    for (; todo > 0; --todo) {
        R::wait();
        __syncwarp();   // other lanes' copies; and every lane has read the slot that is filled next
        const float2 s = step_shifted<PT, GT, SR>(slots + out, (PT *)(p - lane * 16 + p_off), image, g_off, m, v, half, warp, lane, gs, a, lr, decay, key, [&]() {
            if (todo >= R::DEPTH) issue(first + in, R::DEPTH - 1);
            R::commit();
        });
        if (lane == 0) *scale = s;
        in = in + R::SLOT == R::BYTES ? 0 : in + R::SLOT;
        out = out + R::SLOT == R::BYTES ? 0 : out + R::SLOT;
        p += STRIDE * sizeof(PT);
        g += STRIDE * sizeof(GT);
        m += STRIDE;
        v += STRIDE;
        scale += STRIDE / UNIT;
        if (image) image += STRIDE;
        half += STRIDE / 2;
    }
}

// A unit of a matrix with a row pitch: one run of elements, or two where a row ends (the second from the start of the next
// row, its vectors behind the first's).
template <typename T> struct Runs {
    const char *one, *two;   // vectors
    int left;                // elements of the first run
    int skip, gap;           // the first element's place in its vector, and the step from the first run's end to the second run
    int vectors_one, vectors;

    __device__ __forceinline__ Runs(const T *x, int ld, int cols, int row, int col)
    {
        constexpr int ES = sizeof(T);
        const uintptr_t a = (uintptr_t)(x + (int64_t)row * ld + col);
        left = min(cols - col, UNIT);
        skip = (int)(a & 15) / ES;
        one = (const char *)(a & ~(uintptr_t)15);
        vectors = vectors_one = ((skip + left) * ES + 15) / 16;
        two = one;
        gap = 0;
        if (left < UNIT) {
            const uintptr_t b = (uintptr_t)(x + (int64_t)(row + 1) * ld);
            const int skip_two = (int)(b & 15) / ES;
            two = (const char *)(b & ~(uintptr_t)15) - 16 * vectors_one;
            vectors += ((skip_two + UNIT - left) * ES + 15) / 16;
            gap = 16 / ES * vectors_one + skip_two - skip - left;
        }
    }
    __device__ __forceinline__ void copy(uint32_t to, int lane) const
    {
        constexpr int MOST = 16 * (int)sizeof(T);   // and up to three more
#pragma unroll
        for (int k = lane; k < MOST; k += 32)
            if (k < vectors) Ring<T, T, true>::copy16(to + k * 16, (k < vectors_one ? one : two) + k * 16);
        if (MOST + lane < vectors) Ring<T, T, true>::copy16(to + (MOST + lane) * 16, (MOST + lane < vectors_one ? one : two) + (MOST + lane) * 16);
    }
    __device__ __forceinline__ void read(const char *slot, int lane, float2 (&out)[4]) const { load_run<false>((const T *)slot + skip, left, gap, lane, out); }
};

// The 8-bit step of a warp's units of a matrix with long rows and a pitch.  A unit in one run goes on shifted to its alignment,
// one with the end of a row in pairs 64 apart.
template <typename PT, typename GT, bool SR>
__device__ __forceinline__ void step_rows(const DenseRec &t, int64_t base, int todo, int warp, int lane, float gs, const DenseStep &a, float lr, float decay,
                                          UnitKeys key, char *slots)
{
    typedef Ring<PT, GT, true> R;
    constexpr int STRIDE = WARPS * UNIT;
    const int cols = (int)t.cols, ldp = (int)t.ldp, ldg = (int)t.ldg;
    PT *const P = (PT *)t.p;
    const GT *const G = (const GT *)t.g;
    char *m = (char *)t.m + base + lane * 8, *v = (char *)t.v + base + lane * 8;
    float2 *scale = t.scale + base / UNIT;
    uint32_t half = (uint32_t)(base >> 1) + lane * 4;
    int row = (int)(base / t.cols), col = (int)(base - (int64_t)row * cols), in_row = row, in_col = col;
    const uint32_t first = (uint32_t)__cvta_generic_to_shared(slots);
    auto issue = [&](uint32_t to, int units) {
        Runs<PT>(P, ldp, cols, in_row, in_col).copy(to + warp * R::P_WARP, lane);
        Runs<GT>(G, ldg, cols, in_row, in_col).copy(to + R::G_AT + warp * R::G_WARP, lane);
        R::issue_state(to, m + units * STRIDE, v + units * STRIDE, scale + units * (STRIDE / UNIT), warp, lane);
        for (in_col += STRIDE; in_col >= cols; in_col -= cols) ++in_row;
    };
#pragma unroll 1
    for (int k = 0; k < R::DEPTH - 1; ++k) {
        if (k < todo) issue(first + k * R::SLOT, k);
        R::commit();
    }
    if (!isfinite(gs)) return R::drain();
    int in = (R::DEPTH - 1) * R::SLOT, out = 0;
#pragma unroll 1
    for (; todo > 0; --todo) {
        R::wait();
        __syncwarp();   // other lanes' copies; and every lane has read the slot that is filled next
        char *slot = slots + out;
        auto next = [&]() {
            if (todo >= R::DEPTH) issue(first + in, R::DEPTH - 1);
            R::commit();
        };
        float2 s;
        if (cols - col >= UNIT) {
            bf16 *image = sizeof(PT) == 4 && t.image ? t.image + (int64_t)row * t.ldi + col : nullptr;
            s = step_shifted<PT, GT, SR>(slot, P + (int64_t)row * ldp + col, image, (int)((uintptr_t)(G + (int64_t)row * ldg + col) & 15), m, v, half, warp, lane, gs, a,
                                         lr, decay, key, next);
        } else {
            Values x;
            Runs<PT>(P, ldp, cols, row, col).read(slot + warp * R::P_WARP, lane, x.p);
            Runs<GT>(G, ldg, cols, row, col).read(slot + R::G_AT + warp * R::G_WARP, lane, x.g);
            e4m3_unpack(load_code_pairs<true>(slot + R::M_AT + warp * UNIT, true, 0, lane, 0), x.m);
            e4m3_unpack(load_code_pairs<true>(slot + R::V_AT + warp * UNIT, true, 0, lane, 0), x.v);
            x.scale = *(const float2 *)(slot + R::S_AT + warp * 8);
            next();
            s = update_pairs<PATH_ROWS, PT, true, SR>(x, t, (int64_t)row * cols + col, row, col, lane, gs, a, lr, decay, key);
        }
        if (lane == 0) *scale = s;
        in = in + R::SLOT == R::BYTES ? 0 : in + R::SLOT;
        out = out + R::SLOT == R::BYTES ? 0 : out + R::SLOT;
        m += STRIDE;
        v += STRIDE;
        scale += STRIDE / UNIT;
        half += STRIDE / 2;
        for (col += STRIDE; col >= cols; col -= cols) ++row;
    }
}

// Which kernels load vectors through the ring (stochastic rounding of BF16 parameters is bound by instructions, and faster with
// the next unit in registers: 1B set 2.55 against 2.68 ms), and which have one at all.
template <typename PT> __host__ __device__ constexpr bool vectors_in_ring(bool q8, bool sr) { return q8 && (!sr || sizeof(PT) == 4); }
template <typename PT> __host__ __device__ constexpr bool has_ring(bool q8, bool sr, bool mixed) { return q8 && (mixed || vectors_in_ring<PT>(q8, sr)); }

// MIXED: there are chunks of every path.  Where all chunks are vectors, a kernel without the other paths is launched: their
// registers and the wider slots cost the 8-bit form 3 % (130M set: 181 against 175 us; 1B set stochastic 2.61 against 2.55 ms).
template <typename PT, typename GT, bool Q8, bool SR, bool MIXED>
__global__ void __launch_bounds__(WARPS * 32, Q8 ? STEP_Q8_CTAS : STEP_F32_CTAS)
dense_step_kernel(const DenseRec *__restrict__ recs, const DenseChunk *__restrict__ chunks, const DenseStep a)
{
    extern __shared__ __align__(16) char slots[];   // of the ring
    pdl_trigger();
    const DenseChunk ch = chunks[blockIdx.x];
    const DenseRec &t = recs[ch.rec];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float lr = __fmul_rn(a.lr, t.lr_mult);
    const float decay = __fsub_rn(1.f, __fmul_rn(lr, __fmul_rn(a.wd, t.wd_mult)));
    UnitKeys key = {0, 0};
    if constexpr (SR) {
        key.k1 = mix32(a.seed_key ^ mix32(a.step_lo + 0x7f4a7c15u * (uint32_t)(t.index + 1)));
        key.k2 = mix32(key.k1 ^ 0xa511e9b3u);
    }
    pdl_wait();
    // A factor that is not finite ends the step; it is looked at once the first loads are on their way.
    float gs = 1.f;
    if (a.grad_scale) gs = *(const volatile float *)a.grad_scale;
    constexpr int64_t STRIDE = WARPS * UNIT;
    constexpr bool RING = vectors_in_ring<PT>(Q8, SR);
    int64_t base = ((int64_t)ch.first + warp) * UNIT;
    int todo = (ch.units - warp + WARPS - 1) / WARPS;   // units of this warp
    if (todo <= 0) return;
    if (!MIXED || ch.path == PATH_VECTORS) {
        VectorUnit<PT, GT, Q8> u(t, base, lane);
        uint32_t half = (uint32_t)(base >> 1) + lane * 4;   // half of the position of the lane's first element
        RawUnit<PT, GT, Q8> raw;
        Values x;
        if constexpr (RING) {
            typedef Ring<PT, GT, MIXED> R;
            const uint32_t first = (uint32_t)__cvta_generic_to_shared(slots);
            int in = (R::DEPTH - 1) * R::SLOT, out = 0;   // byte offsets of the slots to fill and to read
#pragma unroll
            for (int k = 0; k < R::DEPTH - 1; ++k) {
                if (k < todo) R::issue(first + k * R::SLOT, u, k, warp, lane);
                R::commit();
            }
            if (!isfinite(gs)) return R::drain();
#pragma unroll 1
            for (; todo > 0; --todo) {
                R::wait();
                __syncwarp();   // other lanes' copies; and every lane has read the slot that is filled next
                R::fetch(slots + out, warp, lane, raw);
                if (todo >= R::DEPTH) R::issue(first + in, u, R::DEPTH - 1, warp, lane);
                R::commit();
                in = in + R::SLOT == R::BYTES ? 0 : in + R::SLOT;
                out = out + R::SLOT == R::BYTES ? 0 : out + R::SLOT;
                u.unpack(raw, x);
                u.template step<SR>(x, half, lane, gs, a, lr, decay, key);
                u.advance(STRIDE);
                half += STRIDE / 2;
            }
        } else if constexpr (Q8) {
            u.load(raw, 0);
            if (!isfinite(gs)) return;
#pragma unroll 1
            for (; todo > 0; --todo) {
                u.unpack(raw, x);
                if (todo > 1) u.load(raw, STRIDE);   // on its way while this unit is worked on
                u.template step<SR>(x, half, lane, gs, a, lr, decay, key);
                u.advance(STRIDE);
                half += STRIDE / 2;
            }
        } else {
#pragma unroll 1
            for (; todo > 0; --todo) {
                u.load(raw, 0);
                if (!isfinite(gs)) return;
                u.unpack(raw, x);
                u.template step<SR>(x, half, lane, gs, a, lr, decay, key);
                u.advance(STRIDE);
                half += STRIDE / 2;
            }
        }
    } else if (ch.path == PATH_PLAIN) {
        if constexpr (Q8) step_plain<PT, GT, SR>(t, base, todo, warp, lane, gs, a, lr, decay, key, slots);
        else step_pairs<PATH_PLAIN, PT, GT, Q8, SR>(t, base, todo, lane, gs, a, lr, decay, key);
    } else if (ch.path == PATH_ROWS) {
        if constexpr (Q8) step_rows<PT, GT, SR>(t, base, todo, warp, lane, gs, a, lr, decay, key, slots);
        else step_pairs<PATH_ROWS, PT, GT, Q8, SR>(t, base, todo, lane, gs, a, lr, decay, key);
    } else {
        step_pairs<PATH_ANY, PT, GT, Q8, SR>(t, base, todo, lane, gs, a, lr, decay, key);
    }
}

// ---- norm -----------------------------------------------------------------------------------------------------------

// Sum of eight squares.  FP32 squares overflow above 1.8e19 and lose bits below 1e-19: where the FP32 sum is outside a
// range that rules both out, it is taken again in FP64 (the values are still in registers).
__device__ __forceinline__ double square_sum(float2 (&x)[4])
{
    float2 q = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < 4; ++j) q = fma2(x[j], x[j], q);
    const float s = __fadd_rn(q.x, q.y);
    if (s >= 1e-25f && s <= 1e37f) return (double)s;
    double d = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) d += (double)at(x, j) * (double)at(x, j);
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

// A warp's sum over its units of a chunk, without vectors.
template <int PATH, typename GT>
__device__ __forceinline__ double pairs_squares(const DenseRec &t, int64_t base, int todo, int lane)
{
    constexpr int64_t STRIDE = WARPS * UNIT;
    double sum = 0.0;
    int64_t row = 0, col = 0;
    if constexpr (PATH == PATH_ROWS) {
        row = base / t.cols;
        col = base - row * t.cols;
    }
#pragma unroll 4
    for (; todo > 0; --todo, base += STRIDE) {
        float2 g[4];
        load_matrix<PATH, true>((const GT *)t.g, t, t.ldg, base, row, col, lane, g);
        sum += square_sum(g);
        if constexpr (PATH == PATH_ROWS)
            for (col += STRIDE; col >= t.cols; col -= t.cols) ++row;
    }
    return sum;
}

// The same on any path; on the vector path, 64 bytes of every lane at a time.
template <typename GT>
__device__ __forceinline__ double chunk_squares(const DenseRec &t, const DenseChunk &ch, int warp, int lane)
{
    int64_t base = ((int64_t)ch.first + warp) * UNIT;
    int todo = (ch.units - warp + WARPS - 1) / WARPS;
    if (ch.path == PATH_PLAIN) return pairs_squares<PATH_PLAIN, GT>(t, base, todo, lane);
    if (ch.path == PATH_ROWS) return pairs_squares<PATH_ROWS, GT>(t, base, todo, lane);
    if (ch.path == PATH_ANY) return pairs_squares<PATH_ANY, GT>(t, base, todo, lane);
    constexpr int64_t STRIDE = WARPS * UNIT;
    constexpr int AT_ONCE = 64 / (8 * (int)sizeof(GT));
    double sum = 0.0;
    for (; todo > 0; todo -= AT_ONCE, base += AT_ONCE * STRIDE) {
        Eight<GT> r[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
            if (k < todo) r[k].load((const GT *)t.g + base + k * STRIDE + lane * 8);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if (k >= todo) break;
            float2 g[4];
            r[k].get(g);
            sum += square_sum(g);
        }
    }
    return sum;
}

__global__ void __launch_bounds__(WARPS * 32, NORM_CTAS)
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
        sum += (t.flags & REC_G_BF16) ? chunk_squares<bf16>(t, ch, warp, lane) : chunk_squares<float>(t, ch, warp, lane);
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

// VEC: whole units, moments of both sides aligned to vectors.
template <bool DQ, bool SQ, bool VEC>
__device__ __forceinline__ void copy_units(const DenseRec &d, const DenseRec &s, const DenseChunk &ch, int warp, int lane)
{
    const bool from_pairs = s.flags & REC_PAIR_STATE, to_pairs = d.flags & REC_PAIR_STATE;
    for (int k = warp; k < ch.units; k += WARPS) {
        const int64_t base = ((int64_t)ch.first + k) * UNIT, e = base + lane * 8;
        float2 m[4], v[4];
        float2 scale = make_float2(1.f, 1.f);
        uint2 cm, cr;
        if constexpr (SQ) {
            scale = s.scale[base / UNIT];
            cm = VEC ? load8((const uint8_t *)s.m + e) : load_code_pairs<false>(s.m, from_pairs, base, lane, d.n);
            cr = VEC ? load8((const uint8_t *)s.v + e) : load_code_pairs<false>(s.v, from_pairs, base, lane, d.n);
        } else if constexpr (VEC) {
            Eight<float> rm, rv;
            rm.load((const float *)s.m + e);
            rv.load((const float *)s.v + e);
            rm.get(m);
            rv.get(v);
        } else {
            load_pairs<false>(s.m, from_pairs, base, lane, d.n, m);
            load_pairs<false>(s.v, from_pairs, base, lane, d.n, v);
        }
        if constexpr (!DQ && SQ) {
            e4m3_unpack(cm, m);
            e4m3_unpack(cr, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                m[j] = mul2(m[j], pair(scale.x));
                v[j] = mul2(v[j], pair(scale.y));
                v[j] = mul2(v[j], v[j]);
            }
        } else if constexpr (DQ && !SQ) {
#pragma unroll
            for (int j = 0; j < 8; ++j) at(v, j) = -__fsqrt_rn(at(v, j));
            scale = quantise<false, true>(m, v, v, UnitKeys{0, 0}, EightFrom{0}, cm, cr);
        }
        if constexpr (DQ && VEC) {
            *(uint2 *)((uint8_t *)d.m + e) = cm;
            *(uint2 *)((uint8_t *)d.v + e) = cr;
        } else if constexpr (DQ) {
            store_code_pairs<false>(d.m, to_pairs, base, lane, d.n, cm);
            store_code_pairs<false>(d.v, to_pairs, base, lane, d.n, cr);
        } else if constexpr (VEC) {
            Eight<float>::put((float *)d.m + e, m);
            Eight<float>::put((float *)d.v + e, v);
        } else {
            store_pairs<false>(d.m, to_pairs, base, lane, d.n, m);
            store_pairs<false>(d.v, to_pairs, base, lane, d.n, v);
        }
        if (DQ && lane == 0) d.scale[base / UNIT] = scale;
    }
}
template <bool DQ, bool SQ>
__device__ __forceinline__ void copy_chunk(const DenseRec &d, const DenseRec &s, const DenseChunk &ch, int warp, int lane)
{
    if (ch.path == PATH_VECTORS && (d.flags & s.flags & REC_VEC_STATE)) copy_units<DQ, SQ, true>(d, s, ch, warp, lane);
    else copy_units<DQ, SQ, false>(d, s, ch, warp, lane);
}

__global__ void __launch_bounds__(WARPS * 32, COPY_CTAS)
dense_copy_state_kernel(const DenseRec *__restrict__ drecs, const DenseRec *__restrict__ srecs, const DenseChunk *__restrict__ chunks)
{
    pdl_trigger();
    const DenseChunk ch = chunks[blockIdx.x];
    const DenseRec &d = drecs[ch.rec];
    const DenseRec &s = srecs[ch.rec];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();
    if (d.flags & REC_Q8) {
        if (s.flags & REC_Q8) copy_chunk<true, true>(d, s, ch, warp, lane);
        else copy_chunk<true, false>(d, s, ch, warp, lane);
    } else {
        if (s.flags & REC_Q8) copy_chunk<false, true>(d, s, ch, warp, lane);
        else copy_chunk<false, false>(d, s, ch, warp, lane);
    }
}

}  // namespace tsr

using namespace tsr;

// ---- host side ------------------------------------------------------------------------------------------------------

struct tsr_dense_plan {
    std::vector<tsr_dense_desc> descs;
    DenseLayout layout;
    std::vector<DenseTable::Group> groups;
    int norm_first = 0, copy_first = 0, chunk_count = 0;
    size_t workspace_bytes = 0;
    bool bound = false;
    int device = -1, norm_ctas = 0;
    DenseRec *d_recs = nullptr;
    DenseChunk *d_chunks = nullptr;
    double *d_partial = nullptr;
    uint32_t *d_ticket = nullptr;
    mutable std::string err;
    explicit tsr_dense_plan(const std::vector<tsr_dense_desc> &d) : descs(d), layout(d) {}
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
        if (e__ != cudaSuccess) {                                                                               \
            (void)cudaGetLastError();   /* not left for the caller's next check */                             \
            return dense_fail(plan, TSR_ERR_CUDA, "%s failed: %s", #call, cudaGetErrorString(e__));             \
        }                                                                                                       \
    } while (0)

constexpr int64_t DENSE_MOST = (int64_t)1 << 40;   // elements of a tensor with its pitch; keeps products in 64 bits

template <typename PT, typename GT, bool Q8, bool SR>
cudaError_t step_launch_as(bool mixed, const DenseRec *recs, const DenseChunk *chunks, int count, const DenseStep &a, cudaStream_t s)
{
    const int smem = !has_ring<PT>(Q8, SR, mixed) ? 0 : mixed ? Ring<PT, GT, true>::BYTES : Ring<PT, GT, false>::BYTES;
    return mixed ? launch_dependent(dense_step_kernel<PT, GT, Q8, SR, true>, dim3(count), dim3(WARPS * 32), smem, s, 1, recs, chunks, a)
                 : launch_dependent(dense_step_kernel<PT, GT, Q8, SR, false>, dim3(count), dim3(WARPS * 32), smem, s, 1, recs, chunks, a);
}

template <typename PT, typename GT>
cudaError_t step_launch_as(bool q8, bool sr, bool mixed, const DenseRec *recs, const DenseChunk *chunks, int count, const DenseStep &a, cudaStream_t s)
{
    if (q8) return sr ? step_launch_as<PT, GT, true, true>(mixed, recs, chunks, count, a, s) : step_launch_as<PT, GT, true, false>(mixed, recs, chunks, count, a, s);
    if constexpr (sizeof(PT) == 2)   // (FP32 parameters with FP32 states: nothing is rounded)
        if (sr) return step_launch_as<PT, GT, false, true>(mixed, recs, chunks, count, a, s);
    return step_launch_as<PT, GT, false, false>(mixed, recs, chunks, count, a, s);
}

cudaError_t step_launch(int key, bool sr, bool mixed, const DenseRec *recs, const DenseChunk *chunks, int count, const DenseStep &a, cudaStream_t s)
{
    const bool q8 = key & KEY_Q8;
    switch (key & (KEY_P_BF16 | KEY_G_BF16)) {
    case 0: return step_launch_as<float, float>(q8, sr, mixed, recs, chunks, count, a, s);
    case KEY_P_BF16: return step_launch_as<bf16, float>(q8, sr, mixed, recs, chunks, count, a, s);
    case KEY_G_BF16: return step_launch_as<float, bf16>(q8, sr, mixed, recs, chunks, count, a, s);
    default: return step_launch_as<bf16, bf16>(q8, sr, mixed, recs, chunks, count, a, s);
    }
}

template <typename PT, typename GT, bool SR> cudaError_t step_configure_as()
{
    cudaError_t e = cudaSuccess;
    if (has_ring<PT>(true, SR, false))
        e = cudaFuncSetAttribute(dense_step_kernel<PT, GT, true, SR, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, Ring<PT, GT, false>::BYTES);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(dense_step_kernel<PT, GT, true, SR, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Ring<PT, GT, true>::BYTES);
}
template <typename PT, typename GT> cudaError_t step_configure()   // shared memory of the kernels with a ring
{
    const cudaError_t e = step_configure_as<PT, GT, false>();
    return e != cudaSuccess ? e : step_configure_as<PT, GT, true>();
}

tsr_status dense_ready(const tsr_dense_plan *plan)
{
    if (!plan->bound) return dense_fail(plan, TSR_ERR_NOT_BOUND, "tsr_dense_plan_bind has not been called");
    int dev = -1;
    DENSE_CUDA(plan, cudaGetDevice(&dev));
    if (dev != plan->device) return dense_fail(plan, TSR_ERR_INVALID_ARG, "the plan is bound on device %d, the current device is %d", plan->device, dev);
    return TSR_OK;
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
        const int64_t ps = dense_size_of(d.p_dtype), gs = dense_size_of(d.g_dtype);
        const bool q8 = d.state == TSR_STATE_Q8;
        if ((grad && !p.grad) || (state && (!p.m || !p.v || (q8 && !p.scale))) || (step && !p.param))
            return dense_fail(plan, TSR_ERR_INVALID_ARG, "tensor %zu: NULL pointer", i);
        if ((grad && !dense_aligned(p.grad, gs)) || (state && !q8 && (!dense_aligned(p.m, 4) || !dense_aligned(p.v, 4))) ||
            (state && q8 && !dense_aligned(p.scale, 8)) || (step && (!dense_aligned(p.param, ps) || !dense_aligned(p.image, 2))))
            return dense_fail(plan, TSR_ERR_ALIGNMENT, "tensor %zu: a buffer is not aligned to its element type", i);
        if (step && p.image && d.p_dtype != TSR_F32)
            return dense_fail(plan, TSR_ERR_INVALID_ARG, "tensor %zu: an image needs an FP32 parameter", i);
        if (step && p.image && (d.ldi < d.cols || d.ldi > DENSE_MOST / d.rows)) return dense_fail(plan, TSR_ERR_SHAPE, "tensor %zu: bad ldi", i);
        r.cols = d.cols; r.ldp = d.ldp; r.ldg = d.ldg; r.ldi = d.ldi;
        r.lr_mult = d.lr_mult; r.wd_mult = d.wd_mult;
        r.index = (int32_t)i;
        if (q8) r.flags |= REC_Q8;
        if (d.g_dtype == TSR_BF16) r.flags |= REC_G_BF16;
        bool contiguous = true;
        if (grad) {
            r.g = p.grad;
            contiguous = dense_grad_contiguous(d);
        }
        if (state) {
            r.m = p.m; r.v = p.v;
            const int64_t es = q8 ? 1 : 4;
            if (q8) r.scale = (float2 *)p.scale;
            if (DenseLayout::state_vectors(d, p)) r.flags |= REC_VEC_STATE;
            if (dense_aligned(p.m, 2 * es) && dense_aligned(p.v, 2 * es)) r.flags |= REC_PAIR_STATE;
        }
        if (step) {
            r.p = p.param;
            r.image = (bf16 *)p.image;
            contiguous = dense_step_contiguous(d, p.image != nullptr);
        }
        if (!contiguous) r.flags |= REC_PITCHED;
    }
    DenseTable table = plan->layout.fill(plan->descs, ptrs);
    const std::vector<DenseChunk> &chunks = table.chunks;
    if ((int64_t)chunks.size() > plan->layout.most_chunks)
        return dense_fail(plan, TSR_ERR_WORKSPACE, "the table has %zu chunks, the workspace holds %lld", chunks.size(), (long long)plan->layout.most_chunks);
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return dense_fail(plan, TSR_ERR_CUDA, "no CUDA device available");
    DENSE_CUDA(plan, cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    DENSE_CUDA(plan, (step_configure<float, float>()));
    DENSE_CUDA(plan, (step_configure<bf16, float>()));
    DENSE_CUDA(plan, (step_configure<float, bf16>()));
    DENSE_CUDA(plan, (step_configure<bf16, bf16>()));
    plan->bound = false;
    DENSE_CUDA(plan, cudaDeviceSynchronize());   // nothing that still runs may see the tables change
    char *at = (char *)workspace;
    plan->d_recs = (DenseRec *)at;
    at += round_up((int64_t)(recs.size() * sizeof(DenseRec)), 256);
    plan->d_chunks = (DenseChunk *)at;
    at += round_up(plan->layout.most_chunks * (int64_t)sizeof(DenseChunk), 256);
    plan->d_partial = (double *)at;
    at += NORM_CTAS * SMS * sizeof(double);
    plan->d_ticket = (uint32_t *)at;
    if (!recs.empty()) DENSE_CUDA(plan, cudaMemcpy(plan->d_recs, recs.data(), recs.size() * sizeof(DenseRec), cudaMemcpyHostToDevice));
    if (!chunks.empty()) DENSE_CUDA(plan, cudaMemcpy(plan->d_chunks, chunks.data(), chunks.size() * sizeof(DenseChunk), cudaMemcpyHostToDevice));
    DENSE_CUDA(plan, cudaMemset(plan->d_ticket, 0, sizeof(uint32_t)));
    DENSE_CUDA(plan, cudaDeviceSynchronize());
    plan->groups.swap(table.groups);
    plan->chunk_count = (int)chunks.size();
    plan->norm_first = table.norm_first;
    plan->copy_first = table.copy_first;
    plan->device = dev;
    plan->norm_ctas = NORM_CTAS * std::min(SMS, sms);
    plan->bound = true;
    return TSR_OK;
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
        total += 3 * ((d.rows * d.cols + WARPS * UNIT - 1) / (WARPS * UNIT) + 1);
        if (total > 0x7fffffff) return TSR_ERR_SHAPE;
    }
    try {
        tsr_dense_plan *plan = new tsr_dense_plan(std::vector<tsr_dense_desc>(descs, descs + count));
        plan->workspace_bytes = (size_t)(round_up((int64_t)(plan->descs.size() * sizeof(DenseRec)), 256) +
                                         round_up(plan->layout.most_chunks * (int64_t)sizeof(DenseChunk), 256) +
                                         NORM_CTAS * SMS * (int64_t)sizeof(double) + 256);
        *out = plan;
    } catch (...) {   // the host is out of memory
        return TSR_ERR_INVALID_ARG;
    }
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
    if (!dense_aligned(workspace, 256)) return dense_fail(plan, TSR_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
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
    if (!dense_aligned(grad_scale, 4)) return dense_fail(plan, TSR_ERR_ALIGNMENT, "grad_scale is not aligned to a float");
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
    for (const DenseTable::Group &g : plan->groups) {
        const DenseChunk *chunks = plan->d_chunks + g.first;
        DENSE_CUDA(plan, step_launch(g.key, rounding == TSR_ROUND_STOCHASTIC, g.mixed, plan->d_recs, chunks, g.count, a, (cudaStream_t)stream));
    }
    return TSR_OK;
}

tsr_status tsr_dense_plan_grad_norm(tsr_dense_plan *plan, float max_norm, float *out, void *stream)
{
    if (!plan) return TSR_ERR_INVALID_ARG;
    if (!out) return dense_fail(plan, TSR_ERR_INVALID_ARG, "out is NULL");
    if (!(max_norm > 0.f)) return dense_fail(plan, TSR_ERR_INVALID_ARG, "max_norm must be positive");
    if (!dense_aligned(out, 4)) return dense_fail(plan, TSR_ERR_ALIGNMENT, "out is not aligned to a float");
    tsr_status st = dense_ready(plan);
    if (st != TSR_OK) return st;
    const int count = plan->copy_first - plan->norm_first;
    const int ctas = std::max(1, std::min(plan->norm_ctas, count));
    DENSE_CUDA(plan, launch_dependent(dense_norm_kernel, dim3(ctas), dim3(WARPS * 32), 0, (cudaStream_t)stream, 1,
                                      (const DenseRec *)plan->d_recs, (const DenseChunk *)plan->d_chunks + plan->norm_first, count, max_norm,
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
    const int count = dst->chunk_count - dst->copy_first;
    if (dst == src || count == 0) return TSR_OK;
    DENSE_CUDA(dst, launch_dependent(dense_copy_state_kernel, dim3(count), dim3(WARPS * 32), 0, (cudaStream_t)stream, 1,
                                     (const DenseRec *)dst->d_recs, (const DenseRec *)src->d_recs, (const DenseChunk *)dst->d_chunks + dst->copy_first));
    return TSR_OK;
}

}  // extern "C"
