// What the layer operators (norm, linear, dropout) share: the random words of dropout, activations and their slopes, typed
// loads and stores, and the sum of column partials.
#pragma once
#include "tsr_device.cuh"
#include "tsr_internal.h"
#include "tsr_pdl.cuh"
#include "tsr_umma.cuh"

namespace tsr {

// ---- dropout ----------------------------------------------------------------------------------------------------------
//
// Entry (row, col) of a matrix falls iff its 16 random bits are below threshold = round(65536 p); the others are multiplied by
// 65536 / (65536 - threshold), so that the mean is kept for the probability that is drawn.  Two entries share a 32-bit word, a function of
// (seed, offset, row, col / 2) alone: every kernel that holds an entry, in whatever layout, draws the same bits, and no mask
// is stored.  A row has two keys, as the rows' words would otherwise be shifted copies of one sequence.
struct DropArgs {
    uint32_t threshold;      // 0: nothing falls (and nothing is drawn); 65536: everything
    float scale;
    uint32_t seed_key;       // from the seed, on the host
    uint64_t offset;
    const int64_t *step;     // NULL, or a device word added to offset when the kernel runs
};
struct DropRow { uint32_t k1, k2; };

__device__ __forceinline__ uint32_t drop_call_key(const DropArgs &d)
{
    const uint64_t o = d.offset + (d.step ? (uint64_t)*(const volatile int64_t *)d.step : 0ull);
    const uint32_t k = mix32(d.seed_key ^ mix32((uint32_t)o + 0x7f4a7c15u));
    return mix32(k ^ ((uint32_t)(o >> 32) * 0x85ebca77u));
}
__device__ __forceinline__ DropRow drop_row_key(uint32_t call_key, int64_t row)
{
    DropRow r;
    r.k1 = mix32(call_key ^ mix32((uint32_t)row + 0x9e3779b9u * ((uint32_t)((uint64_t)row >> 32) + 1u)));
    r.k2 = mix32(r.k1 ^ 0xa511e9b3u);
    return r;
}
// The word of columns 2 c and 2 c + 1 (low and high half).
__device__ __forceinline__ uint32_t drop_word(const DropRow &r, uint32_t c)
{
    uint32_t x = c + r.k1;
    x ^= x >> 16;
    x *= 0x85ebca6bu;
    x = x ^ (x >> 13) ^ r.k2;
    x *= 0xc2b2ae35u;
    return x ^ (x >> 16);
}
// A selection, not a product with zero: an entry that falls is zero whatever it was.
__device__ __forceinline__ float drop_lo(uint32_t w, float x, const DropArgs &d) { return (w & 0xffffu) < d.threshold ? 0.f : x * d.scale; }
__device__ __forceinline__ float drop_hi(uint32_t w, float x, const DropArgs &d) { return (w >> 16) < d.threshold ? 0.f : x * d.scale; }
__device__ __forceinline__ float drop_entry(const DropRow &r, uint32_t col, float x, const DropArgs &d)
{
    const uint32_t w = drop_word(r, col >> 1);
    return (col & 1u) ? drop_hi(w, x, d) : drop_lo(w, x, d);
}

// Host: checks and prepares; false on a bad probability.
bool drop_args(const tsr_dropout_desc &d, DropArgs *out);

// ---- activations ------------------------------------------------------------------------------------------------------
// BF16 layers: the exponential and the reciprocal come from the special-function units (2^-22 of the value, and for the exponential 2^-24 of the argument on
// top), in kernels bound by instructions; the result is rounded to 2^-9.  FP32 layers take the longer forms further down.
__device__ __forceinline__ float rcp_f(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float exp_f(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * 1.44269504f));
    return y;
}
__device__ __forceinline__ float sigmoid_f(float x) { return rcp_f(1.f + exp_f(-x)); }
// Limits |x| to `most`; NaN stays.
__device__ __forceinline__ float limited(float x, float most)
{
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(x), "f"(-most));
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(x), "f"(most));
    return x;
}

// ---- pairs (mul2, fma2: tsr_device.cuh) -----------------------------------------------------------------------------
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    unsigned long long d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits_of(a)), "l"(bits_of(b)));
    return *(const float2 *)&d;
}

// Normal distribution: Phi(z) and e = exp(-z^2 / 2).  The tail is t (a1 + t (a2 + ... a5 t^4)) e / 2 with t = 1 / (1 + p |z| / sqrt 2), formula 7.1.26 of
// Abramowitz and Stegun's handbook (C. Hastings): off by 0.75e-7 at most, with two uses of the special-function units and half of the instructions
// of erff, which bound the epilogue of a GELU layer.
__device__ __forceinline__ float normal_cdf(float z, float &e)
{
    const float t = rcp_f(fmaf(0.23164190f, fabsf(z), 1.f));
    e = exp_f(-0.5f * z * z);
    const float tail = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5307027145f, -0.7265760135f), 0.7107068705f), -0.142248368f), 0.127414796f) * e;
    return z >= 0.f ? 1.f - tail : tail;
}

// Two values at a time, for epilogues that are bound by instructions.
template <int ACT>
__device__ __forceinline__ float2 act_pair(float2 z)
{
    const auto logistic = [](float2 x) {      // 1 / (1 + 2^x)
        float2 e;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(x.x));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(x.y));
        e = add2(e, pair(1.f));
        return make_float2(rcp_f(e.x), rcp_f(e.y));
    };
    if constexpr (ACT == TSR_ACT_RELU) return make_float2(z.x < 0.f ? 0.f : z.x, z.y < 0.f ? 0.f : z.y);      // (NaN stays)
    else if constexpr (ACT == TSR_ACT_SILU) return mul2(z, logistic(mul2(z, pair(-1.44269504f))));
    else if constexpr (ACT == TSR_ACT_GELU_TANH)      // (1 + tanh u) / 2 = 1 / (1 + e^(-2 u))
        return mul2(z, logistic(mul2(z, fma2(mul2(z, z), pair(-0.102943240f), pair(-2.30220819f)))));
    else if constexpr (ACT == TSR_ACT_GELU) {
        // z Phi(z) = max(z, 0) - |z| tail(|z|), the tail as in normal_cdf; an infinite z above zero keeps its tail finite
        const float2 a = make_float2(fabsf(z.x == INFINITY ? 3e38f : z.x), fabsf(z.y == INFINITY ? 3e38f : z.y));
        float2 t = fma2(a, pair(0.23164190f), pair(1.f)), e = mul2(mul2(a, a), pair(-0.72134752f));
        t = make_float2(rcp_f(t.x), rcp_f(t.y));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(e.x));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(e.y));
        float2 p = fma2(t, pair(0.5307027145f), pair(-0.7265760135f));
        p = fma2(t, p, pair(0.7107068705f));
        p = fma2(t, p, pair(-0.142248368f));
        p = fma2(t, p, pair(0.127414796f));
        p = mul2(mul2(p, t), mul2(e, make_float2(-a.x, -a.y)));
        return add2(make_float2(fmaxf(z.x, 0.f), fmaxf(z.y, 0.f)), p);
    } else return z;
}
__device__ __forceinline__ float act_approx(int act, float z)
{
    switch (act) {
    case TSR_ACT_RELU: return z < 0.f ? 0.f : z;      // (NaN stays)
    case TSR_ACT_GELU: return act_pair<TSR_ACT_GELU>(pair(z)).x;
    case TSR_ACT_GELU_TANH: return z * sigmoid_f(1.59576912f * fmaf(0.044715f * z * z, z, z));   // (1 + tanh u) / 2 = sigmoid(2 u)
    case TSR_ACT_SILU: return z * sigmoid_f(z);
    default: return z;
    }
}
// Derivative.  Beyond the limits it is 0 or 1, and products of an infinity with zero are kept out; NaN stays.
__device__ __forceinline__ float slope_approx(int act, float z)
{
    switch (act) {
    case TSR_ACT_RELU: return z > 0.f ? 1.f : z != z ? z : 0.f;
    case TSR_ACT_GELU: {
        const float c = limited(z, 16.f);
        float e;
        const float cdf = normal_cdf(c, e);
        return fmaf(c * 0.39894228f, e, cdf);
    }
    case TSR_ACT_GELU_TANH: {
        const float c = limited(z, 16.f), c2 = c * c;
        const float g = sigmoid_f(1.59576912f * fmaf(0.044715f * c2, c, c));
        return fmaf(c * g * (1.f - g), 1.59576912f * fmaf(0.134145f, c2, 1.f), g);
    }
    case TSR_ACT_SILU: {
        const float c = limited(z, 1e30f), g = sigmoid_f(c);
        return g * fmaf(c, 1.f - g, 1.f);
    }
    default: return 1.f;
    }
}

// FP32 layers, two values at a time: within a few units of the last place.  2^(x c) from the special-function unit, whose argument in FP32 would be off by
// 2^-24 of itself: the rest of the product, x c - h, is multiplied on (c2: what c leaves of its constant).  |x c| stays below 128.
__device__ __forceinline__ float2 exp2_full(float2 x, float c, float c2)
{
    const float2 h = mul2(x, pair(c)), l = fma2(x, pair(c2), fma2(x, pair(c), mul2(h, pair(-1.f))));
    float2 e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(h.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(h.y));
    return fma2(e, mul2(l, pair(0.693147181f)), e);
}
__device__ __forceinline__ float2 limited(float2 x, float most) { return make_float2(limited(x.x, most), limited(x.y, most)); }
// e^-x; beyond 88.6 the logistic function is zero and one (a reciprocal below 2^-126 is flushed).
__device__ __forceinline__ float2 exp_minus(float2 x) { return exp2_full(limited(x, 88.6f), -1.44269504f, -1.92596303e-8f); }
// 1 / x with a step of Newton's method behind the special-function unit.
__device__ __forceinline__ float2 rcp_full(float2 x)
{
    const float2 r = make_float2(rcp_f(x.x), rcp_f(x.y));
    return fma2(r, fma2(mul2(x, pair(-1.f)), r, pair(1.f)), r);
}
__device__ __forceinline__ float2 logistic_full(float2 x) { return rcp_full(add2(pair(1.f), exp_minus(x))); }
// Phi(z) and e = exp(-z^2 / 2), |z| <= 16.  Up to |z| = 1 by 1/2 + z Q(z^2), beyond by the tail t P(t) e with t = 1 / (1 + 0.4 |z|), Hastings' form with eight
// terms, which keeps its digits far below zero.  (Q and P fitted by least squares with Lawson's weights: 3e-10, and 4e-8 of the tail.)
__device__ __forceinline__ float2 normal_cdf_full(float2 z, float2 &e)
{
    const float2 s = mul2(z, z), t = rcp_full(fma2(make_float2(fabsf(z.x), fabsf(z.y)), pair(0.4f), pair(1.f)));
    e = exp2_full(s, -0.721347520f, -9.62981516e-9f);
    float2 p = fma2(t, pair(-0.0375880674f), pair(0.190647230f)), q = fma2(s, pair(-7.66467929e-6f), pair(1.13512659e-4f));
    p = fma2(t, p, pair(-0.352870584f));
    q = fma2(s, q, pair(-1.18635304e-3f));
    p = fma2(t, p, pair(0.227039829f));
    q = fma2(s, q, pair(9.97333135e-3f));
    p = fma2(t, p, pair(0.00408836780f));
    q = fma2(s, q, pair(-0.0664903596f));
    p = fma2(t, p, pair(0.151508555f));
    q = fma2(s, q, pair(0.398942292f));
    p = fma2(t, p, pair(0.157496333f));
    q = fma2(z, q, pair(0.5f));
    p = mul2(mul2(fma2(t, p, pair(0.159678325f)), t), e);
    const float2 r = add2(pair(1.f), mul2(p, pair(-1.f)));
    return make_float2(s.x <= 1.f ? q.x : z.x > 0.f ? r.x : p.x, s.y <= 1.f ? q.y : z.y > 0.f ? r.y : p.y);
}
template <int ACT>
__device__ __forceinline__ float2 act_pair_full(float2 z)
{
    if constexpr (ACT == TSR_ACT_GELU) {
        float2 e;
        return mul2(z, normal_cdf_full(limited(z, 16.f), e));
    } else if constexpr (ACT == TSR_ACT_GELU_TANH) return mul2(z, logistic_full(mul2(pair(1.59576912f), fma2(mul2(mul2(z, z), pair(0.044715f)), z, z))));
    else if constexpr (ACT == TSR_ACT_SILU) return mul2(z, logistic_full(z));
    else return act_pair<ACT>(z);
}
template <int ACT>
__device__ __forceinline__ float2 slope_pair_full(float2 z)
{
    if constexpr (ACT == TSR_ACT_GELU) {
        const float2 c = limited(z, 16.f);
        float2 e;
        const float2 cdf = normal_cdf_full(c, e);
        return fma2(mul2(c, pair(0.39894228f)), e, cdf);
    } else if constexpr (ACT == TSR_ACT_GELU_TANH) {
        const float2 c = limited(z, 16.f), c2 = mul2(c, c), g = logistic_full(mul2(pair(1.59576912f), fma2(mul2(c2, pair(0.044715f)), c, c)));
        return fma2(mul2(mul2(c, g), fma2(g, pair(-1.f), pair(1.f))), mul2(pair(1.59576912f), fma2(pair(0.134145f), c2, pair(1.f))), g);
    } else if constexpr (ACT == TSR_ACT_SILU) {
        const float2 c = limited(z, 1e30f), g = logistic_full(c);
        return mul2(g, fma2(c, fma2(g, pair(-1.f), pair(1.f)), pair(1.f)));
    } else return make_float2(slope_approx(ACT, z.x), slope_approx(ACT, z.y));
}
__device__ __forceinline__ float act_full(int act, float z)
{
    switch (act) {
    case TSR_ACT_RELU: return act_pair_full<TSR_ACT_RELU>(pair(z)).x;
    case TSR_ACT_GELU: return act_pair_full<TSR_ACT_GELU>(pair(z)).x;
    case TSR_ACT_GELU_TANH: return act_pair_full<TSR_ACT_GELU_TANH>(pair(z)).x;
    case TSR_ACT_SILU: return act_pair_full<TSR_ACT_SILU>(pair(z)).x;
    default: return z;
    }
}
// T: the layer's type.
template <typename T>
__device__ __forceinline__ float act_value(int act, float z) { return sizeof(T) == 4 ? act_full(act, z) : act_approx(act, z); }
template <typename T, int ACT>
__device__ __forceinline__ float2 slope_pair(float2 z)
{
    if constexpr (sizeof(T) == 4) return slope_pair_full<ACT>(z);
    else return make_float2(slope_approx(ACT, z.x), slope_approx(ACT, z.y));
}

// ---- typed access -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ float load_f(const float *p) { return *p; }
__device__ __forceinline__ float load_f(const bf16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ float load_as(const void *p, int64_t i, bool is_bf16)
{
    return is_bf16 ? __bfloat162float(((const bf16 *)p)[i]) : ((const float *)p)[i];
}
__device__ __forceinline__ void store_as(void *p, int64_t i, bool is_bf16, float v)
{
    if (is_bf16) ((bf16 *)p)[i] = __float2bfloat16_rn(v);
    else ((float *)p)[i] = v;
}
__device__ __forceinline__ void store_f(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_f(bf16 *p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *(const uint32_t *)&h;
}
// Eight consecutive entries; p aligned to 16 bytes.
__device__ __forceinline__ void unpack8(const uint4 &r, float (&v)[8])
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void load8(const bf16 *p, float (&v)[8]) { unpack8(*(const uint4 *)p, v); }
__device__ __forceinline__ void load8(const float *p, float (&v)[8])
{
    const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store8(bf16 *p, const float (&v)[8])
{
    *(uint4 *)p = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]);
    *(float4 *)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// 16 bytes that begin m bytes (an even number) into a and reach into b: by one word, by two words, by half a word; selections, since code for each place
// (four of them, side by side on an SM) starved the warps of instructions.
__device__ __forceinline__ uint4 shift16(const uint4 &a, const uint4 &b, uint32_t m)
{
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t t[7], u[5];
#pragma unroll
    for (int i = 0; i < 7; ++i) t[i] = m & 4u ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) u[i] = m & 8u ? t[i + 2] : t[i];
    const uint32_t s = (m & 2u) * 8u;
    return make_uint4(__funnelshift_r(u[0], u[1], s), __funnelshift_r(u[1], u[2], s), __funnelshift_r(u[2], u[3], s), __funnelshift_r(u[3], u[4], s));
}
// Eight entries from an address of any alignment: the two 16-byte granules that hold them (each holds one of them at least, so neither
// lies outside of what may be read), shifted into place.  NC: nobody writes there while the kernel runs.
template <bool NC = true>
__device__ __forceinline__ uint4 load16_any(const bf16 *p)
{
    const uint32_t m = (uint32_t)(uintptr_t)p & 15u;
    const uint4 *base = (const uint4 *)((uintptr_t)p & ~(uintptr_t)15);
    const uint4 a = NC ? __ldg(base) : *base;
    return m == 0 ? a : shift16(a, NC ? __ldg(base + 1) : base[1], m);
}
// The same of FP32 entries: plain loads, whose address a vector of four may not fit.
template <bool NC = true>
__device__ __forceinline__ void load8_any(const bf16 *p, float (&v)[8]) { unpack8(load16_any<NC>(p), v); }
template <bool NC = true>
__device__ __forceinline__ void load8_any(const float *p, float (&v)[8])
{
    if (((uintptr_t)p & 15) == 0) {
        const float4 a = NC ? __ldg((const float4 *)p) : *(const float4 *)p, b = NC ? __ldg((const float4 *)p + 1) : ((const float4 *)p)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = NC ? __ldg(p + i) : p[i];
    }
}
// ... of which n < 8 exist; the others are zero.
template <typename T>
__device__ __forceinline__ void load8_part(const T *p, int n, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? load_f(p + i) : 0.f;
}

// A float in the shared memory of the cluster's CTA `rank`, at the place of `here` (between cluster barriers, which order it).
__device__ __forceinline__ float shared_of(const float *here, int rank)
{
    uint32_t at;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(here)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at));
    return v;
}

// ---- host helpers -----------------------------------------------------------------------------------------------------
inline int type_bytes(int32_t dtype) { return dtype == TSR_BF16 ? 2 : 4; }
inline bool type_ok(int32_t dtype) { return dtype == TSR_F32 || dtype == TSR_BF16; }
inline bool aligned_to(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
// a pitch that a tensor map can hold, and rows * ld entries that stay addressable in 63 bits
inline bool extent_ok(int64_t rows, int64_t cols, int64_t ld)
{
    return ld >= cols && ld < ((int64_t)1 << 37) && (rows <= 1 || rows <= ((int64_t)1 << 56) / (ld > 0 ? ld : 1));
}

cudaError_t norm_status_read(int32_t *status, cudaStream_t stream);
int device_sms();   // multiprocessors of the current device (looked up once per device); 0 without one

// Sums of column partials: out[c] (= or +=) sum over p < parts of partial[p * ldp + c], in order of p.  Two sets at once (out2 may
// be NULL; its partials follow the first set's `parts` rows).
cudaError_t column_finish(const float *partial, int parts, int64_t ldp, int64_t cols, void *out, bool out_bf16, void *out2, bool out2_bf16,
                          bool accumulate, cudaStream_t stream);

}  // namespace tsr
