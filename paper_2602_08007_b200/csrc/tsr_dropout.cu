// y = residual + dropout(x): one pass, bound by HBM (formulas in tsr.h; the random words in tsr_layers.cuh).  A thread takes eight
// neighbours of a row: four words, one key of the row.  Where rows do not start on 16 bytes, the eight are those that leave y as whole vectors, whatever
// the alignment of x and residual (then shifted into place); only the first and the last ones of a row go entry by entry.
// Measured: 32768 x 2048 BF16 with residual 63 us (6.4 TB/s, what a copy reaches); 16384 x 2047 without 44 us (28 for 2048; 106 entry by entry).
#include <algorithm>

#include "tsr_layers.cuh"

namespace tsr {

struct DropoutArgs {
    const void *x, *res;
    void *y;
    int64_t ldx, ldr, ldy, rows;
    int32_t cols, units;        // units of eight entries per row, the most of any row
    DropArgs drop;
};

// WHOLE: all rows start on 16 bytes and are multiples of eight entries.
template <typename T, bool WHOLE, bool RES>
__global__ void __launch_bounds__(256)
dropout_kernel(const DropoutArgs a)
{
    constexpr int A = 16 / (int)sizeof(T);
    pdl_trigger();
    pdl_wait();
    const uint32_t call_key = drop_call_key(a.drop);
    const int64_t total = a.rows * a.units;
    const bool small = total < ((int64_t)1 << 32);
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
        const int64_t r = small ? (int64_t)((uint32_t)u / (uint32_t)a.units) : u / a.units;
        T *y = (T *)a.y + r * a.ldy;
        const int c = (int)(u - r * a.units) * 8 - (WHOLE ? 0 : (int)((uintptr_t)y / sizeof(T) % A)), n = a.cols - c;
        if (!WHOLE && n <= 0) continue;
        const bool full = WHOLE || (c >= 0 && n >= 8);
        const T *x = (const T *)a.x + r * a.ldx + c;
        const T *res = (const T *)a.res + r * a.ldr + c;
        y += c;
        const DropRow key = drop_row_key(call_key, r);
        float v[8], o[8];
        if (WHOLE) {
            load8(x, v);
            if (RES) load8(res, o);
        } else if (full) {
            load8_any<false>(x, v);      // (y may be x or the residual)
            if (RES) load8_any<false>(res, o);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = c + j >= 0 && j < n;
                v[j] = in ? load_f(x + j) : 0.f;
                if (RES) o[j] = in ? load_f(res + j) : 0.f;
            }
        }
        // the words from column c on; of an odd column they begin with a word's high half
        uint32_t w[5];
#pragma unroll
        for (int j = 0; j < (WHOLE ? 4 : 5); ++j) w[j] = drop_word(key, (uint32_t)((c >> 1) + j));
        if (!WHOLE) {
            const uint32_t odd = (uint32_t)(c & 1) * 16u;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = __funnelshift_r(w[j], w[j + 1], odd);
        }
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            v[j] = drop_lo(w[j / 2], v[j], a.drop);
            v[j + 1] = drop_hi(w[j / 2], v[j + 1], a.drop);
            if (RES) { v[j] += o[j]; v[j + 1] += o[j + 1]; }
        }
        if (full) store8(y, v);
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j) if (c + j >= 0 && j < n) store_f(y + j, v[j]);
        }
    }
}

template <typename T>
static cudaError_t dropout_as(const DropoutArgs &a, bool whole, int sms, cudaStream_t s)
{
    const dim3 grid((unsigned)std::min<int64_t>((a.rows * a.units + 255) / 256, (int64_t)sms * 64));
    if (a.res) return whole ? launch_dependent(dropout_kernel<T, true, true>, grid, dim3(256), 0, s, 1, a) : launch_dependent(dropout_kernel<T, false, true>, grid, dim3(256), 0, s, 1, a);
    return whole ? launch_dependent(dropout_kernel<T, true, false>, grid, dim3(256), 0, s, 1, a) : launch_dependent(dropout_kernel<T, false, false>, grid, dim3(256), 0, s, 1, a);
}

}  // namespace tsr

using namespace tsr;

extern "C" tsr_status tsr_dropout(const tsr_dropout_desc *desc, int32_t dtype, int64_t rows, int64_t cols, tsr_matrix x, tsr_matrix residual, tsr_matrix y, void *stream)
{
    DropoutArgs a = {};
    if (!desc) return TSR_ERR_INVALID_ARG;
    if (!type_ok(dtype)) return TSR_ERR_UNSUPPORTED;
    if (rows < 0 || cols < 0 || rows > (int64_t)1 << 40 || cols > 0x7fffffff - 1023) return TSR_ERR_SHAPE;
    if (!drop_args(*desc, &a.drop)) return TSR_ERR_INVALID_ARG;
    const tsr_matrix *all[3] = {&x, &residual, &y};
    const int es = type_bytes(dtype);
    bool whole = cols % 8 == 0;
    for (int i = 0; i < 3; ++i) {
        const tsr_matrix &m = *all[i];
        if (!m.data) {
            if (i != 1 && rows > 0 && cols > 0) return TSR_ERR_INVALID_ARG;
            continue;
        }
        if (!extent_ok(rows, cols, m.ld)) return TSR_ERR_SHAPE;
        if (!aligned_to(m.data, es)) return TSR_ERR_ALIGNMENT;
        whole = whole && aligned_to(m.data, 16) && (rows <= 1 || m.ld * es % 16 == 0);
    }
    if (rows == 0 || cols == 0) return TSR_OK;
    const int sms = device_sms();
    if (!sms) return TSR_ERR_CUDA;
    a.x = x.data; a.ldx = x.ld; a.res = residual.data; a.ldr = residual.ld; a.y = y.data; a.ldy = y.ld;
    a.rows = rows; a.cols = (int)cols; a.units = (int)((cols + (whole ? 0 : 16 / es - 1) + 7) / 8);
    const cudaError_t e = dtype == TSR_BF16 ? dropout_as<bf16>(a, whole, sms, (cudaStream_t)stream) : dropout_as<float>(a, whole, sms, (cudaStream_t)stream);
    return e == cudaSuccess ? TSR_OK : TSR_ERR_CUDA;
}
