// Internal interface between the linear layer's host side (tsr_linear.cu) and its tensor-core kernel (tsr_linear_gemm.cu).
#pragma once
#include "tsr_layers.cuh"

namespace tsr {

struct LinearEpilogue {
    void *out;              // of the kernel's output type; split K: the FP32 slabs
    const void *res;        // the same type as out, may be out; NULL: none
    void *pre;              // the same type as out; NULL: none
    const void *bias;       // NULL: none
    int64_t ldo, ldr, ldp;
    int32_t bias_bf16, act;
    int32_t out_tma, res_tma, pre_tma;   // the matrix is described by a tensor map
    DropArgs drop;
};

struct alignas(64) LinearGemm {
    // operands: K-major boxes of 128 bytes x (128 or width / CG) rows, MN-major boxes of 64 entries x 64 rows, 128-byte swizzle;
    // out, residual and pre: boxes of 128 bytes x 32 rows, 128-byte swizzle
    CUtensorMap tmA, tmB, tmOut, tmRes, tmPre;
    int32_t M, N;
    int32_t kb_total, kb_per;            // K blocks of 128 bytes, and of them per split
    int32_t width, m_tiles, n_tiles, tiles;   // tile width (a multiple of 64), tiles in all (times splits)
    int32_t a_mn, b_mn, b_boxes;         // operand forms; MN-major boxes of B per CTA
    int32_t a_plane_rows, b_plane_rows;  // FP32: rows from the high to the low plane
    uint32_t stage_tx;                   // bytes of a stage, of all CTAs of a tile
    int32_t slab_rows;                   // split K: rows from one slab to the next
    int32_t whole_edge;                  // rows of out and pre may be written in whole 16-byte units
    LinearEpilogue e;
};

cudaError_t linear_gemm_launch(const LinearGemm &g, int cg, bool f32_operands, bool f32_out, int sms, cudaStream_t stream);
cudaError_t layer_status_read(int32_t *status, cudaStream_t stream);

}  // namespace tsr
