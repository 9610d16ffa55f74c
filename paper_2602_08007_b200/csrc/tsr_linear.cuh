// Internal interface between the linear layer's host side (tsr_linear.cu) and its tensor-core kernel (tsr_linear_gemm.cu).
#pragma once
#include "tsr_layers.cuh"

namespace tsr {

struct LinearEpilogue {
    void *out;              // of the kernel's output type
    const void *res;        // the same type as out, may be out; NULL: none
    void *pre;              // the same type as out; NULL: none
    const void *bias;       // NULL: none
    int64_t ldo, ldr, ldp;
    int32_t bias_bf16, act;
    int32_t out_tma, res_tma, pre_tma;   // the matrix is described by a tensor map
    DropArgs drop;
    float scale;            // of the product, where there is nothing but a residual besides; 1 otherwise
};

// Tiles of a product and the work items made of them: the first `whole` tiles one item each, the others `splits` items of kb_per K blocks.
struct LinearTiles {
    int32_t M, N;
    int32_t width, m_tiles, n_tiles;     // tile width, a multiple of 64
    int32_t whole, splits, items;
    int32_t kb_total, kb_per;            // K blocks (64 entries; 32 of FP32 operands)
};

struct alignas(64) LinearGemm : LinearTiles {
    // operands: K-major boxes of 64 entries x (128 or width / CG) rows, MN-major boxes of 64 x 64, 128-byte swizzle; of FP32 operands half as
    // much of K (K-major: 64-byte swizzle) of all three planes (third dimension); out, residual, pre and slabs: boxes of 128 bytes x 32 rows, 128-byte swizzle
    CUtensorMap tmA, tmB, tmOut, tmRes, tmPre, tmSlab;
    int32_t a_mn, b_mn, a_rows, a_boxes, b_boxes;   // operand forms; rows of a K-major box of A, MN-major boxes per CTA
    int32_t stages, stage_bytes, b_offset;   // the ring in shared memory
    uint32_t stage_tx;                   // bytes of a stage, of all CTAs of a tile
    int32_t whole_edge;                  // rows of out and pre may be written in whole 16-byte units
    struct { const bf16 *p; int64_t ld, plane; } parts[2];   // FP32 operands: where their planes lie
    int32_t K;
    LinearEpilogue e;
};

constexpr int LG_MAX_STAGES = 8;

struct LinearTile { int m0, n0, kb0, kb1, part, n_eff; };    // part: slab of the item, -1 for a whole tile

// Tiles in groups of eight rows of tiles, column by column: what runs at the same time shares operand rows in L2.
__host__ __device__ __forceinline__ void linear_tile_at(const LinearTiles &g, int t, int tile_m, int &m0, int &n0)
{
    const int per = 8 * g.n_tiles, grp = t / per, first = grp * 8, left = g.m_tiles - first, gm = left < 8 ? left : 8, in = t - grp * per;
    m0 = (first + in % gm) * tile_m;
    n0 = in / gm * g.width;
}
__device__ __forceinline__ LinearTile linear_tile(const LinearTiles &g, int item, int tile_m)
{
    LinearTile r;
    int t = item, split = 0;
    r.part = -1;
    r.kb0 = 0;
    r.kb1 = g.kb_total;
    if (item >= g.whole) {
        r.part = item - g.whole;
        const int tail = r.part / g.splits;
        split = r.part - tail * g.splits;
        t = g.whole + tail;
        r.kb0 = split * g.kb_per;
        r.kb1 = min(g.kb_total, r.kb0 + g.kb_per);
    }
    linear_tile_at(g, t, tile_m, r.m0, r.n0);
    r.n_eff = min(g.width, (g.N - r.n0 + 15) & ~15);
    return r;
}

int linear_stages(int stage_bytes, bool pre);      // how many stages of the ring fit beside the epilogue's boxes
cudaError_t linear_gemm_launch(const LinearGemm &g, int cg, bool f32_operands, bool f32_out, int sms, cudaStream_t stream);
cudaError_t linear_status_read(int32_t *status, cudaStream_t stream);

}  // namespace tsr
