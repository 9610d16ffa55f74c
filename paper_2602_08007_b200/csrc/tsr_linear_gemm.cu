// Products of the linear layer on the 5th-generation tensor cores, with the layer's epilogue (formulas in tsr.h).
//
//   D[M x N] = A[M x K] B[N x K]^T,   then per entry  z = D + bias;  pre = z;  out = residual + dropout(act(z))
//
// One persistent CTA per SM (CG = 1, tiles of 128 x width) or one pair of CTAs per two SMs (CG = 2, 256 x width, tcgen05 with
// cta_group::2).  Either operand is K-major or MN-major (a row-major matrix contracted over its rows, read as it lies), so
// that x W^T, dz W and dz^T x need no transposed copies.  Roles, as in the grouped GEMM of the optimizer: warp 0 loads
// A, warp 2 loads B (each CTA of a pair its half of the tile's B rows, no multicast), warp 1 issues the MMAs into one of two
// accumulators in tensor memory, warps 4 to 11 run the epilogue of one tile beside the MMAs of the next.
//
// Epilogue: a lane holds a row.  A warp's 32 rows x 128 bytes of output form a box in shared memory (128-byte swizzle: free of bank
// conflicts when the lanes walk their rows), of which it has two, and a third for pre.  The residual is fetched into the box by TMA
// while the MMAs still run, the result replaces it in place, and the box leaves by TMA.  Matrices whose pitch or address TMA
// does not take go between box and memory by plain row accesses instead; the arithmetic is the same.
// K split over several CTAs: each stores its FP32 slab, and linear_finish_kernel adds the slabs in order and runs the epilogue.
//
// What bounds it: an SM takes in 64 bytes of operands a clock, which 256 x 256 tiles of a pair just feed (64 bytes per clock of MMA);
// narrower tiles are bound by that intake.  Every mbarrier wait is bounded; on expiry the CTA notes it in the status
// word, stops storing, waits for copies in flight, frees its tensor memory and returns.
#include "tsr_linear.cuh"
#include "tsr_umma.cuh"

namespace tsr {

constexpr int LG_THREADS = 384, LG_EPI_WARPS = 8;
__device__ int g_layer_status;

template <int PLANES>
struct LinearSmem {
    static constexpr int P = PLANES == 3 ? 2 : 1;              // operand planes: FP32 data as high and low TF32 parts
    static constexpr int A_BYTES = UM_BM * 128, B_BYTES = UM_BM * 128;   // one plane; at most 128 rows of B per CTA
    static constexpr int STAGE_BYTES = P * (A_BYTES + B_BYTES);
    static constexpr int STAGES = PLANES == 3 ? 2 : 4;
    static constexpr int BOX_BYTES = 4096, BOXES = 3;          // per epilogue warp: two for the result, one for pre
    static constexpr int BOX_OFFSET = STAGES * STAGE_BYTES;
    static constexpr int BAR_OFFSET = BOX_OFFSET + LG_EPI_WARPS * BOXES * BOX_BYTES;
    static constexpr int NBARS = 2 * STAGES + 4 + 2 * LG_EPI_WARPS;
    static constexpr int TOTAL = BAR_OFFSET + NBARS * 8 + 16 + 1024;   // + slack for 1024-byte alignment
};
static_assert(LinearSmem<1>::TOTAL <= 227 * 1024 && LinearSmem<3>::TOTAL <= 227 * 1024, "shared memory of an SM");

__device__ __forceinline__ void tc_mma_tf32(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::tf32 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

struct LinearTile { int m0, n0, kb0, kb1, split, n_eff; };

// Tiles in groups of eight rows of tiles, column by column: what runs at the same time shares operand rows in L2.
__device__ __forceinline__ LinearTile linear_tile(const LinearGemm &g, int t, int tile_m)
{
    LinearTile r;
    const int per_split = g.m_tiles * g.n_tiles;
    r.split = t / per_split;
    t -= r.split * per_split;
    const int per = 8 * g.n_tiles, grp = t / per, first = grp * 8, gm = min(8, g.m_tiles - first), in = t - grp * per;
    r.m0 = (first + in % gm) * tile_m;
    r.n0 = in / gm * g.width;
    r.kb0 = r.split * g.kb_per;
    r.kb1 = min(g.kb_total, r.kb0 + g.kb_per);
    r.n_eff = min(g.width, (g.N - r.n0 + 15) & ~15);
    return r;
}

// bias of 32 columns from col on, added to v (columns beyond N are left alone)
__device__ __forceinline__ void add_bias(float (&v)[32], const LinearEpilogue &e, int col, int N)
{
    if (e.bias_bf16) {
        const bf16 *b = (const bf16 *)e.bias + col;
        if (col + 32 <= N && ((uintptr_t)b & 15) == 0) {
#pragma unroll
            for (int j = 0; j < 32; j += 8) {
                float x[8];
                unpack8(__ldg((const uint4 *)(b + j)), x);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[j + i] += x[i];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) if (col + j < N) v[j] += __bfloat162float(b[j]);
        }
    } else {
        const float *b = (const float *)e.bias + col;
        if (col + 32 <= N && ((uintptr_t)b & 15) == 0) {
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const float4 x = __ldg((const float4 *)(b + j));
                v[j] += x.x; v[j + 1] += x.y; v[j + 2] += x.z; v[j + 3] += x.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) if (col + j < N) v[j] += b[j];
        }
    }
}

__device__ __forceinline__ void activate(float (&v)[32], int act)
{
    switch (act) {   // outside of the loop over the columns
    case TSR_ACT_RELU:
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = act_value(TSR_ACT_RELU, v[j]);
        break;
    case TSR_ACT_GELU:
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = act_value(TSR_ACT_GELU, v[j]);
        break;
    case TSR_ACT_GELU_TANH:
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = act_value(TSR_ACT_GELU_TANH, v[j]);
        break;
    case TSR_ACT_SILU:
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = act_value(TSR_ACT_SILU, v[j]);
        break;
    default: break;
    }
}

// A lane's row of a box: 16-byte unit u of row r lies at r * 128 + ((u ^ (r & 7)) << 4).
__device__ __forceinline__ uint4 *box_unit(uint8_t *box, int row, int u) { return (uint4 *)(box + row * 128 + ((u ^ (row & 7)) << 4)); }

// Between a box and a matrix that TMA does not take: one row after another, the lanes side by side.
template <bool F32>
__device__ __forceinline__ void box_from_rows(uint8_t *box, const void *src, int64_t ld, int nrows, int ncols, int lane)
{
    constexpr int CW = F32 ? 32 : 64;
#pragma unroll 4
    for (int r = 0; r < nrows; ++r) {
#pragma unroll
        for (int c = lane; c < CW; c += 32) {
            if (F32) {
                const float x = c < ncols ? ((const float *)src)[r * ld + c] : 0.f;
                *(float *)((uint8_t *)box_unit(box, r, c >> 2) + (c & 3) * 4) = x;
            } else {
                const bf16 x = c < ncols ? ((const bf16 *)src)[r * ld + c] : __float2bfloat16_rn(0.f);
                *(bf16 *)((uint8_t *)box_unit(box, r, c >> 3) + (c & 7) * 2) = x;
            }
        }
    }
}
template <bool F32>
__device__ __forceinline__ void box_to_rows(uint8_t *box, void *dst, int64_t ld, int nrows, int ncols, int lane)
{
    constexpr int CW = F32 ? 32 : 64;
#pragma unroll 4
    for (int r = 0; r < nrows; ++r) {
#pragma unroll
        for (int c = lane; c < CW; c += 32) {
            if (c >= ncols) continue;
            if (F32) ((float *)dst)[r * ld + c] = *(float *)((uint8_t *)box_unit(box, r, c >> 2) + (c & 3) * 4);
            else ((bf16 *)dst)[r * ld + c] = *(bf16 *)((uint8_t *)box_unit(box, r, c >> 3) + (c & 7) * 2);
        }
    }
}

template <int CG, int PLANES, bool F32>
__global__ void __cluster_dims__(CG, 1, 1) __launch_bounds__(LG_THREADS, 1)
linear_gemm_kernel(const __grid_constant__ LinearGemm g)
{
    using SM = LinearSmem<PLANES>;
    constexpr int STAGES = SM::STAGES, TILE_M = CG * UM_BM, P = SM::P;
    constexpr uint32_t TMEM_COLS = CG == 2 ? 512 : 256, ACC_COLS = TMEM_COLS / 2;
    constexpr int BK = PLANES == 3 ? 32 : 64;        // entries of a 128-byte K block

    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint64_t *bars = (uint64_t *)(smem + SM::BAR_OFFSET);
    uint64_t *bar_full = bars, *bar_empty = bars + STAGES;
    uint64_t *bar_acc_full = bars + 2 * STAGES, *bar_acc_empty = bar_acc_full + 2, *bar_res = bar_acc_empty + 2;
    uint32_t *tmem_slot = (uint32_t *)(bars + SM::NBARS);
    __shared__ int s_timeout;

    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long budget = UM_WAIT_CLOCKS;
    const uint32_t rank = CG == 2 ? cluster_ctarank() : 0u;
    const int first = CG == 2 ? (int)(blockIdx.x >> 1) : (int)blockIdx.x, stride = CG == 2 ? (int)(gridDim.x >> 1) : (int)gridDim.x;

    if (threadIdx.x == 0) {
        s_timeout = 0;
        for (int s = 0; s < STAGES; ++s) { mbar_init(smem_u32(bar_full + s), 1); mbar_init(smem_u32(bar_empty + s), 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(bar_acc_full + b), 1); mbar_init(smem_u32(bar_acc_empty + b), CG * LG_EPI_WARPS); }
        for (int b = 0; b < 2 * LG_EPI_WARPS; ++b) mbar_init(smem_u32(bar_res + b), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if constexpr (CG == 2)
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
        else
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();      // the peer's barriers are initialised before anything signals them
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    if (warp == 1) {   // (only now, when both CTAs of a pair hold their columns: the permit belongs to the pair)
        if constexpr (CG == 2) asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        else asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();

    if (warp == 0 || warp == 2) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            const bool is_a = warp == 0;
            const bool mn = PLANES == 1 && (is_a ? g.a_mn : g.b_mn);
            const int boxes = is_a ? 2 : g.b_boxes, plane_rows = is_a ? g.a_plane_rows : g.b_plane_rows;
            const CUtensorMap *map = is_a ? &g.tmA : &g.tmB;
            const uint32_t base = smem_u32(smem) + (is_a ? 0 : P * SM::A_BYTES);
            for (int t = first; ok && t < g.tiles; t += stride) {
                const LinearTile tile = linear_tile(g, t, TILE_M);
                const int row = is_a ? tile.m0 + (int)rank * UM_BM : tile.n0 + (int)rank * (tile.n_eff / CG);
                for (int kb = tile.kb0; kb < tile.kb1; ++kb) {
                    if (!mbar_wait(smem_u32(bar_empty + stage), phase ^ 1u, budget)) { s_timeout = 1; ok = false; break; }
                    // the copies of both CTAs of a pair report their bytes to the leader's barrier
                    const uint32_t full = CG == 2 ? leader_addr(smem_u32(bar_full + stage)) : smem_u32(bar_full + stage);
                    if (is_a && rank == 0) mbar_expect_tx(smem_u32(bar_full + stage), g.stage_tx);
                    const uint32_t st = base + stage * SM::STAGE_BYTES;
                    const int kx = kb * BK;
                    if (mn) {
                        for (int j = 0; j < boxes; ++j) {
                            if constexpr (CG == 2) tma_load_2d_pair(st + j * 8192, map, full, row + 64 * j, kx);
                            else tma_load_2d(st + j * 8192, map, full, row + 64 * j, kx);
                        }
                    } else {
#pragma unroll
                        for (int pl = 0; pl < P; ++pl) {
                            if constexpr (CG == 2) tma_load_2d_pair(st + pl * SM::A_BYTES, map, full, kx, row + pl * plane_rows);
                            else tma_load_2d(st + pl * SM::A_BYTES, map, full, kx, row + pl * plane_rows);
                        }
                    }
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            uint32_t tc = 0, phase = 0;
            int stage = 0;
            bool ok = true;
            const uint64_t a_hi = g.a_mn ? UMMA_DESC_HI_MN : UMMA_DESC_HI_K, b_hi = g.b_mn ? UMMA_DESC_HI_MN : UMMA_DESC_HI_K;
            const uint32_t a_step = g.a_mn ? 2048u : 32u, b_step = g.b_mn ? 2048u : 32u;
            const uint32_t form = (g.a_mn ? UMMA_IDESC_A_MN_MAJOR : 0u) | (g.b_mn ? UMMA_IDESC_B_MN_MAJOR : 0u);
            for (int t = first; ok && t < g.tiles; t += stride, ++tc) {
                const LinearTile tile = linear_tile(g, t, TILE_M);
                // (M = 256 for a pair, 128 for one CTA; FP32 accumulator; BF16 = 1, TF32 = 2)
                const uint32_t type = PLANES == 3 ? 2u : 1u;
                const uint32_t idesc = form | (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)(tile.n_eff >> 3) << 17) | ((uint32_t)(TILE_M >> 4) << 24);
                const uint32_t buf = tc & 1u;
                if (!mbar_wait(smem_u32(bar_acc_empty + buf), ((tc >> 1) & 1u) ^ 1u, budget)) { s_timeout = 1; break; }
                tc_fence_after();
                const uint32_t d = tmem_base + buf * ACC_COLS;
                for (int kb = tile.kb0; kb < tile.kb1; ++kb) {
                    const int s = stage;
                    if (!mbar_wait(smem_u32(bar_full + s), phase, budget)) { s_timeout = 1; ok = false; break; }
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                    tc_fence_after();
                    const uint32_t a = smem_u32(smem + s * SM::STAGE_BYTES), b = a + P * SM::A_BYTES;
                    if constexpr (PLANES == 3) {
                        // (A plane, B plane): low x high and high x low first, the large products last
#pragma unroll
                        for (int pr = 0; pr < 3; ++pr)
#pragma unroll
                            for (int k4 = 0; k4 < 4; ++k4) {
                                const uint64_t ad = umma_desc_at(UMMA_DESC_HI_K, a + (pr == 0 ? SM::A_BYTES : 0) + k4 * 32);
                                const uint64_t bd = umma_desc_at(UMMA_DESC_HI_K, b + (pr == 1 ? SM::B_BYTES : 0) + k4 * 32);
                                const uint32_t acc = ((kb - tile.kb0) | pr | k4) ? 1u : 0u;
                                if constexpr (CG == 2) tc_mma_tf32_pair(d, ad, bd, idesc, acc);
                                else tc_mma_tf32(d, ad, bd, idesc, acc);
                            }
                    } else {
#pragma unroll
                        for (int k4 = 0; k4 < 4; ++k4) {
                            const uint64_t ad = umma_desc_at(a_hi, a + k4 * a_step), bd = umma_desc_at(b_hi, b + k4 * b_step);
                            const uint32_t acc = ((kb - tile.kb0) | k4) ? 1u : 0u;
                            if constexpr (CG == 2) tc_mma_bf16_pair(d, ad, bd, idesc, acc);
                            else tc_mma_bf16(d, ad, bd, idesc, acc);
                        }
                    }
                    if constexpr (CG == 2) tc_commit_pair(smem_u32(bar_empty + s));
                    else tc_commit(smem_u32(bar_empty + s));
                }
                if constexpr (CG == 2) tc_commit_pair(smem_u32(bar_acc_full + buf));
                else tc_commit(smem_u32(bar_acc_full + buf));
            }
        }
    } else if (warp >= 4) {
        // warp e reads tensor-memory lanes 32 (e % 4) .. and the boxes of even or odd position in the tile's columns
        const LinearEpilogue &e = g.e;
        const int ew = warp - 4, q = warp & 3, half = ew >> 2;
        uint8_t *boxes = smem + SM::BOX_OFFSET + ew * SM::BOXES * SM::BOX_BYTES, *pre_box = boxes + 2 * SM::BOX_BYTES;
        constexpr int CW = F32 ? 32 : 64;
        const uint32_t res_bar = smem_u32(bar_res + 2 * ew);
        const uint32_t call_key = e.drop.threshold ? drop_call_key(e.drop) : 0u;
        uint32_t nb = 0;          // boxes taken so far: box nb & 1; its barrier has then been used nb >> 1 times
        uint32_t tc = 0;
        bool ok = true;
        for (int t = first; ok && t < g.tiles; t += stride, ++tc) {
            const LinearTile tile = linear_tile(g, t, TILE_M);
            const uint32_t buf = tc & 1u;
            const int row0 = tile.m0 + (int)rank * UM_BM + q * 32, nrows = min(32, g.M - row0);
            const int n_end = min(g.N, tile.n0 + g.width);
            const int first_col = tile.n0 + half * CW;
            const int cnt = nrows > 0 && first_col < n_end ? (n_end - first_col + 2 * CW - 1) / (2 * CW) : 0;   // boxes of this warp
            auto fetch = [&](uint32_t b, int k) {      // residual of the warp's k-th box of the tile into box b, through TMA
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    mbar_expect_tx(res_bar + 8 * b, SM::BOX_BYTES);
                    tma_load_2d(smem_u32(boxes + b * SM::BOX_BYTES), &g.tmRes, res_bar + 8 * b, first_col + 2 * CW * k, row0);
                }
            };
            if (e.res && e.res_tma && cnt) {
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");   // both boxes have left
                __syncwarp();
                for (int k = 0; k < min(2, cnt); ++k) fetch((nb + k) & 1u, k);
            }
            const DropRow drop_row = e.drop.threshold ? drop_row_key(call_key, row0 + lane) : DropRow{0, 0};
            if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(bar_acc_full + buf), (tc >> 1) & 1u, budget))) { s_timeout = 1; break; }
            tc_fence_after();
            for (int k = 0; k < cnt; ++k, ++nb) {
                const int col0 = first_col + 2 * CW * k, ncols = min(CW, n_end - col0);
                uint8_t *box = boxes + (nb & 1u) * SM::BOX_BYTES;
                if (lane == 0) {      // the box, and the pre box, have been read by the stores that used them last
                    if (e.pre) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    else asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                }
                __syncwarp();
                if (e.res) {
                    if (e.res_tma) {
                        if (!__all_sync(0xffffffffu, mbar_wait(res_bar + 8 * (nb & 1u), (nb >> 1) & 1u, budget))) { s_timeout = 1; ok = false; break; }
                    } else {
                        box_from_rows<F32>(box, (const uint8_t *)e.res + ((int64_t)row0 * e.ldr + col0) * (F32 ? 4 : 2), e.ldr, nrows, ncols, lane);
                        __syncwarp();
                    }
                }
#pragma unroll 1
                for (int h = 0; h < CW / 32; ++h) {
                    const int col = col0 + 32 * h;
                    uint32_t r[32];
                    tc_ld_32x32(tmem_base + ((uint32_t)(q * 32) << 16) + buf * ACC_COLS + (uint32_t)(col - tile.n0), r);
                    if (k + 1 == cnt && h + 1 == CW / 32) {     // the warp has read its part of the accumulator
                        tc_fence_before();
                        if (lane == 0) { if constexpr (CG == 2) mbar_arrive_leader(smem_u32(bar_acc_empty + buf)); else mbar_arrive_rank(smem_u32(bar_acc_empty + buf), 0); }
                    }
                    float v[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
                    if (e.bias) add_bias(v, e, col, g.N);
                    if (e.pre) {
#pragma unroll
                        for (int u = 0; u < (F32 ? 8 : 4); ++u) {
                            if (F32) *(float4 *)box_unit(pre_box, lane, u) = make_float4(v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]);
                            else *box_unit(pre_box, lane, 4 * h + u) = make_uint4(pack_bf16(v[8 * u], v[8 * u + 1]), pack_bf16(v[8 * u + 2], v[8 * u + 3]),
                                                                                 pack_bf16(v[8 * u + 4], v[8 * u + 5]), pack_bf16(v[8 * u + 6], v[8 * u + 7]));
                        }
                    }
                    if (e.act) activate(v, e.act);
                    if (e.drop.threshold) {
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const uint32_t w = drop_word(drop_row, (uint32_t)(col + j) >> 1);
                            v[j] = drop_lo(w, v[j], e.drop);
                            v[j + 1] = drop_hi(w, v[j + 1], e.drop);
                        }
                    }
#pragma unroll
                    for (int u = 0; u < (F32 ? 8 : 4); ++u) {
                        if constexpr (F32) {
                            float4 *at = (float4 *)box_unit(box, lane, u);
                            float4 x = make_float4(v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]);
                            if (e.res) { const float4 o = *at; x.x += o.x; x.y += o.y; x.z += o.z; x.w += o.w; }
                            *at = x;
                        } else {
                            uint4 *at = box_unit(box, lane, 4 * h + u);
                            if (e.res) {
                                float o[8];
                                unpack8(*at, o);
#pragma unroll
                                for (int i = 0; i < 8; ++i) v[8 * u + i] += o[i];
                            }
                            *at = make_uint4(pack_bf16(v[8 * u], v[8 * u + 1]), pack_bf16(v[8 * u + 2], v[8 * u + 3]),
                                             pack_bf16(v[8 * u + 4], v[8 * u + 5]), pack_bf16(v[8 * u + 6], v[8 * u + 7]));
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                // A TMA store is clipped at the matrix edge in units of 16 bytes: where the last one is not whole, the last box goes by rows.
                const bool whole = g.whole_edge || col0 + CW <= g.N;
                const bool out_tma = e.out_tma && whole, pre_tma = e.pre_tma && whole;
                if (lane == 0) {
                    if (out_tma) tma_store_2d(&g.tmOut, smem_u32(box), col0, row0 + tile.split * g.slab_rows);
                    if (e.pre && pre_tma) tma_store_2d(&g.tmPre, smem_u32(pre_box), col0, row0);
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                }
                if (!out_tma) box_to_rows<F32>(box, (uint8_t *)e.out + ((int64_t)row0 * e.ldo + col0) * (F32 ? 4 : 2), e.ldo, nrows, ncols, lane);
                if (e.pre && !pre_tma) box_to_rows<F32>(pre_box, (uint8_t *)e.pre + ((int64_t)row0 * e.ldp + col0) * (F32 ? 4 : 2), e.ldp, nrows, ncols, lane);
                __syncwarp();
                if (e.res && e.res_tma && k + 2 < cnt) {       // (FP32: four boxes of a 256-wide tile)
                    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();
                    fetch(nb & 1u, k + 2);
                }
            }
            if (cnt == 0) {
                tc_fence_before();
                if (lane == 0) { if constexpr (CG == 2) mbar_arrive_leader(smem_u32(bar_acc_empty + buf)); else mbar_arrive_rank(smem_u32(bar_acc_empty + buf), 0); }
            }
        }
        // stores still read their boxes; residual copies that nobody waited for are waited for at the end
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    if (s_timeout) __nanosleep(2000000);   // let copies in flight land before the CTA goes away
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();      // neither CTA leaves while the peer still uses its shared or tensor memory
    if (warp == 1) {
        tc_fence_after();
        if constexpr (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
    if (threadIdx.x == 0 && s_timeout) atomicMax(&g_layer_status, (int)TSR_ERR_TIMEOUT);
}

template <int CG, int PLANES, bool F32>
static cudaError_t gemm_launch_as(const LinearGemm &g, int sms, cudaStream_t stream)
{
    using SM = LinearSmem<PLANES>;
    static bool configured[64] = {};      // per device; setting it twice is harmless
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !configured[dev]) {
        e = cudaFuncSetAttribute(linear_gemm_kernel<CG, PLANES, F32>, cudaFuncAttributeMaxDynamicSharedMemorySize, SM::TOTAL);
        if (e != cudaSuccess) return e;
        if (dev < 64) configured[dev] = true;
    }
    const int slots = sms / CG, n = g.tiles < slots ? g.tiles : slots;
    return launch_dependent(linear_gemm_kernel<CG, PLANES, F32>, dim3(CG * n), dim3(LG_THREADS), (size_t)SM::TOTAL, stream, 1, g);
}

cudaError_t linear_gemm_launch(const LinearGemm &g, int cg, bool f32_operands, bool f32_out, int sms, cudaStream_t stream)
{
    if (f32_operands) return cg == 2 ? gemm_launch_as<2, 3, true>(g, sms, stream) : gemm_launch_as<1, 3, true>(g, sms, stream);
    if (f32_out) return cg == 2 ? gemm_launch_as<2, 1, true>(g, sms, stream) : gemm_launch_as<1, 1, true>(g, sms, stream);
    return cg == 2 ? gemm_launch_as<2, 1, false>(g, sms, stream) : gemm_launch_as<1, 1, false>(g, sms, stream);
}

cudaError_t layer_status_read(int32_t *status, cudaStream_t stream)
{
    int zero = 0, v = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(&v, g_layer_status, sizeof(int), 0, cudaMemcpyDeviceToHost, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    if (e == cudaSuccess && v) e = cudaMemcpyToSymbolAsync(g_layer_status, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    *status = v;
    return e;
}

}  // namespace tsr
