// Products of the linear layer on the 5th-generation tensor cores, with the layer's epilogue (formulas in tsr.h).
//
//   D[M x N] = A[M x K] B[N x K]^T,   then per entry  z = D + bias;  pre = z;  out = residual + dropout(act(z)),  or  out = residual + scale D
//
// One persistent CTA per SM (CG = 1, tiles of 128 x width) or one pair of CTAs per two SMs (CG = 2, 256 x width, tcgen05 with
// cta_group::2).  Either operand is K-major or MN-major (a row-major matrix contracted over its rows, read as it lies), so
// that x W^T, dz W and dz^T x need no transposed copies.  Roles, as in the grouped GEMM of the optimizer: warp 0 loads
// A, warp 2 loads B (each CTA of a pair its half of the tile's B rows, no multicast), warp 1 issues the MMAs into one of two
// accumulators in tensor memory, warps 4 to 11 run the epilogue of one tile beside the MMAs of the next.
//
// FP32 operands come as three BF16 planes (x = p1 + p2 + p3, 24 bits) and D = p1 q1 + (p1 q2 + p2 q1) + (p2 q2 + p1 q3 + p3 q1): six BF16 products
// cost the tensor cores what three TF32 products cost, keep two bits more, move three quarters of the bytes and take MN-major operands.  The
// tensor cores cut off what falls below the accumulator's last bit, which adds up over a long K (10^-5 of the result at K = 4096); the
// accumulator is therefore emptied every 128 entries of K into FP32 registers of the epilogue warps, added to nearest.  K blocks are 32 entries there,
// of which three stages fit beside the boxes.
//
// An infinity x = p1 against parts of q of both signs, or zero ones, comes out as NaN where x q is infinite.  So entries that are NaN are formed again from x and q
// themselves, in FP32 (formed_again): a compare per entry in all other cases.
//
// Epilogue: a lane holds a row.  A warp's 32 rows x 128 bytes of output form a box in shared memory (128-byte swizzle: free of bank
// conflicts when the lanes walk their rows), of which it has two, and a third for pre.  The residual is fetched into the box by TMA
// while the MMAs still run, the result replaces it in place, and the box leaves by TMA.  Matrices whose pitch or address TMA
// does not take go between box and memory by plain row accesses instead; the arithmetic is the same.
//
// Work items: whole tiles first, a multiple of what runs at once; the tiles of the last, partly filled wave (all of them in a small product) may be
// split along K.  The parts store FP32 slabs, and linear_finish_kernel adds a tile's slabs in order and runs its epilogue.
//
// What bounds it: in the main loop the tensor cores (a K block of 256 x 256 takes a pair 493 clocks, of FP32 operands 764; 512 and 768 nominal, at the
// 1.5 to 1.7 GHz that the power limit leaves).  An SM takes in 64 bytes of operands a clock, which 256 x 256 tiles of a pair just feed (64 bytes per
// clock of MMA); narrower tiles are bound by that intake, and tiles with a short K by the epilogue (5003 x 768 -> 2048: 20 us, with GELU 28: two uses
// of the special-function units per entry).  Measured: 8192^3 BF16 at 0.96 of the library's product, 8192 x 2048 -> 2048 at 1.0.  The ring takes what shared memory the boxes leave: five stages of 32 KB rather than four are worth 3 to 6 %.
// Every mbarrier wait is bounded; on expiry the CTA notes it in the status
// word, stops storing, waits for copies in flight, frees its tensor memory and returns.
#include "tsr_linear.cuh"
#include "tsr_umma.cuh"

namespace tsr {

constexpr int LG_THREADS = 384, LG_EPI_WARPS = 8;
__device__ int g_linear_status;

// Shared memory: ring of stages (A, then B; geometry in LinearGemm), boxes, barriers.
constexpr int LG_BOX_BYTES = 4096;
constexpr int LG_NBARS = 2 * LG_MAX_STAGES + 4 + 2 * LG_EPI_WARPS;
constexpr int LG_TAIL_BYTES = LG_NBARS * 8 + 16;
constexpr int LG_SMEM = 227 * 1024 - 64;                  // (the static word beside it)
constexpr int LG_RING = LG_SMEM - 1024 - LG_TAIL_BYTES;   // of ring and boxes, after the alignment to 1024 bytes

int linear_stages(int stage_bytes, bool pre)
{
    const int n = (LG_RING - LG_EPI_WARPS * (pre ? 3 : 2) * LG_BOX_BYTES) / stage_bytes;
    return n < LG_MAX_STAGES ? n : LG_MAX_STAGES;
}

template <int ACT, bool F32>
__device__ __forceinline__ void activate(float (&v)[32])
{
    if constexpr (ACT != TSR_ACT_NONE) {
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
            const float2 x = make_float2(v[j], v[j + 1]), z = F32 ? act_pair_full<ACT>(x) : act_pair<ACT>(x);
            v[j] = z.x;
            v[j + 1] = z.y;
        }
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

// Eight entries along K of one row of an FP32 operand, from its planes; `mn`: the operand is stored with K as its rows, of which `last` exist.
__device__ __forceinline__ void whole_entries(const bf16 *p, int64_t ld, int64_t plane, bool mn, int row, int k, int last, float (&v)[8])
{
    if (!mn) {      // (rows are padded with zeros to whole units)
        float part[8];
        load8(p + row * ld + k, v);
        load8(p + plane + row * ld + k, part);
        float rest[8];
        load8(p + 2 * plane + row * ld + k, rest);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += part[i] + rest[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bf16 *at = p + (int64_t)(k + i) * ld + row;
            v[i] = k + i < last ? load_f(at) + (load_f(at + plane) + load_f(at + 2 * plane)) : 0.f;
        }
    }
}
// 32 columns of the warp's 32 rows over the K range of the item; the entries that are NaN are replaced.  It ends where they have all become NaN again.
__device__ __forceinline__ void formed_again(const LinearGemm &g, int row0, int col0, int first, int last, int lane, float (&v)[32])
{
    float s[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) s[j] = 0.f;
    const int row = min(row0 + lane, g.M - 1), col = min(col0 + lane, g.N - 1);
#pragma unroll 1
    for (int k = first; k < last; k += 8) {
        float a[8], b[8];
        whole_entries(g.parts[0].p, g.parts[0].ld, g.parts[0].plane, g.a_mn, row, k, last, a);
        whole_entries(g.parts[1].p, g.parts[1].ld, g.parts[1].plane, g.b_mn, col, k, last, b);
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int j = 0; j < 32; ++j) s[j] = fmaf(a[0], __shfl_sync(0xffffffffu, b[0], j), s[j]);
#pragma unroll
            for (int n = 0; n < 7; ++n) { a[n] = a[n + 1]; b[n] = b[n + 1]; }
        }
        bool open = false;
#pragma unroll
        for (int j = 0; j < 32; ++j) open |= v[j] != v[j] && s[j] == s[j];
        if (!__any_sync(0xffffffffu, open)) break;
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = v[j] != v[j] ? s[j] : v[j];
}

// One MMA, issued by the lane for which `leader` is set; the whole warp runs through here, so that the descriptors stay in uniform registers.  They are
// given as halves: the lower one moves with the address (bits 0 .. 13 = address >> 4), the upper one is the operand's form.
template <int CG>
__device__ __forceinline__ void mma_bf16(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate, uint32_t leader)
{
    if constexpr (CG == 2)
        asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 a, b;\n\tmov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
                     "@q tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %5, p;\n\t}"
                     ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 a, b;\n\tmov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
                     "@q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n\t}"
                     ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
__device__ __forceinline__ uint32_t elect_one()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r;
}

__device__ __forceinline__ void bulk_wait_read(int pending)
{
    if (pending) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
    else asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"((uint64_t)map), "r"(bar), "r"(x), "r"(y), "r"(0) : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"((uint64_t)map), "r"(bar), "r"(x), "r"(y), "r"(0) : "memory");
}

// PLANES: 1, BF16 operands; 3, FP32 operands in three BF16 planes.  F32: type of out, residual and pre.  EPI: the activation of a full epilogue, or
// EPI_PLAIN: out = residual + scale D.  (One kernel for all of them spent a third of its time waiting for instructions.)
constexpr int EPI_PLAIN = -1;
template <int CG, int PLANES, bool F32, int EPI>
__global__ void __cluster_dims__(CG, 1, 1) __launch_bounds__(LG_THREADS, 1)
linear_gemm_kernel(const __grid_constant__ LinearGemm g)
{
    constexpr bool FULL = EPI != EPI_PLAIN;
    constexpr int TILE_M = CG * UM_BM, BK = PLANES == 3 ? 32 : 64;      // entries of a K block
    constexpr uint32_t TMEM_COLS = CG == 2 ? 512 : 256, ACC_COLS = TMEM_COLS / 2;
    constexpr int CW = F32 ? 32 : 64;                // columns of a box
    constexpr int PAIRS[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};   // planes of A and B, the small products first
    constexpr int CHUNK = PLANES == 3 ? 4 : 1 << 30; // K blocks per emptying of the accumulator

    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const int stages = g.stages, stage_bytes = g.stage_bytes;
    uint8_t *box_area = smem + stages * stage_bytes;
    uint64_t *bars = (uint64_t *)(smem + LG_RING);
    uint64_t *bar_full = bars, *bar_empty = bars + LG_MAX_STAGES;
    uint64_t *bar_acc_full = bars + 2 * LG_MAX_STAGES, *bar_acc_empty = bar_acc_full + 2, *bar_res = bar_acc_empty + 2;
    uint32_t *tmem_slot = (uint32_t *)(bars + LG_NBARS);
    __shared__ int s_timeout;

    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long budget = UM_WAIT_CLOCKS;
    const uint32_t rank = CG == 2 ? cluster_ctarank() : 0u;
    const int first = CG == 2 ? (int)(blockIdx.x >> 1) : (int)blockIdx.x, stride = CG == 2 ? (int)(gridDim.x >> 1) : (int)gridDim.x;

    if (threadIdx.x == 64) {      // the maps are on their way while barriers and tensor memory are set up
        asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&g.tmA) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&g.tmB) : "memory");
    }
    if (threadIdx.x == 0) {
        s_timeout = 0;
        for (int s = 0; s < stages; ++s) { mbar_init(smem_u32(bar_full + s), 1); mbar_init(smem_u32(bar_empty + s), 1); }
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

    // FP32: the sums of the epilogue warps (128 registers) come from the registers that loaders and MMA warp leave, 3 x 168 = 56 + 2 x 224.
    if (warp < 4) {
        if constexpr (PLANES == 3) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 0 || warp == 2) {      // the whole warp; one lane asks
            const uint32_t leader = elect_one();
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            const bool is_a = warp == 0, mn = is_a ? g.a_mn : g.b_mn;
            const int boxes = mn ? is_a ? g.a_boxes : g.b_boxes : 1;
            const CUtensorMap *map = is_a ? &g.tmA : &g.tmB;
            const uint32_t base = smem_u32(smem) + (is_a ? 0u : (uint32_t)g.b_offset);
            constexpr uint32_t GROUP = PLANES * 64 * BK * 2;      // an MN-major operand's groups of 64 columns follow one another
            for (int t = first; ok && t < g.items; t += stride) {
                const LinearTile tile = linear_tile(g, t, TILE_M);
                const int row = is_a ? tile.m0 + (int)rank * UM_BM : tile.n0 + (int)rank * (tile.n_eff / CG);
                for (int kb = tile.kb0; kb < tile.kb1; ++kb) {
                    if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(bar_empty + stage), phase ^ 1u, budget))) { s_timeout = 1; ok = false; break; }
                    if (leader) {
                        // the copies of both CTAs of a pair report their bytes to the leader CTA's barrier
                        const uint32_t full = CG == 2 ? leader_addr(smem_u32(bar_full + stage)) : smem_u32(bar_full + stage);
                        if (is_a && rank == 0) mbar_expect_tx(smem_u32(bar_full + stage), g.stage_tx);
                        uint32_t to = base + stage * stage_bytes;
                        int x = mn ? row : kb * BK;
                        const int y = mn ? kb * BK : row;
                        for (int j = 0; j < boxes; ++j, to += GROUP, x += 64) {
                            if constexpr (PLANES == 1) {
                                if constexpr (CG == 2) tma_load_2d_pair(to, map, full, x, y);
                                else tma_load_2d(to, map, full, x, y);
                            } else {      // the three planes at once
                                if constexpr (CG == 2) tma_load_3d_pair(to, map, full, x, y);
                                else tma_load_3d(to, map, full, x, y);
                            }
                        }
                    }
                    if (++stage == stages) { stage = 0; phase ^= 1u; }
                }
            }
        } else if (warp == 1) {
            if (rank == 0) {      // the whole warp; one lane issues
                uint32_t tc = 0, phase = 0;      // tc: accumulators filled so far
                int stage = 0;
                bool ok = true;
                const uint32_t leader = elect_one();
                // Operand forms.  K-major: rows of 128 bytes, eight of them 1024 apart; MN-major: groups of 64 columns 8 KB apart.  Three planes: K-major rows
                // of 64 bytes (64-byte swizzle, layout type 4; eight rows 512 bytes apart), MN-major groups of 64 columns x 32 rows, the three
                // planes of a group one behind the other.
                constexpr uint64_t K3 = ((uint64_t)1 << 16) | ((uint64_t)(512 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)4 << 61);
                constexpr uint64_t MN3 = ((uint64_t)(3 * 4096 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
                const uint64_t mn_form = PLANES == 3 ? MN3 : UMMA_DESC_HI_MN, k_form = PLANES == 3 ? K3 : UMMA_DESC_HI_K;
                const uint64_t a_form = g.a_mn ? mn_form : k_form, b_form = g.b_mn ? mn_form : k_form;
                const uint32_t a_hi = (uint32_t)(a_form >> 32), b_hi = (uint32_t)(b_form >> 32);
                // in units of 16 bytes: from one MMA's 16 entries of K to the next, from plane to plane
                const uint32_t a_step = (g.a_mn ? 2048u : 32u) >> 4, b_step = (g.b_mn ? 2048u : 32u) >> 4;
                const uint32_t a_plane = (g.a_mn ? 4096u : (uint32_t)g.a_rows * 64u) >> 4, b_plane = (g.b_mn ? 4096u : (uint32_t)(g.width / CG) * 64u) >> 4;
                const uint32_t a_first = (uint32_t)a_form + (smem_u32(smem) >> 4), b_first = (uint32_t)b_form + ((smem_u32(smem) + g.b_offset) >> 4);
                const uint32_t stage_step = (uint32_t)stage_bytes >> 4;
                // (M = 256 for a pair, 128 for one CTA; FP32 accumulator; BF16 operands)
                const uint32_t form = (g.a_mn ? UMMA_IDESC_A_MN_MAJOR : 0u) | (g.b_mn ? UMMA_IDESC_B_MN_MAJOR : 0u) | (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TILE_M >> 4) << 24);
                uint32_t a = a_first, b = b_first;
                for (int t = first; ok && t < g.items; t += stride) {
                    const LinearTile tile = linear_tile(g, t, TILE_M);
                    const uint32_t idesc = form | ((uint32_t)(tile.n_eff >> 3) << 17);
                    for (int k0 = tile.kb0; ok && k0 < tile.kb1; ++tc) {
                        const int k1 = tile.kb1 - k0 > CHUNK ? k0 + CHUNK : tile.kb1;
                        const uint32_t buf = tc & 1u;
                        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(bar_acc_empty + buf), ((tc >> 1) & 1u) ^ 1u, budget))) { s_timeout = 1; ok = false; break; }
                        tc_fence_after();
                        const uint32_t d = tmem_base + buf * ACC_COLS;
                        uint32_t acc = 0;      // the first MMA overwrites
                        for (int kb = k0; kb < k1; ++kb) {
                            if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(bar_full + stage), phase, budget))) { s_timeout = 1; ok = false; break; }
                            tc_fence_after();
    #pragma unroll
                            for (int pr = PLANES == 3 ? 0 : 5; pr < 6; ++pr)
    #pragma unroll
                                for (int k4 = 0; k4 < BK / 16; ++k4) {
                                    mma_bf16<CG>(d, a + PAIRS[pr][0] * a_plane + k4 * a_step, a_hi, b + PAIRS[pr][1] * b_plane + k4 * b_step, b_hi, idesc, acc, leader);
                                    acc = 1;
                                }
                            if (leader) {
                                if constexpr (CG == 2) tc_commit_pair(smem_u32(bar_empty + stage));
                                else tc_commit(smem_u32(bar_empty + stage));
                            }
                            a += stage_step;
                            b += stage_step;
                            if (++stage == stages) { stage = 0; phase ^= 1u; a = a_first; b = b_first; }
                        }
                        if (leader) {
                            if constexpr (CG == 2) tc_commit_pair(smem_u32(bar_acc_full + buf));
                            else tc_commit(smem_u32(bar_acc_full + buf));
                        }
                        k0 = k1;
                    }
                }
            }
        }
    } else {
        if constexpr (PLANES == 3) asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        // warp e reads tensor-memory lanes 32 (e % 4) .. and the boxes of even or odd position in the tile's columns
        const LinearEpilogue &e = g.e;
        const int ew = warp - 4, q = warp & 3, half = ew >> 2;
        uint8_t *boxes = box_area + ew * (FULL && e.pre ? 3 : 2) * LG_BOX_BYTES, *pre_box = boxes + 2 * LG_BOX_BYTES;
        const uint32_t res_bar = smem_u32(bar_res + 2 * ew), lanes = tmem_base + ((uint32_t)(q * 32) << 16);
        const bool drops = FULL && e.drop.threshold;
        const uint32_t call_key = drops ? drop_call_key(e.drop) : 0u;
        uint32_t nb = 0, res_phase = 0;     // boxes taken so far (the next is nb & 1); phases of the two boxes' barriers
        uint32_t tc = 0;
        bool ok = true;
        for (int t = first; ok && t < g.items; t += stride) {
            const LinearTile tile = linear_tile(g, t, TILE_M);
            const bool slab = tile.part >= 0;
            const int row0 = tile.m0 + (int)rank * UM_BM + q * 32, nrows = min(32, g.M - row0);
            const int n_end = min(g.N, tile.n0 + g.width);
            const int cw = slab ? 32 : CW;
            const int first_col = tile.n0 + half * cw;
            const int cnt = nrows > 0 && first_col < n_end ? (n_end - first_col + 2 * cw - 1) / (2 * cw) : 0;   // boxes of this warp
            const bool res = e.res && !slab;
            auto release = [&](uint32_t buf) {      // the warp has read its part of the accumulator
                tc_fence_before();
                if (lane == 0) { if constexpr (CG == 2) mbar_arrive_leader(smem_u32(bar_acc_empty + buf)); else mbar_arrive_rank(smem_u32(bar_acc_empty + buf), 0); }
            };
            auto acc_full = [&](uint32_t n) -> bool {
                if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(bar_acc_full + (n & 1u)), (n >> 1) & 1u, budget))) { s_timeout = 1; return false; }
                tc_fence_after();
                return true;
            };
            auto fetch = [&](uint32_t b, int k) {      // residual of the warp's k-th box of the tile into box b, through TMA
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    mbar_expect_tx(res_bar + 8 * b, LG_BOX_BYTES);
                    tma_load_2d(smem_u32(boxes + b * LG_BOX_BYTES), &g.tmRes, res_bar + 8 * b, first_col + 2 * CW * k, row0);
                }
            };
            if (res && e.res_tma && cnt) {
                if (lane == 0) bulk_wait_read(0);      // both boxes have left
                __syncwarp();
                for (int k = 0; k < min(2, cnt); ++k) fetch((nb + k) & 1u, k);
            }
            const DropRow drop_row = drops && !slab ? drop_row_key(call_key, row0 + lane) : DropRow{0, 0};
            // bias of the warp's groups of 32 columns, a column per lane
            float bias[4] = {0.f, 0.f, 0.f, 0.f};
            if (FULL && e.bias && !slab) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = F32 ? first_col + 64 * i + lane : first_col + 128 * (i >> 1) + 32 * (i & 1) + lane;
                    if (c < n_end) bias[i] = load_as(e.bias, c, e.bias_bf16);
                }
            }

            float sum[PLANES == 3 ? 4 : 1][32];
            if constexpr (PLANES == 3) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int j = 0; j < 32; ++j) sum[k][j] = 0.f;
                for (int k0 = tile.kb0; k0 < tile.kb1; k0 += CHUNK, ++tc) {
                    if (!acc_full(tc)) { ok = false; break; }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (k >= cnt) continue;
                        uint32_t r[32];
                        tc_ld_32x32(lanes + (tc & 1u) * ACC_COLS + (uint32_t)(first_col + 64 * k - tile.n0), r);
#pragma unroll
                        for (int j = 0; j < 32; ++j) sum[k][j] += __uint_as_float(r[j]);
                    }
                    release(tc & 1u);
                }
                if (!ok) break;
            } else {
                if (!acc_full(tc)) break;
            }

            // One box: its values from tensor memory, or the sums in src
            auto one_box = [&](int k, const float (&src)[32]) -> bool {
                const int col0 = first_col + 2 * cw * k, ncols = min(cw, n_end - col0);
                uint8_t *box = boxes + (nb & 1u) * LG_BOX_BYTES;
                if (lane == 0) bulk_wait_read(FULL && e.pre ? 0 : 1);      // the box, and the pre box, have been read by the stores that used them last
                __syncwarp();
                if (res) {
                    if (e.res_tma) {
                        const uint32_t b = nb & 1u;
                        if (!__all_sync(0xffffffffu, mbar_wait(res_bar + 8 * b, (res_phase >> b) & 1u, budget))) { s_timeout = 1; return false; }
                        res_phase ^= 1u << b;
                    } else {
                        box_from_rows<F32>(box, (const uint8_t *)e.res + ((int64_t)row0 * e.ldr + col0) * (F32 ? 4 : 2), e.ldr, nrows, ncols, lane);
                        __syncwarp();
                    }
                }
#pragma unroll 1
                for (int h = 0; h < cw / 32; ++h) {
                    const int col = col0 + 32 * h;
                    float v[32];
                    if constexpr (PLANES == 3) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = src[j];
                    } else {
                        uint32_t r[32];
                        tc_ld_32x32(lanes + (tc & 1u) * ACC_COLS + (uint32_t)(col - tile.n0), r);
                        if (k + 1 == cnt && h + 1 == cw / 32) release(tc & 1u);
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
                    }
                    if (slab) {
#pragma unroll
                        for (int u = 0; u < 8; ++u) *(float4 *)box_unit(box, lane, u) = make_float4(v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]);
                        continue;
                    }
                    if (FULL && e.bias) {
                        const int i = F32 ? k : 2 * k + h;
                        const float mine = i == 0 ? bias[0] : i == 1 ? bias[1] : i == 2 ? bias[2] : bias[3];
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] += __shfl_sync(0xffffffffu, mine, j);
                    }
                    if (FULL && e.pre) {
#pragma unroll
                        for (int u = 0; u < (F32 ? 8 : 4); ++u) {
                            if (F32) *(float4 *)box_unit(pre_box, lane, u) = make_float4(v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]);
                            else *box_unit(pre_box, lane, 4 * h + u) = make_uint4(pack_bf16(v[8 * u], v[8 * u + 1]), pack_bf16(v[8 * u + 2], v[8 * u + 3]),
                                                                                 pack_bf16(v[8 * u + 4], v[8 * u + 5]), pack_bf16(v[8 * u + 6], v[8 * u + 7]));
                        }
                    }
                    if constexpr (FULL) activate<EPI, F32>(v);
                    if constexpr (!FULL) {
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const float2 x = mul2(make_float2(v[j], v[j + 1]), pair(e.scale));
                            v[j] = x.x;
                            v[j + 1] = x.y;
                        }
                    }
                    if (drops) {
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
                            if (res) { const float4 o = *at; x.x += o.x; x.y += o.y; x.z += o.z; x.w += o.w; }
                            *at = x;
                        } else {
                            uint4 *at = box_unit(box, lane, 4 * h + u);
                            if (res) {
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
                const bool whole = g.whole_edge || col0 + cw <= g.N;
                const bool out_tma = e.out_tma && whole, pre_tma = FULL && e.pre_tma && whole;
                if (lane == 0) {
                    if (slab) tma_store_2d(&g.tmSlab, smem_u32(box), col0 - tile.n0, tile.part * TILE_M + (int)rank * UM_BM + q * 32);
                    else if (out_tma) tma_store_2d(&g.tmOut, smem_u32(box), col0, row0);
                    if (FULL && e.pre && pre_tma && !slab) tma_store_2d(&g.tmPre, smem_u32(pre_box), col0, row0);
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                }
                if (!slab) {
                    if (!out_tma) box_to_rows<F32>(box, (uint8_t *)e.out + ((int64_t)row0 * e.ldo + col0) * (F32 ? 4 : 2), e.ldo, nrows, ncols, lane);
                    if (FULL && e.pre && !pre_tma) box_to_rows<F32>(pre_box, (uint8_t *)e.pre + ((int64_t)row0 * e.ldp + col0) * (F32 ? 4 : 2), e.ldp, nrows, ncols, lane);
                }
                __syncwarp();
                if (res && e.res_tma && k + 2 < cnt) {       // (FP32 out: four boxes of a 256-wide tile)
                    if (lane == 0) bulk_wait_read(0);
                    __syncwarp();
                    fetch(nb & 1u, k + 2);
                }
                ++nb;
                return true;
            };
            if constexpr (PLANES == 3) {
#pragma unroll 1
                for (int k = 0; ok && k < cnt; ++k) {      // (one copy of the epilogue's code: the sums move up to the first place)
                    const int col0 = first_col + 64 * k, ncols = min(32, n_end - col0);
                    float2 z = pair(0.f);      // NaN where an entry is (or infinite); outside of the matrix there may be anything
                    if (ncols == 32) {
#pragma unroll
                        for (int j = 0; j < 32; j += 2) z = fma2(make_float2(sum[0][j], sum[0][j + 1]), pair(0.f), z);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) z.x = fmaf(j < ncols ? sum[0][j] : 0.f, 0.f, z.x);
                    }
                    z.x += z.y;
                    if (__any_sync(0xffffffffu, lane < nrows && z.x != z.x)) formed_again(g, row0, col0, tile.kb0 * BK, min(tile.kb1 * BK, g.K), lane, sum[0]);
                    ok = one_box(k, sum[0]);
#pragma unroll
                    for (int i = 0; i < 3; ++i)
#pragma unroll
                        for (int j = 0; j < 32; ++j) sum[i][j] = sum[i + 1][j];
                }
            } else {
#pragma unroll 1
                for (int k = 0; ok && k < cnt; ++k) ok = one_box(k, sum[0]);
                if (cnt == 0) release(tc & 1u);
                ++tc;
            }
        }
        // stores still read their boxes
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
    if (threadIdx.x == 0 && s_timeout) atomicMax(&g_linear_status, (int)TSR_ERR_TIMEOUT);
}

template <int CG, int PLANES, bool F32, int EPI>
static cudaError_t gemm_launch_as(const LinearGemm &g, int sms, cudaStream_t stream)
{
    static bool configured[64] = {};      // per device; setting it twice is harmless
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !configured[dev]) {
        e = cudaFuncSetAttribute(linear_gemm_kernel<CG, PLANES, F32, EPI>, cudaFuncAttributeMaxDynamicSharedMemorySize, LG_SMEM);
        if (e != cudaSuccess) return e;
        if (dev < 64) configured[dev] = true;
    }
    const int slots = sms / CG, n = g.items < slots ? g.items : slots;
    return launch_dependent(linear_gemm_kernel<CG, PLANES, F32, EPI>, dim3(CG * n), dim3(LG_THREADS), (size_t)LG_SMEM, stream, 1, g);
}

template <int PLANES, bool F32, int EPI>
static cudaError_t gemm_launch_cg(const LinearGemm &g, int cg, int sms, cudaStream_t stream)
{
    return cg == 2 ? gemm_launch_as<2, PLANES, F32, EPI>(g, sms, stream) : gemm_launch_as<1, PLANES, F32, EPI>(g, sms, stream);
}

template <int PLANES, bool F32>
static cudaError_t gemm_launch_epi(const LinearGemm &g, int cg, int sms, cudaStream_t stream)
{
    const LinearEpilogue &e = g.e;
    if (!e.bias && !e.pre && !e.act && !e.drop.threshold) return gemm_launch_cg<PLANES, F32, EPI_PLAIN>(g, cg, sms, stream);
    switch (e.act) {
    case TSR_ACT_RELU: return gemm_launch_cg<PLANES, F32, TSR_ACT_RELU>(g, cg, sms, stream);
    case TSR_ACT_GELU: return gemm_launch_cg<PLANES, F32, TSR_ACT_GELU>(g, cg, sms, stream);
    case TSR_ACT_GELU_TANH: return gemm_launch_cg<PLANES, F32, TSR_ACT_GELU_TANH>(g, cg, sms, stream);
    case TSR_ACT_SILU: return gemm_launch_cg<PLANES, F32, TSR_ACT_SILU>(g, cg, sms, stream);
    default: return gemm_launch_cg<PLANES, F32, TSR_ACT_NONE>(g, cg, sms, stream);
    }
}

cudaError_t linear_gemm_launch(const LinearGemm &g, int cg, bool f32_operands, bool f32_out, int sms, cudaStream_t stream)
{
    if (f32_operands) return gemm_launch_epi<3, true>(g, cg, sms, stream);
    if (f32_out) return gemm_launch_cg<1, true, EPI_PLAIN>(g, cg, sms, stream);      // (a weight's gradient)
    return gemm_launch_epi<1, false>(g, cg, sms, stream);
}

cudaError_t linear_status_read(int32_t *status, cudaStream_t stream)
{
    int zero = 0, v = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(&v, g_linear_status, sizeof(int), 0, cudaMemcpyDeviceToHost, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    if (e == cudaSuccess && v) e = cudaMemcpyToSymbolAsync(g_linear_status, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    *status = v;
    return e;
}

}  // namespace tsr
