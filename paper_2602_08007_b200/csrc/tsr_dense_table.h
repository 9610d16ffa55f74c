// The table of chunks of a dense plan: how tensors are cut, what room the table needs and what stands in it.  Plain C++ without
// CUDA: it follows from the descriptors and the alignment of pointers, which are not followed.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <vector>

#include "tsr.h"

namespace tsr {

constexpr int UNIT = TSR_DENSE_BLOCK;      // elements of a warp's piece of work
static_assert(UNIT == 32 * 8, "a lane holds eight elements of a unit");
constexpr int WARPS = 8;                   // per CTA
// Most units of a warp in one chunk, by what goes over it.  FP32 steps overlap by having many CTAs at a time and are faster
// short (1B set: 4.80 ms with 2 units, 4.96 with 8); the others have work per CTA or load ahead (8-bit step: 130M set 175 us
// with 8 units, 213 with 2, 1B set stochastic 2.55 and 2.87 ms; 1B norm: 384 us with 16, 442 with 4).  Without vectors short
// chunks balance better (40 M pitched elements, 8-bit step: 100 us with 4 units, 103 with 8), and those of narrow pitched
// matrices are slow ones.
constexpr int STEP_F32_UNITS = 2, STEP_Q8_UNITS = 8, COPY_UNITS = 16, NORM_UNITS = 16, PAIRS_UNITS = 4, ANY_UNITS = 1;
// Fewer chunks than this are made shorter, so that they fill the GPU (8-bit step of 4 M elements: 11.0 us, 15.7 with a bound of
// 2048).  Conversions hold more CTAs on an SM and want twice as many.
constexpr int MANY_CHUNKS = 512;

// How a call goes over a chunk.  VECTORS: everything that it touches is contiguous and aligned to vectors of eight
// elements.  PLAIN: contiguous, any alignment.  ROWS: rows of 256 elements or more, so that a unit meets the end of a row
// once at most.  All three hold whole units only.  ANY: the rest, the last units of tensors and narrow matrices.
enum DensePath : int32_t { PATH_ANY = 0, PATH_VECTORS = 1, PATH_PLAIN = 2, PATH_ROWS = 3 };

// Units [first, first + units) of tensor rec.
struct alignas(16) DenseChunk { int32_t rec; uint32_t first; int32_t units; int32_t path; };

inline bool dense_aligned(const void *p, int64_t bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }
inline int64_t dense_size_of(int32_t dtype) { return dtype == TSR_BF16 ? 2 : 4; }

// ld: the largest pitch in use
inline DensePath dense_path(bool contiguous, bool vectors, const tsr_dense_desc &d, int64_t ld)
{
    if (contiguous) return vectors ? PATH_VECTORS : PATH_PLAIN;
    return d.cols >= UNIT && ld < (1 << 30) && d.rows < (1 << 30) ? PATH_ROWS : PATH_ANY;   // (32-bit rows and columns)
}

// Rows of the gradient, of all that a step touches, follow one another directly.
inline bool dense_grad_contiguous(const tsr_dense_desc &d) { return d.rows <= 1 || d.ldg == d.cols; }
inline bool dense_step_contiguous(const tsr_dense_desc &d, bool image)
{
    return d.rows <= 1 || (d.ldg == d.cols && d.ldp == d.cols && (!image || d.ldi == d.cols));
}
inline DensePath dense_norm_path(const tsr_dense_desc &d, bool vectors) { return dense_path(dense_grad_contiguous(d), vectors, d, d.ldg); }
// states: the moments are aligned to vectors; vectors: everything else is too
inline DensePath dense_step_path(const tsr_dense_desc &d, bool image, bool states, bool vectors)
{
    if (d.state == TSR_STATE_Q8 && !states) return PATH_ANY;   // the ring takes codes eight by eight
    return dense_path(dense_step_contiguous(d, image), states && vectors, d, std::max(std::max(d.ldp, d.ldg), image ? d.ldi : 0));
}

// Cuts of a tensor of n elements: chunks of `length` units, the first `whole` units on path `how`, then the partial last unit,
// a chunk of its own where that path takes whole units only.
struct DenseCuts {
    int64_t units, whole, length;
    DenseCuts(int64_t n, DensePath how, int at_once)
    {
        length = at_once;
        if (how == PATH_ANY) length = std::min(at_once, WARPS * ANY_UNITS);
        if (how == PATH_PLAIN || how == PATH_ROWS) length = std::min(at_once, WARPS * PAIRS_UNITS);
        units = (n + UNIT - 1) / UNIT;
        whole = how != PATH_ANY ? n / UNIT : units;
    }
    int64_t count() const { return (whole + length - 1) / length + (whole < units); }
};

struct DenseTable {
    // One table: the chunks of the stepped tensors group by group, then those of the norm, then those of copies.
    struct Group { int key, first, count; bool mixed; };   // tensors that share types: one launch each
    std::vector<DenseChunk> chunks;
    std::vector<Group> groups;
    int norm_first = 0, copy_first = 0;
};

enum { KEY_P_BF16 = 1, KEY_G_BF16 = 2, KEY_Q8 = 4, KEY_COUNT = 8 };

inline int dense_key(const tsr_dense_desc &d)
{
    return (d.p_dtype == TSR_BF16 ? KEY_P_BF16 : 0) | (d.g_dtype == TSR_BF16 ? KEY_G_BF16 : 0) | (d.state == TSR_STATE_Q8 ? KEY_Q8 : 0);
}

// Lengths of chunks, and the room that they take at most, whatever the pointers.
struct DenseLayout {
    int step_units[2], norm_units, copy_units;   // units of a chunk when stepping (FP32 and 8-bit states), taking the norm and copying states
    int64_t most_chunks = 0;

    explicit DenseLayout(const std::vector<tsr_dense_desc> &descs)
    {
        // As long as may be, but so many that the GPU fills.
        auto fit = [&](int most, int many) {
            for (;; most /= 2) {
                int64_t chunks = 0, length = (int64_t)most * WARPS * UNIT;
                for (const tsr_dense_desc &d : descs) chunks += (d.rows * d.cols + length - 1) / length + 1;
                if (most == 1 || chunks >= many) return most * WARPS;
            }
        };
        step_units[TSR_STATE_F32] = fit(STEP_F32_UNITS, MANY_CHUNKS);
        step_units[TSR_STATE_Q8] = fit(STEP_Q8_UNITS, MANY_CHUNKS);
        norm_units = fit(NORM_UNITS, MANY_CHUNKS);
        copy_units = fit(COPY_UNITS, 2 * MANY_CHUNKS);
        for (const tsr_dense_desc &d : descs) {
            const int64_t n = d.rows * d.cols;
            int64_t step = 0, norm = 0;
            for (int k = 0; k < 8; ++k) {   // every path that a binding can come to
                const bool image = k & 1, states = k & 2, vectors = k & 4;
                if (d.flags == 0) step = std::max(step, DenseCuts(n, dense_step_path(d, image, states, vectors), step_units[d.state]).count());
                if (d.flags != TSR_DENSE_STATE_ONLY) norm = std::max(norm, DenseCuts(n, dense_norm_path(d, vectors), norm_units).count());
            }
            most_chunks += step + norm + (d.flags != TSR_DENSE_NORM_ONLY ? DenseCuts(n, PATH_VECTORS, copy_units).count() : 0);
        }
    }

    // Paths of tensor i of a binding (tensors without elements have none).
    static DensePath norm_path(const tsr_dense_desc &d, const tsr_dense_ptrs &p)
    {
        return dense_norm_path(d, dense_aligned(p.grad, 8 * dense_size_of(d.g_dtype)));
    }
    static bool state_vectors(const tsr_dense_desc &d, const tsr_dense_ptrs &p)
    {
        const int64_t bytes = d.state == TSR_STATE_Q8 ? 8 : 32;
        return dense_aligned(p.m, bytes) && dense_aligned(p.v, bytes);
    }
    static DensePath step_path(const tsr_dense_desc &d, const tsr_dense_ptrs &p)
    {
        return dense_step_path(d, p.image != nullptr, state_vectors(d, p),
                               dense_aligned(p.grad, 8 * dense_size_of(d.g_dtype)) && dense_aligned(p.param, 8 * dense_size_of(d.p_dtype)) && dense_aligned(p.image, 16));
    }

    DenseTable fill(const std::vector<tsr_dense_desc> &descs, const tsr_dense_ptrs *ptrs) const
    {
        DenseTable t;
        t.chunks.reserve((size_t)most_chunks);
        auto add = [&](size_t i, DensePath how, int at_once) {
            const DenseCuts cut(descs[i].rows * descs[i].cols, how, at_once);
            for (int64_t k = 0; k < cut.whole; k += cut.length)
                t.chunks.push_back({(int32_t)i, (uint32_t)k, (int32_t)std::min(cut.length, cut.whole - k), how});
            if (cut.whole < cut.units) t.chunks.push_back({(int32_t)i, (uint32_t)cut.whole, 1, PATH_ANY});
        };
        for (int key = 0; key < KEY_COUNT; ++key) {
            const int first = (int)t.chunks.size();
            for (size_t i = 0; i < descs.size(); ++i)
                if (descs[i].flags == 0 && dense_key(descs[i]) == key) add(i, step_path(descs[i], ptrs[i]), step_units[descs[i].state]);
            const int got = (int)t.chunks.size() - first;
            const bool mixed = std::any_of(t.chunks.begin() + first, t.chunks.end(), [](const DenseChunk &c) { return c.path != PATH_VECTORS; });
            if (got) t.groups.push_back({key, first, got, mixed});
        }
        t.norm_first = (int)t.chunks.size();
        for (size_t i = 0; i < descs.size(); ++i)
            if (descs[i].flags != TSR_DENSE_STATE_ONLY) add(i, norm_path(descs[i], ptrs[i]), norm_units);
        t.copy_first = (int)t.chunks.size();
        for (size_t i = 0; i < descs.size(); ++i)
            if (descs[i].flags != TSR_DENSE_NORM_ONLY) add(i, PATH_VECTORS, copy_units);
        return t;
    }
};

}  // namespace tsr
