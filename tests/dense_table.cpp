// Host check of a dense plan's table: whatever the shapes, types, pitches and pointers, what is filled in fits the room that was
// reserved before the pointers were known, covers every unit once, and takes no path that its pointers do not allow.
#include "tsr_dense_table.h"

#include <stdio.h>
#include <stdlib.h>

using namespace tsr;

static uint64_t state = 88172645463325252ull;
static uint64_t pick(uint64_t n) { state ^= state << 13; state ^= state >> 7; state ^= state << 17; return (state >> 11) % n; }

static int failures = 0;
#define CHECK(cond, i, d) \
    do { if (!(cond) && ++failures < 20) printf("tensor %zu (%lld x %lld, pitches %lld %lld %lld, state %d): %s\n", i, (long long)d.rows, (long long)d.cols, \
                                               (long long)d.ldp, (long long)d.ldg, (long long)d.ldi, d.state, #cond); } while (0)

static void check(const std::vector<tsr_dense_desc> &descs, const std::vector<tsr_dense_ptrs> &ptrs)
{
    const DenseLayout layout(descs);
    const DenseTable t = layout.fill(descs, ptrs.data());
    if ((int64_t)t.chunks.size() > layout.most_chunks && ++failures < 20)
        printf("%zu chunks, room for %lld: first tensor %lld x %lld, pitches %lld %lld, state %d, m %p\n", t.chunks.size(), (long long)layout.most_chunks,
               (long long)descs[0].rows, (long long)descs[0].cols, (long long)descs[0].ldp, (long long)descs[0].ldg, descs[0].state, ptrs[0].m);
    const int ends[4] = {0, t.norm_first, t.copy_first, (int)t.chunks.size()};
    for (int list = 0; list < 3; ++list) {
        std::vector<int64_t> next(descs.size(), 0);
        for (int c = ends[list]; c < ends[list + 1]; ++c) {
            const DenseChunk &k = t.chunks[c];
            const size_t i = k.rec;
            const tsr_dense_desc &d = descs[i];
            const tsr_dense_ptrs &p = ptrs[i];
            const int64_t n = d.rows * d.cols;
            CHECK((int64_t)k.first == next[i] && k.units > 0, i, d);
            next[i] += k.units;
            CHECK(k.path == PATH_ANY || next[i] * UNIT <= n, i, d);
            const bool row = d.rows <= 1, q8 = d.state == TSR_STATE_Q8;
            const bool codes = !q8 || (((uintptr_t)p.m | (uintptr_t)p.v) & 7) == 0;
            if (list == 0) {
                const bool together = row || (d.ldp == d.cols && d.ldg == d.cols && (!p.image || d.ldi == d.cols));
                if (k.path != PATH_ANY) CHECK(codes, i, d);
                if (k.path == PATH_VECTORS || k.path == PATH_PLAIN) CHECK(together, i, d);
                if (k.path == PATH_ROWS) CHECK(d.cols >= UNIT && std::max(d.ldp, d.ldg) < (1 << 30) && (!p.image || d.ldi < (1 << 30)), i, d);
                if (k.path == PATH_VECTORS) {
                    const int ps = d.p_dtype == TSR_BF16 ? 16 : 32, gs = d.g_dtype == TSR_BF16 ? 16 : 32, ms = q8 ? 8 : 32;
                    CHECK((uintptr_t)p.param % ps == 0 && (uintptr_t)p.grad % gs == 0 && (uintptr_t)p.m % ms == 0 && (uintptr_t)p.v % ms == 0 && (uintptr_t)p.image % 16 == 0, i, d);
                }
            } else if (list == 1) {
                if (k.path == PATH_VECTORS || k.path == PATH_PLAIN) CHECK(row || d.ldg == d.cols, i, d);
                if (k.path == PATH_VECTORS) CHECK((uintptr_t)p.grad % (d.g_dtype == TSR_BF16 ? 16 : 32) == 0, i, d);
                if (k.path == PATH_ROWS) CHECK(d.cols >= UNIT && d.ldg < (1 << 30), i, d);
            }
        }
        for (size_t i = 0; i < descs.size(); ++i) {
            const tsr_dense_desc &d = descs[i];
            const bool in = list == 0 ? d.flags == 0 : list == 1 ? d.flags != TSR_DENSE_STATE_ONLY : d.flags != TSR_DENSE_NORM_ONLY;
            CHECK(next[i] == (in ? (d.rows * d.cols + UNIT - 1) / UNIT : 0), i, d);
        }
    }
    for (size_t g = 0; g < t.groups.size(); ++g)
        for (int c = t.groups[g].first; c < t.groups[g].first + t.groups[g].count; ++c)
            if ((t.chunks[c].path != PATH_VECTORS && !t.groups[g].mixed) || dense_key(descs[t.chunks[c].rec]) != t.groups[g].key)
                if (++failures < 20) printf("chunk %d is in the wrong group\n", c);
}

// off_state: bytes off the alignment of vectors (m, and v beside it); off: elements of parameter, gradient and image
static void add(std::vector<tsr_dense_desc> &descs, std::vector<tsr_dense_ptrs> &ptrs, int64_t rows, int64_t cols, const int64_t (&more)[3], int types, int off_m, int off_v, int off)
{
    tsr_dense_desc d = {rows, cols, cols + more[0], cols + more[1], cols + more[2], (types & 1) ? TSR_BF16 : TSR_F32, (types & 2) ? TSR_BF16 : TSR_F32,
                        (types & 4) ? TSR_STATE_Q8 : TSR_STATE_F32, 0, 1.f, 1.f};
    const uintptr_t base = 1 << 20;
    const int es = (types & 4) ? 1 : 4;
    const bool image = (types & 8) && !(types & 1);
    descs.push_back(d);
    ptrs.push_back({(void *)(base + off * ((types & 1) ? 2 : 4)), (const void *)(base + off * ((types & 2) ? 2 : 4)), (void *)(base + off_m * es), (void *)(base + off_v * es),
                    (float *)base, image ? (void *)(base + 2 * off) : nullptr});
}

int main()
{
    const int64_t sizes[][2] = {{1, 1}, {1, 255}, {1, 256}, {1, 257}, {1, 300}, {1, 2047}, {1, 2049}, {1, 70000}, {1, 1 << 20}, {1, 2 << 20}, {1, 4 << 20}, {1, 4000001},
                                {1, 40000000}, {32000, 2048}, {2048, 5461}, {100, 255}, {100, 256}, {100, 257}, {300000, 7}, {3000000, 1}, {2, 3000000}, {0, 5}, {5, 0}};
    const int64_t pitches[][3] = {{0, 0, 0}, {3, 0, 0}, {0, 3, 0}, {0, 0, 3}, {1, 2, 8}, {(int64_t)1 << 30, 0, 0}, {0, (int64_t)1 << 30, 0}, {0, 0, (int64_t)1 << 30}};
    long plans = 0;
    for (const auto &s : sizes)
        for (const auto &more : pitches)
            for (int types = 0; types < 16; ++types)
                for (int off = 0; off < 2; ++off)
                    for (int off_state = 0; off_state < 4; ++off_state) {
                        std::vector<tsr_dense_desc> descs;
                        std::vector<tsr_dense_ptrs> ptrs;
                        add(descs, ptrs, s[0], s[1], more, types, off_state & 1, (off_state >> 1) * 2, off);
                        check(descs, ptrs);
                        ++plans;
                    }
    for (int k = 0; k < 3000; ++k) {   // several tensors, some with a flag
        std::vector<tsr_dense_desc> descs;
        std::vector<tsr_dense_ptrs> ptrs;
        for (uint64_t i = 0, count = 1 + pick(12); i < count; ++i) {
            const int64_t n = (int64_t)1 << pick(23), cols = 1 + (int64_t)pick((uint64_t)n), rows = std::max<int64_t>(1, n / cols);
            const int64_t more[3] = {(int64_t)(pick(2) * pick(9)), (int64_t)(pick(2) * pick(9)), (int64_t)(pick(2) * pick(9))};
            add(descs, ptrs, rows, cols, more, (int)pick(16), (int)(pick(2) * pick(9)), (int)(pick(2) * pick(9)), (int)(pick(2) * pick(9)));
            descs.back().flags = pick(5) ? 0 : (int32_t)(1 + pick(2));
        }
        check(descs, ptrs);
        ++plans;
    }
    printf("%ld plans, %d failures\n", plans, failures);
    return failures != 0;
}
