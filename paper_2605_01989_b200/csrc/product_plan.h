// How a matrix product is cut into tiles and parts: host arithmetic alone, which builds without CUDA.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "device.h"

namespace dblp {

constexpr uint32_t kStep = 64;                                  // of the summed dimension a stage
constexpr uint32_t kRowMax = 4;                                 // rows that the kernels for few rows take

// A 16-bit operand: its rows (m of A, n of B) and the summed dimension, one of which is contiguous.
struct Operand {
    const void* p;
    const void* lo;             // second word of each element (terms = 3), or null
    int64_t stride;             // of the other dimension, in elements
    int64_t each;               // from one product of a batch to the next
    bool mn;                    // the rows are contiguous, not the summed dimension
};

struct Product {
    Operand a, b;
    uint32_t M, N, K, batch;
    int dtype;                  // of both operands
    int terms;                  // 1, or 3: hi hi + hi lo + lo hi
    bool few;                   // few rows (M) may be computed as columns
    bool symmetric;             // M = N and the result equals its transpose: computed once, written twice
};

struct ProductPlan {
    int cg;
    uint32_t bn, mt, nt, tiles, whole, rest, parts, per, steps, term_steps;
    bool turned;                                                // A and B change places
    bool copy_a, copy_b;
    uint32_t a_to, b_to;                                        // rows of the copies
    size_t a_bytes, b_bytes, partial_bytes;                     // in workspace
    uint32_t items;                                             // whole tiles and parts
    uint32_t longest;                                           // stages of the longest item
    bool several;                                               // blocks have several items: results may go by TMA
};

inline bool tma_reads(const Operand& o, uint32_t outer, uint32_t inner, uint32_t batch)
{
    if (((uintptr_t)o.p | (uintptr_t)o.lo) % 16 != 0) return false;
    if (outer > 1 && (o.stride % 8 != 0 || o.stride < (int64_t)inner || o.stride >= (1ll << 38))) return false;
    return batch <= 1 || o.each % 8 == 0;
}

inline uint64_t count_tiles(bool symmetric, uint32_t tm, uint32_t bn, uint32_t mt, uint32_t nt)
{
    if (!symmetric) return (uint64_t)mt * nt;
    uint64_t n = 0;
    for (uint32_t i = 0; i < mt; ++i) n += nt - (uint32_t)((uint64_t)i * tm / bn);
    return n;
}

inline ProductPlan plan_product(const Product& p)
{
    ProductPlan r{};
    auto padded = [](size_t b) { return (b + 255) & ~(size_t)255; };
    const uint32_t ai = p.a.mn ? p.M : p.K, ao = p.a.mn ? p.K : p.M, bi = p.b.mn ? p.N : p.K, bo = p.b.mn ? p.K : p.N;
    r.copy_a = !tma_reads(p.a, ao, ai, p.batch);
    r.copy_b = !tma_reads(p.b, bo, bi, p.batch);
    r.a_to = (ai + 7) & ~7u;
    r.b_to = (bi + 7) & ~7u;
    r.a_bytes = r.copy_a ? padded((size_t)ao * r.a_to * 2) : 0;
    r.b_bytes = r.copy_b ? padded((size_t)bo * r.b_to * 2) : 0;
    r.term_steps = (p.K + kStep - 1) / kStep;
    r.steps = r.term_steps * p.terms;
    // Few rows become the columns of narrow tiles, which read B (weights) once and waste no products on rows that are not there.
    r.turned = p.few && p.M <= 128 && p.M < p.N && !p.a.mn;
    const uint32_t M = r.turned ? p.N : p.M, N = r.turned ? p.M : p.N;
    // The shape and the cut with the shortest estimate, in cycles: `step` is what a stage was measured to take (64 x 8192 x 8192 and the
    // like), by issue for small tiles and by L2 for large ones.  Tiles fill the machine in rounds; those of the last, incomplete
    // round (all, where there is no other) may be done in parts, which cost a second kernel and their way through memory.
    double best = 1e300;
    const struct { int cg; uint32_t bn; double step; } shapes[] = {{2, 256, 560}, {2, 128, 360}, {1, 256, 720}, {1, 128, 490}, {1, 64, 360}, {1, 32, 340}, {1, 16, 320}};
    for (const auto& c : shapes) {
        if (r.turned ? (c.cg == 2 || (c.bn >= 2 * N && c.bn > 16)) : c.bn < 64) continue;
        if (r.turned && c.bn < N && c.bn < 128) continue;
        const uint32_t tm = 128 * c.cg, mt = (uint32_t)(((uint64_t)M + tm - 1) / tm), nt = (N + c.bn - 1) / c.bn;
        const uint64_t tiles = count_tiles(p.symmetric, tm, c.bn, mt, nt), slots = kSms / c.cg, all = tiles * p.batch, last = all % slots;
        if (all >= 1ull << 30) continue;
        for (uint32_t parts = 1; parts <= 16 && parts <= r.steps; ++parts) {
            if (parts > 1 && last == 0) break;
            const uint32_t per = (r.steps + parts - 1) / parts;
            if ((r.steps + per - 1) / per != parts) continue;
            const uint64_t rounds = all / slots, cut = (last * parts + slots - 1) / slots;
            double t = (double)(rounds * r.steps + cut * per) * c.step + 4000 + 10.0 * c.bn;
            if (parts > 1) t += 5000 + (double)last * parts * tm * c.bn * 8 / 2500;
            if (t < best) {
                best = t;
                r.cg = c.cg;
                r.bn = c.bn;
                r.mt = mt;
                r.nt = nt;
                r.tiles = (uint32_t)tiles;
                r.parts = parts;
                r.per = per;
                r.rest = parts > 1 ? (uint32_t)last : 0;
                r.whole = (uint32_t)(all - r.rest);
            }
        }
    }
    r.items = r.whole + r.rest * r.parts;
    r.longest = r.whole ? r.steps : r.per;
    // For one tile a block TMA's latency (1.5 us) is longer than what it saves.
    r.several = r.cg && !r.turned && !p.symmetric && r.items > kSms / r.cg;
    r.partial_bytes = padded((size_t)r.rest * r.parts * 128 * r.cg * r.bn * 4);
    return r;
}

// Stages that the tensor cores add up by themselves where sums are taken in runs.  One term: error of 8192 products of random signs 9.1e-6 of
// the result in one run, 4.7e-7 in runs of 512 terms, 2.4e-7 of 256; plain fp32 9.6e-7 (all of one sign: 2.8e-6 for f16, 9e-7 for bf16).
// Three terms, for results that the next products amplify: runs of 192 terms, 128 below 1024 rows or columns, 64 below 512, so that the orthogonalised
// update stays as near as the iteration in fp32, whose own error grows with the size.  In runs of 256 throughout 384 x 640 is off by 5.1e-6, with
// this 2.0e-6 (fp32 2.5e-6), at 152 and 160 us; 700 x 4000 6.8e-6 and 3.7e-6 (3.7e-6), 312 and 354 us; 6400 x 1600 5.9e-6 and 4.6e-6 (5.1e-6), 1.15 and 1.22 ms.
inline uint32_t run_stages(const Product& p)
{
    if (p.terms == 1) return 8;
    const uint32_t low = p.M < p.N ? p.M : p.N;
    return low < 512 ? 1 : (low < 1024 ? 2 : 3);
}

// Whether the kernels for up to four rows take it: B in whole 16-byte groups of one of its rows; where the summed dimension is the
// contiguous one, in whole groups altogether, and A aligned like it.
inline bool rows_take(const Product& p)
{
    if (!p.few || p.M > kRowMax || p.a.mn || p.K == 0) return false;
    if (p.b.mn) return p.N % 8 == 0 && tma_reads(p.b, p.K, p.N, 1);
    return p.K % 8 == 0 && tma_reads(p.b, p.N, p.K, 1) && tma_reads(p.a, p.M, p.K, 1);
}

}  // namespace dblp
