// Matrix products on the tensor cores, with an epilogue on sixteen columns of a row at a time.
//
// A work item is a tile of the result: 128 rows a block (256 for a pair of blocks, which share B's columns) by up to 256
// columns, or a part of the summed dimension of such a tile.  A block is persistent and walks over items; two warps load (TMA, 64
// of the summed dimension a stage), one issues the products, eight write the sums of the item before out of the other half of
// tensor memory.
//   operands   either dimension of an operand may be the contiguous one: the shared-memory layout serves both ways, so x w, dy w^T
//              and x^T dy read the same tensors without a transposed copy.  Rows that TMA cannot address (not on 16 bytes) are
//              copied first.
//   epilogue   a thread has a row of 32 sums.  Whole pieces of 32 x 32 go out by TMA from shared memory where blocks have several tiles,
//              from the threads where they have one; edges and unaligned matrices an element a lane.  Read by columns, a piece is a
//              piece of the transposed result: this is how the mirror of a symmetric result is written, and how few rows are
//              computed (as columns of the tile).
//   parts      tiles of the last, incomplete round are cut along the summed dimension; the parts' sums are added in order by a
//              second kernel with the same epilogue.
//   fp32       the tensor cores' sums truncate; where the result is fp32, and where a sum is long, they are taken out in runs (run_stages) and
//              added up in registers.
//   bound      256 x 256 tiles by the tensor pipe under the power cap, like the library's product (a pair needs 64 bytes a cycle and
//              multiprocessor from L2, about what it gives: five stages instead of six cost 10 %, four 30 %); tiles of 128 columns by
//              the 340 cycles that a stage takes to issue; with bias, gelu and a second result by the writing warps: 22 900
//              cycles a tile of 1600 before edges left their code, 12 800 of products.
//   measured   8192 x 8192 x 8192 bf16 691 to 760 us (1.45 to 1.59 PFLOP/s; the library's 649 to 690 on the same machines), 8192 x 1600 -> 6400
//              110 us (1.52), with bias, gelu and pre-activation 135 us (1.25).
#pragma once

#include "product.cuh"
#include "tc.cuh"

namespace dblp {

constexpr int kProdThreads = 384, kProdWriters = 8;             // warps 0 .. 7 write, 8 and 10 load A and B, 9 issues products, 11 idles
// With runs a writer holds 128 sums: registers move to the writers' two warpgroups from the third.  An increase waits until the block's
// own registers allow it, so the shares may not be more than what the block was launched with: 168 a thread, the most that 384
// threads can have.  build.py looks at what the compiler gave.
constexpr int kRunRegs = 168, kRunWriterRegs = 224, kRunOtherRegs = 56;
static_assert(kProdWriters * 32 * kRunWriterRegs + (kProdThreads - kProdWriters * 32) * kRunOtherRegs == kProdThreads * kRunRegs, "registers of a block");
constexpr uint32_t kMaxStages = 8;
constexpr uint32_t kPieceBytes = 32 * 32 * 4;                   // what a writing warp brings through shared memory at a time
constexpr uint32_t kProdSmem = 227 * 1024 - 512;                // what a block may use, less its barriers

struct ProductArgs {
    CUtensorMap a[2], b[2], o[2];                               // first and second words; results, pieces of 32 x 32
    uint32_t M, N, tm, bn, mt, nt;                              // tiles of tm = 128 (256) rows x bn columns
    uint32_t steps, term_steps;                                 // stages of a tile (terms together), of a term
    uint32_t whole, rest, parts, per, items;                    // tiles done whole; tiles done in parts of `per` stages; items in all
    uint32_t group, tiles;                                      // tile rows walked together; tiles of one product
    FastDiv by_tiles, by_rest, by_all, by_group, by_last;
    uint32_t stages, stage_bytes, b_bytes, acc_cols, idesc;
    uint32_t run;                                               // stages that the tensor cores add up by themselves (RUNS)
    uint32_t a_mn, b_mn, symmetric, turned, direct, bulk;       // bulk: bit k, result k goes by TMA (bit 2: it is fp32); 0: none does
    float* partial;                                             // [rest][parts][tm][bn]
    unsigned long long* timeouts;
};

struct ProdItem {
    uint32_t i, j, b, k0, k1;                                   // tile, product, stages
    uint32_t slot;                                              // where its sums go in `partial`; kWhole: to the epilogue
};
constexpr uint32_t kWhole = 0xFFFFFFFFu;

// Tile number g of all products.
__host__ __device__ __forceinline__ void place_tile(const ProductArgs& a, uint32_t g, ProdItem& t)
{
    t.b = a.by_tiles.div(g);
    uint32_t y = g - t.b * a.tiles;
    if (a.symmetric) {                                          // tiles that reach the diagonal or lie above it, row by row
        uint32_t i = 0, first = 0;
        while (y >= a.nt - first) {
            y -= a.nt - first;
            ++i;
            first = i * a.tm / a.bn;
        }
        t.i = i;
        t.j = first + y;
    } else {                                                    // `group` tile rows together, column by column: operands stay in L2
        const uint32_t q = a.by_all.div(y), first = q * a.group, r = y - q * a.group * a.nt;
        const bool last = first + a.group > a.mt;
        t.j = last ? a.by_last.div(r) : a.by_group.div(r);
        t.i = first + r - t.j * (last ? a.mt - first : a.group);
    }
}

__host__ __device__ __forceinline__ ProdItem prod_item(const ProductArgs& a, uint32_t x)
{
    ProdItem t;
    t.k0 = 0;
    t.k1 = a.steps;
    t.slot = kWhole;
    if (x >= a.whole) {
        const uint32_t y = x - a.whole, part = a.by_rest.div(y), n = y - part * a.rest;
        t.k0 = part * a.per;
        t.k1 = t.k0 + a.per < a.steps ? t.k0 + a.per : a.steps;
        t.slot = n * a.parts + part;
        x = a.whole + n;
    }
    place_tile(a, x, t);
    return t;
}

// Elements 0 .. n - 1 by one lane, what eight of them read fetched together.
template <typename F, typename A> __device__ __forceinline__ void one_by_one(uint32_t n, const F& fetch, const A& apply)
{
    for (uint32_t i = 0; i < n; i += 8) {
        float2 f[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k)
            if (i + k < n) f[k] = fetch(i + k);
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k)
            if (i + k < n) apply(i + k, f[k]);
    }
}

// Where the run of stages that begins at stage k ends: the tensor cores add up a run by themselves.  The second and third terms are
// smaller than the first by 2^-11, and so is what truncation takes from them: they are one run.
__device__ __forceinline__ uint32_t run_end(const ProductArgs& a, uint32_t k, uint32_t k1)
{
    return min(k < a.term_steps ? min(k + a.run, a.term_steps) : a.steps, k1);
}

// 32 x 32 sums, a row a lane, from (r0, c0) on.  Whole pieces of matrices that allow 32-byte accesses are written from the lane that has
// the row; what the epilogue reads is fetched before `sums` brings v.  The others, and results written by columns, go through
// 4 KB of shared memory, where the 16-byte chunk c of row r is at place c ^ (r % 8): no bank conflicts in any direction.  Edges and
// unaligned matrices are written an element a lane, a row at a time.
template <typename E, typename F>
__device__ __forceinline__ void write_piece(const ProductArgs& a, const E& e, uint32_t b, uint32_t r0, uint32_t c0, float* v, uint8_t* piece, const F& sums)
{
    const uint32_t M = a.M, N = a.N, lane = threadIdx.x & 31;
    if (r0 >= M || c0 >= N || (a.symmetric && c0 < r0)) return;
    if (!E::kMirror && a.bulk) {                                // the piece may still be on its way out
        if (lane == 0) bulk_wait_read<0>();
        __syncwarp();
    }
    auto value = [&](uint32_t r, uint32_t c) { return *reinterpret_cast<const float*>(piece + r * 128 + (((c >> 2) ^ (r & 7)) << 4) + (c & 3) * 4); };
    const bool direct = a.direct && !a.turned && (E::kPadded || (r0 + 32 <= M && c0 + 32 <= N)), mirror = E::kMirror && a.symmetric && c0 > r0;
    if (direct) {
        typename E::Fetched f[2];
        const bool in = r0 + lane < M;
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i)
            if (in && c0 + 16 * i < N) e.fetch(b, r0 + lane, c0 + 16 * i, f[i]);
        sums();
        float copy[32], *y = v;                                 // the mirror needs the sums as they are
        if constexpr (E::kMirror) {
            y = copy;
#pragma unroll
            for (int i = 0; i < 32; ++i) y[i] = v[i];
        }
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i)
            if (in && c0 + 16 * i < N) e.apply(b, r0 + lane, c0 + 16 * i, f[i], y + 16 * i, ToMemory());
        if (!mirror) return;
    } else {
        sums();
    }
    __syncwarp();
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
        *reinterpret_cast<float4*>(piece + lane * 128 + ((i ^ (lane & 7)) << 4)) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    __syncwarp();
    if constexpr (E::kMirror) {                                 // column `lane` of the piece is part of a row of the transposed result
        if (c0 + lane < N) {
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i) {
                if (r0 + 16 * i >= M) continue;
                typename E::Fetched f;
                float y[16];
                e.fetch(b, c0 + lane, r0 + 16 * i, f);
#pragma unroll
                for (uint32_t k = 0; k < 16; ++k) y[k] = value(16 * i + k, lane);
                e.apply(b, c0 + lane, r0 + 16 * i, f, y, ToMemory());
            }
        }
    } else if constexpr (E::kPadded) {
    } else if (a.turned) {                                      // rows of the result are the piece's columns
        const uint32_t n = min(32u, N - c0);
        if (a.direct && r0 + 32 <= M && n > 4) {
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i) {
                const uint32_t c = lane / 2 + 16 * i, first = (lane & 1) * 16;
                if (c >= n) continue;
                typename E::Fetched f;
                float y[16];
                e.fetch(b, c0 + c, r0 + first, f);
#pragma unroll
                for (uint32_t k = 0; k < 16; ++k) y[k] = value(first + k, c);
                e.apply(b, c0 + c, r0 + first, f, y, ToMemory());
            }
        } else if (r0 + lane < M) {
            one_by_one(n, [&](uint32_t c) { return e.fetch1(b, c0 + c, r0 + lane); },
                       [&](uint32_t c, float2 f) { e.apply1(b, c0 + c, r0 + lane, f, value(lane, c)); });
        }
    } else if (c0 + lane < N) {
        one_by_one(min(32u, M - r0), [&](uint32_t r) { return e.fetch1(b, r0 + r, c0 + lane); },
                   [&](uint32_t r, float2 f) { e.apply1(b, r0 + r, c0 + lane, f, value(r, lane)); });
    }
    __syncwarp();
}

// A whole piece by way of shared memory and TMA.
template <typename E, typename F>
__device__ __forceinline__ void write_bulk(const ProductArgs& a, const E& e, uint32_t b, uint32_t r0, uint32_t c0, float* v, uint8_t* piece, const F& sums)
{
    const uint32_t lane = threadIdx.x & 31;
    typename E::Fetched f[2];
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) e.fetch(b, r0 + lane, c0 + 16 * i, f[i]);
    sums();
    if (lane == 0) bulk_wait_read<0>();                         // the last piece has left
    __syncwarp();
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) e.apply(b, r0 + lane, c0 + 16 * i, f[i], v + 16 * i, ToPiece{piece, 16 * i});
    fence_async_smem();
    __syncwarp();
    if (lane == 0) {
        if (a.bulk & 1) tma_store3(&a.o[0], piece, (int)c0, (int)r0, (int)b);
        if (a.bulk & 2) tma_store3(&a.o[1], piece + (a.bulk & 4 ? 0 : 2048), (int)c0, (int)r0, (int)b);
        bulk_commit();
    }
    __syncwarp();
}

// The same sums as they are, for the join.
template <typename F>
__device__ __forceinline__ void write_partial(const ProductArgs& a, const ProdItem& t, uint32_t r0, uint32_t c0, float* v, const F& sums)
{
    if (r0 >= a.M || c0 >= a.N || (a.symmetric && c0 < r0)) return;
    sums();
    float* p = a.partial + ((size_t)t.slot * a.tm + (r0 - t.i * a.tm) + (threadIdx.x & 31)) * a.bn + (c0 - t.j * a.bn);
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
        if (8 * i < a.bn) store32(p + 8 * i, reinterpret_cast<const uint32_t*>(v) + 8 * i);
}

template <int CG, bool RUNS, typename E>
__global__ void __launch_bounds__(kProdThreads, 1) k_product(const __grid_constant__ ProductArgs a, const __grid_constant__ E e)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_free[2], idle;
    __shared__ uint32_t tmem_slot, dead;
    uint8_t* ring = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0, first_item = blockIdx.x / CG, item_stride = gridDim.x / CG;

    if (tid == 0) {
        dead = 0;
        for (uint32_t i = 0; i < a.stages; ++i) { bar_init(&full[i], 1); bar_init(&empty[i], 1); }
        for (int i = 0; i < 2; ++i) { bar_init(&acc_full[i], 1); bar_init(&acc_free[i], kProdWriters * CG); }
        bar_init(&idle, 1);
        fence_bar_init();
    }
    if (warp == 9) tmem_alloc_cols<CG>(&tmem_slot, 2 * a.acc_cols);
    if (warp == 8 || warp == 10) prefetch_map(warp == 8 ? a.a : a.b);
    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();
    tc_fence_after();
    const uint32_t tmem = uniform(tmem_slot);
    const Guard g{&dead, a.timeouts};
    wait_before();
    after_start();

    if (warp >= kProdWriters) {
        if (RUNS) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRunOtherRegs));
        if (warp == 8 || warp == 10) {                              // ---- loads: A by one warp, B by another
            const bool is_a = warp == 8, mn = is_a ? a.a_mn : a.b_mn;
            const CUtensorMap* words = is_a ? a.a : a.b;
            const uint32_t boxes = is_a ? 2 : a.b_bytes / 8192, tile = is_a ? 128 * CG : a.bn, mine = rank * (tile / CG);
            const uint32_t full_at = uniform(smem_addr(full)), full_to = CG == 2 ? uniform(in_block(full, 0)) : full_at;
            const uint32_t dst0 = uniform(smem_addr(ring)) + (is_a ? 0 : 128 * 128), end = a.term_steps * kStep;
            uint32_t st = 0, phase = 1, total = 0;                  // the first round of waits passes at once
            bool ok = true, ready = true;
            for (uint32_t x = first_item; x < a.items && ok; x += item_stride) {
                const ProdItem t = prod_item(a, x);
                const int at_row = (int)((is_a ? t.i : t.j) * tile + mine), b = (int)t.b;
                uint32_t term = t.k0 / a.term_steps, at = (t.k0 - term * a.term_steps) * kStep, left = t.k1 - t.k0;
                const CUtensorMap* map = &words[is_a ? term == 2 : term == 1];
                for (; left; --left, ++total) {
                    if (!__all_sync(0xFFFFFFFFu, ready)) ok = warp_wait(&empty[st], phase, g);
                    if (!ok) break;
                    const uint32_t dst = dst0 + st * a.stage_bytes, bar = full_to + st * 8;
                    if (is_a && rank == 0) warp_expect(full_at + st * 8, CG * a.stage_bytes);
                    if (++st == a.stages) { st = 0; phase ^= 1; }
                    ready = bar_test(&empty[st], phase);             // the next stage's, beside this one's loads
                    if (mn)
                        for (uint32_t c = 0; c < boxes; ++c) warp_tma3<CG>(dst + c * 8192, map, bar, at_row + (int)c * 64, (int)at, b);
                    else
                        warp_tma3<CG>(dst, map, bar, (int)at, at_row, b);
                    if ((at += kStep) == end) {
                        at = 0;
                        ++term;
                        map = &words[is_a ? term == 2 : term == 1];
                    }
                }
            }
            if (is_a && rank == 0 && lane == 0) {                   // every copy lands before the block (its pair) may end
                for (uint32_t i = 0; i < min(total, a.stages); ++i) {
                    const uint32_t n = total - 1 - i;
                    bar_drain(&full[n % a.stages], (n / a.stages) & 1);
                }
            }
        } else if (warp == 9) {                                     // ---- products
            if (rank == 0) {
                uint32_t st = 0, phase = 0, w = 0;
                bool ok = true, ready = false;
                const uint64_t a0 = a.a_mn ? desc_mn(smem_addr(ring), 8192) : desc_k(smem_addr(ring));
                const uint64_t b0 = a.b_mn ? desc_mn(smem_addr(ring) + 128 * 128, 8192) : desc_k(smem_addr(ring) + 128 * 128);
                const uint32_t a_step = a.a_mn ? 2048 / 16 : 32 / 16, b_step = a.b_mn ? 2048 / 16 : 32 / 16, stage = a.stage_bytes / 16;
                for (uint32_t x = first_item; x < a.items && ok; x += item_stride) {
                    const ProdItem t = prod_item(a, x);
                    const uint32_t k0 = uniform(t.k0), k1 = uniform(t.k1);
                    uint32_t acc = 0, end = k0;
                    for (uint32_t k = k0; k < k1; ++k) {
                        const bool start = k == end;
                        if (start) {
                            if (w >= 2) ok = warp_wait(&acc_free[w & 1], ((w >> 1) - 1) & 1, g);
                            if (!ok) break;
                            acc = tmem + (w & 1) * a.acc_cols;
                            end = RUNS ? run_end(a, k, k1) : k1;
                        }
                        if (!__all_sync(0xFFFFFFFFu, ready)) ok = warp_wait(&full[st], phase, g);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t now = st;
                        if (++st == a.stages) { st = 0; phase ^= 1; }
                        ready = bar_test(&full[st], phase);         // the next stage's, beside this one's products
                        mma4_commit<CG>(acc, a0 + uniform(now * stage), b0 + uniform(now * stage), a_step, b_step, a.idesc, !start, &empty[now]);
                        if (k + 1 == end) {
                            commit_cg<CG>(&acc_full[w & 1]);
                            ++w;
                        }
                    }
                }
                __syncwarp();
                mma_commit_idle<CG>(&idle);                         // products in flight end before the memory is freed, whoever gave up
                bar_drain(&idle, 0);
            }
        }
    } else {                                                    // ---- sums to their places
        if (RUNS) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRunWriterRegs));
        uint8_t* piece = ring + a.stages * a.stage_bytes + warp * kPieceBytes;
        const uint32_t lanes = (warp & 3) * 32, half = (warp >> 2) * 32;
        uint32_t w = 0;
        bool ok = true;
        for (uint32_t x = first_item; x < a.items && ok; x += item_stride) {
            const ProdItem t = prod_item(a, x);
            const uint32_t r0 = (t.i * CG + rank) * 128 + lanes, c0 = t.j * a.bn + half;
            auto write = [&](uint32_t c, float* v, const auto& sums) {
                if (t.slot != kWhole) write_partial(a, t, r0, c0 + c, v, sums);
                else if (!E::kMirror && a.bulk && r0 + 32 <= a.M && c0 + c + 32 <= a.N) write_bulk(a, e, t.b, r0, c0 + c, v, piece, sums);
                else write_piece(a, e, t.b, r0, c0 + c, v, piece, sums);
            };
            if (RUNS) {
                float2 sums[4][16] = {};
                for (uint32_t k = t.k0; k < t.k1; k = run_end(a, k, t.k1), ++w) {
                    ok = warp_wait(&acc_full[w & 1], (w >> 1) & 1, g);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t acc = tmem + (w & 1) * a.acc_cols + (lanes << 16) + half;
#pragma unroll
                    for (uint32_t p = 0; p < 4; ++p) {
                        if (half + 64 * p >= a.bn) continue;
                        uint32_t v[32];
                        tmem_ld32(acc + 64 * p, v);
                        tmem_wait_ld<32>(v);
#pragma unroll
                        for (int i = 0; i < 16; ++i) sums[p][i] = add2(sums[p][i], pair(v[2 * i], v[2 * i + 1]));
                    }
                    tc_fence_before();
                    if (CG == 2) warp_arrive_in(in_block(&acc_free[w & 1], 0));
                    else warp_arrive(&acc_free[w & 1]);
                }
                if (!ok) break;
#pragma unroll
                for (uint32_t p = 0; p < 4; ++p)
                    if (half + 64 * p < a.bn) write(64 * p, reinterpret_cast<float*>(sums[p]), [] {});
            } else {
                ok = warp_wait(&acc_full[w & 1], (w >> 1) & 1, g);
                if (!ok) break;
                tc_fence_after();
                const uint32_t acc = tmem + (w & 1) * a.acc_cols + (lanes << 16) + half;
                for (uint32_t c = 0; half + c < a.bn; c += 64) {
                    float v[32];
                    auto sums = [&] {
                        __syncwarp();
                        tmem_ld32(acc + c, reinterpret_cast<uint32_t*>(v));
                        tmem_wait_ld<32>(reinterpret_cast<uint32_t*>(v));
                    };
                    write(c, v, sums);
                }
                tc_fence_before();
                if (CG == 2) warp_arrive_in(in_block(&acc_free[w & 1], 0));
                else warp_arrive(&acc_free[w & 1]);
                ++w;
            }
        }
    }
    if (lane == 0) bulk_wait<0>();
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();
    tc_fence_after();
    if (warp == 9) tmem_free_cols<CG>(tmem, 2 * a.acc_cols);
}

// Tiles that were done in parts: a block a piece of 32 x 32.  Warp i adds up parts i, i + 8, ..., the first warp the eight sums, in
// order, and writes.  (One warp a piece, part after part: 10 us for 10 parts, a trip to memory each.)
constexpr int kJoinWarps = 8;
template <typename E> __global__ void __launch_bounds__(32 * kJoinWarps) k_product_join(const __grid_constant__ ProductArgs a, const __grid_constant__ E e)
{
    __shared__ __align__(128) float4 sums[kJoinWarps][8][32];
    wait_before();
    after_start();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, across = (a.bn + 31) / 32, each = a.tm / 32 * across;
    const uint32_t n = blockIdx.x / each, y = blockIdx.x - n * each, pr = y / across, pc = y - pr * across;
    ProdItem t;
    place_tile(a, a.whole + n, t);
    const uint32_t r0 = t.i * a.tm + pr * 32, c0 = t.j * a.bn + pc * 32;
    if (r0 >= a.M || c0 >= a.N || (a.symmetric && c0 < r0)) return;
    if (warp < a.parts) {
        const float* p = a.partial + ((size_t)(n * a.parts + warp) * a.tm + pr * 32 + lane) * a.bn + pc * 32;
        float2 v[16] = {};
#pragma unroll 2
        for (uint32_t s = warp; s < a.parts; s += kJoinWarps, p += (size_t)kJoinWarps * a.tm * a.bn) {
            uint32_t w[32];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (8 * i < a.bn) load32(p + 8 * i, w + 8 * i);
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i)
                if (2 * i < a.bn) v[i] = add2(v[i], pair(w[2 * i], w[2 * i + 1]));
        }
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) sums[warp][i][lane] = make_float4(v[2 * i].x, v[2 * i].y, v[2 * i + 1].x, v[2 * i + 1].y);
    }
    __syncthreads();
    if (warp) return;
    float v[32];
    write_piece(a, e, t.b, r0, c0, v, (uint8_t*)sums, [&] {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            float4 x = sums[0][i][lane];
            for (uint32_t k = 1; k < min(a.parts, (uint32_t)kJoinWarps); ++k) {
                const float4 q = sums[k][i][lane];
                x = make_float4(x.x + q.x, x.y + q.y, x.z + q.z, x.w + q.w);
            }
            v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
        }
    });
}

// Nothing to sum: the epilogue of zeros.
template <typename E> __global__ void __launch_bounds__(256) k_product_none(const __grid_constant__ E e, uint32_t M, uint32_t N)
{
    const uint64_t x = (uint64_t)blockIdx.x * 256 + threadIdx.x, m = x / N;
    const uint32_t n = (uint32_t)(x - m * N);
    if (m < M) e.apply1(0, (uint32_t)m, n, e.fetch1(0, (uint32_t)m, n), 0.0f);
}

// ---- up to four rows -------------------------------------------------------------------------------------------------------
// No tensor cores: B (the weights) passes once, 16 bytes a lane, through fp32 multiply-adds with A's rows; bound by the memory's
// latency and rate.  (1 x 1600 -> 6400 with bias and gelu: 10.0 us as columns of a tile.)
constexpr int kRowThreads = 256;
constexpr uint32_t kRowCols = 64, kRowLoads = 8;
struct RowsArgs {
    const void *x, *w;
    int64_t xs, ws;
    uint32_t M, N, K, splits, per;              // per: of the summed dimension a block, where it is cut
};

template <typename T> __device__ __forceinline__ void fma8(const uint4& w, float x, float2* acc)
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = fma2(unpack2<T>(u[i]), make_float2(x, x), acc[i]);
}

// B's columns are contiguous: a block takes 64 of them, eight lanes a line of 128 bytes, 32 lines at once.  The blocks of a cluster
// share the summed dimension; the first adds their sums in order.
template <typename T, int M, typename E> __global__ void __launch_bounds__(kRowThreads) k_rows_wide(const __grid_constant__ RowsArgs a, const __grid_constant__ E e)
{
    __shared__ float part[32][M][kRowCols + 4], sums[8][M][kRowCols];
    const uint32_t g = threadIdx.x & 7, line = threadIdx.x >> 3, rank = a.splits > 1 ? cluster_rank() : 0, first = blockIdx.x / a.splits * kRowCols;
    const uint32_t n = first + g * 8, k0 = rank * a.per, k1 = min(a.K, k0 + a.per);
    const T *w = (const T*)a.w + n, *x = (const T*)a.x;
    float2 acc[M][4] = {};
    if (n < a.N)
        for (uint32_t k = k0 + line; k < k1; k += 32 * kRowLoads) {
            uint4 q[kRowLoads];
            float f[kRowLoads][M];
#pragma unroll
            for (uint32_t u = 0; u < kRowLoads; ++u) {
                const uint32_t r = min(k + 32 * u, k1 - 1);
                q[u] = __ldg(reinterpret_cast<const uint4*>(w + (int64_t)r * a.ws));
#pragma unroll
                for (int m = 0; m < M; ++m) f[u][m] = k + 32 * u < k1 && (uint32_t)m < a.M ? to_f32(x[m * a.xs + r]) : 0.0f;
            }
#pragma unroll
            for (uint32_t u = 0; u < kRowLoads; ++u)
                if (k + 32 * u < k1)
#pragma unroll
                    for (int m = 0; m < M; ++m) fma8<T>(q[u], f[u][m], acc[m]);
        }
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<float2*>(&part[line][m][g * 8 + 2 * i]) = acc[m][i];
    __syncthreads();
    if (a.splits > 1) cluster_sync();                           // the first block is there before anything is written to it
    for (uint32_t i = threadIdx.x; i < M * kRowCols; i += kRowThreads) {
        float t = 0.0f;
#pragma unroll
        for (int l = 0; l < 32; ++l) t += part[l][i / kRowCols][i % kRowCols];
        if (a.splits > 1) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(in_block(&sums[rank][i / kRowCols][i % kRowCols], 0)), "f"(t) : "memory");
        else sums[0][i / kRowCols][i % kRowCols] = t;
    }
    if (a.splits > 1) cluster_sync();
    else __syncthreads();
    if (rank) return;
    for (uint32_t i = threadIdx.x; i < a.M * kRowCols; i += kRowThreads) {
        const uint32_t m = i / kRowCols, c = i % kRowCols;
        if (first + c >= a.N) continue;
        float t = sums[0][m][c];
        for (uint32_t r = 1; r < a.splits; ++r) t += sums[r][m][c];
        e.apply1(0, m, first + c, e.fetch1(0, m, first + c), t);
    }
}

// The summed dimension is contiguous: a warp takes two of B's rows.
template <typename T, int M, typename E> __global__ void __launch_bounds__(kRowThreads) k_rows_long(const __grid_constant__ RowsArgs a, const __grid_constant__ E e)
{
    const uint32_t lane = threadIdx.x & 31, n0 = (blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5)) * 2;
    if (n0 >= a.N) return;
    const T *w[2] = {(const T*)a.w + (int64_t)n0 * a.ws, (const T*)a.w + (int64_t)min(n0 + 1, a.N - 1) * a.ws}, *x = (const T*)a.x;
    float2 acc[2][M] = {};
    for (uint32_t k = lane * 8; k < a.K; k += 1024) {
        uint4 q[2][4], f[M][4];
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            const uint32_t at = k + 256 * u;
            const bool in = at < a.K;                           // K is a multiple of 8
            const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 2; ++j) q[j][u] = in ? __ldg(reinterpret_cast<const uint4*>(w[j] + at)) : zero;
#pragma unroll
            for (int m = 0; m < M; ++m) f[m][u] = in && (uint32_t)m < a.M ? __ldg(reinterpret_cast<const uint4*>(x + m * a.xs + at)) : zero;
        }
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u)
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t ww[4] = {q[j][u].x, q[j][u].y, q[j][u].z, q[j][u].w}, xx[4] = {f[m][u].x, f[m][u].y, f[m][u].z, f[m][u].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[j][m] = fma2(unpack2<T>(ww[i]), unpack2<T>(xx[i]), acc[j][m]);
                }
    }
    float mine = 0.0f;
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float t = acc[j][m].x + acc[j][m].y;
#pragma unroll
            for (int s = 16; s; s >>= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, s);
            if (lane == (uint32_t)(m * 2 + j)) mine = t;
        }
    const uint32_t m = lane / 2, n = n0 + (lane & 1);
    if (m < a.M && n < a.N) e.apply1(0, m, n, e.fetch1(0, m, n), mine);
}

template <typename T, int M, typename E> static int launch_rows(const Product& p, const E& e, cudaStream_t s)
{
    RowsArgs a{p.a.p, p.b.p, p.a.stride, p.b.stride, p.M, p.N, p.K, 1, p.K};
    if (!p.b.mn) {
        k_rows_long<T, M, E><<<(p.N + 15) / 16, kRowThreads, 0, s>>>(a, e);
        DBLP_LAUNCHED();
        return DBLP_OK;
    }
    const uint32_t blocks = (p.N + kRowCols - 1) / kRowCols;
    while (a.splits < 8 && blocks * a.splits < 2 * kSms && p.K / (a.splits * 2) >= 32 * kRowLoads / 2) a.splits *= 2;
    a.per = (p.K + a.splits - 1) / a.splits;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = a.splits;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(blocks * a.splits);
    cfg.blockDim = dim3(kRowThreads);
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = a.splits > 1 ? 1 : 0;
    const auto kernel = k_rows_wide<T, M, E>;
    DBLP_NEXT(cudaLaunchKernelEx(&cfg, kernel, a, e));
    return DBLP_OK;
}
template <typename E> static int product_rows(const Product& p, const E& e, cudaStream_t s)
{
    using T = typename E::In;
    if (p.M == 1) return launch_rows<T, 1>(p, e, s);
    return p.M == 2 ? launch_rows<T, 2>(p, e, s) : launch_rows<T, 4>(p, e, s);
}

template <int CG, bool RUNS, typename E> static int launch_product(const ProductArgs& a, const E& e, bool chained, cudaStream_t s)
{
    constexpr auto kernel = k_product<CG, RUNS, E>;
    DBLP_CUDA(allow_shared<kernel>(kProdSmem));
    if (RUNS) {                                                 // the split of registers inside counts on this
        static std::atomic<int> regs{0};
        if (regs.load(std::memory_order_acquire) == 0) {
            cudaFuncAttributes fa;
            DBLP_CUDA(cudaFuncGetAttributes(&fa, kernel));
            regs.store(fa.numRegs, std::memory_order_release);
        }
        DBLP_REQUIRE(regs.load(std::memory_order_acquire) == kRunRegs, DBLP_ECUDA, "product: built with %d registers a thread, not %d", regs.load(), kRunRegs);
    }
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg{};
    const uint32_t slots = kSms / CG;
    cfg.gridDim = dim3((a.items < slots ? a.items : slots) * CG);
    cfg.blockDim = dim3(kProdThreads);
    cfg.dynamicSmemBytes = 1024 + a.stages * a.stage_bytes + kProdWriters * kPieceBytes;
    cfg.stream = s;
    cfg.attrs = attr;
    if (CG == 2) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim.x = 2;
        attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    if (chained) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
        ++cfg.numAttrs;
    }
    DBLP_NEXT(cudaLaunchKernelEx(&cfg, kernel, a, e));
    return DBLP_OK;
}

template <bool RUNS, typename E> int run_product(const Product& p, const E& e, void* ws, bool chained, cudaStream_t s)
{
    if constexpr (E::kNothing) if (p.K == 0) {
        const uint64_t blocks = ((uint64_t)p.M * p.N + 255) / 256;
        DBLP_REQUIRE(blocks < 1ull << 31, DBLP_ECAPACITY, "product: 2^39 elements or more");
        k_product_none<E><<<(unsigned)blocks, 256, 0, s>>>(e, p.M, p.N);
        DBLP_LAUNCHED();
        return DBLP_OK;
    }
    if constexpr (E::kFewRows)
        if (rows_take(p)) return product_rows(p, e, s);
    const ProductPlan r = plan_product(p);
    DBLP_REQUIRE(r.cg, DBLP_ECAPACITY, "product: 2^30 tiles or more");
    unsigned long long* timeouts = timeout_counter();
    DBLP_REQUIRE(timeouts, DBLP_ECUDA, "product: no device counter: %s", cudaGetErrorString(cudaGetLastError()));
    Operand oa = p.a, ob = p.b;
    char* at = (char*)ws;
    if (r.copy_a) {
        if (int rc = repack(oa, at, r.a_to, oa.mn ? p.K : p.M, oa.mn ? p.M : p.K, s)) return rc;
        oa.p = at;
        oa.stride = r.a_to;
        at += r.a_bytes;
        chained = true;
    }
    if (r.copy_b) {
        if (int rc = repack(ob, at, r.b_to, ob.mn ? p.K : p.N, ob.mn ? p.N : p.K, s)) return rc;
        ob.p = at;
        ob.stride = r.b_to;
        at += r.b_bytes;
        chained = true;
    }
    if (r.turned) {
        const Operand t = oa;
        oa = ob;
        ob = t;
    }
    ProductArgs a{};
    a.M = r.turned ? p.N : p.M;
    a.N = r.turned ? p.M : p.N;
    for (int i = 0; i < (p.terms > 1 ? 2 : 1); ++i) {
        if (int rc = make_map(&a.a[i], i ? oa.lo : oa.p, oa.stride, oa, a.M, p.K, p.batch, 128, p.dtype)) return rc;
        if (int rc = make_map(&a.b[i], i ? ob.lo : ob.p, ob.stride, ob, a.N, p.K, p.batch, r.bn / r.cg, p.dtype)) return rc;
    }
    a.tm = 128 * r.cg;
    a.bn = r.bn;
    a.mt = r.mt;
    a.nt = r.nt;
    a.steps = r.steps;
    a.term_steps = r.term_steps;
    a.run = run_stages(p);
    a.whole = r.whole;
    a.rest = r.rest;
    a.parts = r.parts;
    a.per = r.per;
    a.items = r.items;
    a.group = 8 / r.cg;
    a.tiles = r.tiles;
    a.by_tiles = FastDiv(r.tiles);
    a.by_rest = FastDiv(r.rest ? r.rest : 1);
    a.by_all = FastDiv(a.group * r.nt);
    a.by_group = FastDiv(a.group);
    a.by_last = FastDiv(r.mt % a.group ? r.mt % a.group : a.group);
    a.a_mn = oa.mn;
    a.b_mn = ob.mn;
    a.symmetric = p.symmetric;
    a.turned = r.turned;
    a.b_bytes = (r.bn / r.cg) * 128;
    a.stage_bytes = 128 * 128 + a.b_bytes;
    const uint32_t room = (kProdSmem - 1024 - kProdWriters * kPieceBytes) / a.stage_bytes;
    a.stages = room < kMaxStages ? room : kMaxStages;
    a.acc_cols = r.bn < 32 ? 32 : r.bn;
    a.idesc = p.dtype == DBLP_BF16 ? mma_desc<__nv_bfloat16>(128 * r.cg, r.bn, oa.mn, ob.mn) : mma_desc<__half>(128 * r.cg, r.bn, oa.mn, ob.mn);
    a.timeouts = timeouts;
    a.direct = e.sectors();
    if (a.direct && r.several) {
        const Output o[2] = {e.output(0), e.output(1)};
        const bool down = p.M <= 1 || ((!o[0].p || o[0].stride > 0) && (!o[1].p || o[1].stride > 0));      // TMA knows no negative strides
        if (down && !(o[0].p && o[1].p && o[1].bytes == 4)) {   // a 16-bit and an fp32 piece together are more than there is room for
            for (int k = 0; k < 2; ++k) {
                if (!o[k].p) continue;
                if (int rc = make_store_map(&a.o[k], o[k], p)) return rc;
                a.bulk |= 1u << k | (o[k].bytes == 4 ? 4u : 0u);
            }
        }
    }
    a.partial = (float*)at;
    auto launch = [&](auto runs) -> int {
        constexpr bool R = decltype(runs)::value;
        return r.cg == 2 ? launch_product<2, R>(a, e, chained, s) : launch_product<1, R>(a, e, chained, s);
    };
    int rc = 0;
    if constexpr (RUNS) rc = launch(std::true_type());
    else if constexpr (E::kTerms == kAnyTerms) rc = launch(std::false_type());
    else rc = (uint64_t)r.longest * kStep > E::kTerms ? launch(std::true_type()) : launch(std::false_type());
    if (rc) return rc;
    if (r.rest == 0) return DBLP_OK;
    const uint64_t pieces = (uint64_t)r.rest * (a.tm / 32) * ((r.bn + 31) / 32);
    DBLP_NEXT(launch_next(k_product_join<E>, dim3((unsigned)pieces), 32 * kJoinWarps, 0, s, a, e));
    return DBLP_OK;
}

// One epilogue's kernels; RUNS as the calls of run_product ask for it.
#define DBLP_PRODUCT(RUNS, ...) template int run_product<RUNS>(const Product&, const __VA_ARGS__&, void*, bool, cudaStream_t)

}  // namespace dblp
