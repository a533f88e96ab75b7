// dblp_attention_grad on the tensor cores: one pass over the (key tile, query tile) pairs that recomputes the probabilities.
//
//   k_grad_rows   per query row -D_i = -<dout_i, out_i> and -lse_i log2(e), padded to whole tiles: 2 x 4 bytes a row, so
//                 that the main kernel needs neither out nor a reduction.
//   k_grad        one block takes a share of the key tiles of one (sequence, key head) and walks, for each of them, over
//                 all query tiles of the heads that share it.  With keys as rows and queries as columns:
//                     s = k q^T          p = 2^(scale log2(e) s - lse log2(e))
//                     dp = v dout^T      ds = p (dp - D)
//                     dv += p dout       dk += ds q       dq(query tile) = ds^T k
//                 p and ds are 16-bit left operands: p in tensor memory, ds in shared memory, where the same bytes are read
//                 once along the rows (dk) and once across them (dq).  dk and dv stay in tensor memory until the key tile
//                 is done and are written once; shared key heads sum in the same accumulator.
//   k_grad_dq     adds the shares' dq, scales and rounds; k_grad_dkv does the same for key heads whose query heads were
//                 split into groups.
// Order.  A block adds the dq of its key tiles to its own fp32 buffer, in the order of its walk: no two blocks add to one
// place, so the sums do not depend on timing.  The number of shares R is chosen so that the shares
// fill the machine; each costs a buffer of q's size in fp32.
//   warps         0-15 p and ds, each thread one key and 32 queries, with head_dim up to 64 in two groups half a step apart;
//                 16-19 dq to memory, 20 TMA, 21 products.
// Bound.  A pair of 128 x 128 tiles with head_dim 64 costs 1280 cycles of products, 768 of exponentials (1024 without the quarter
// that is taken off the special function unit) and, for its 32 KB of dq at the 16 bytes a cycle and SM that the L2 was measured to add
// in fp32, about 2050; the chain between them makes it about 3600.  With 128, dq has no columns of its own and dp of the next
// pair waits until it has been read.
//   measured      8 x 1024 tokens, 25 heads of 64, causal: 188 us (357 TFLOP/s), of which rows and dq about 40; 8192 tokens, 16
//                 heads of 128 on 4, causal: 1.05 to 1.12 ms (615 to 655 TFLOP/s); 8192 x 8192, 16 heads of 64: 1.14 to 1.17 ms
//                 (585 to 602 TFLOP/s).
#include <math.h>

#include "attention.cuh"

namespace dblp {

constexpr int kGradThreads = 704;
constexpr uint32_t kPairWarps = 16, kDqWarp = 16, kTmaWarp = 20, kMmaWarp = 21;

struct GradArgs {
    TileSource q, k, v, go;
    Heads dk, dv;
    const float* rows;         // [B][Hq][tiles][2][128]: -lse log2(e), then -D
    float* dq;                 // [R][B][Hq][tiles][4][DP / 4][32][4]: query 32 a + l, columns 4 c .. 4 c + 3 at [a][c][l]
    AttnShape s;
    float scale, scale_log2;
    float* dkv;                // [G][2][B][Hkv][k_tiles * 128][DP]: dv, dk of one head group; null when G = 1
    uint32_t q_tiles, k_tiles, shares, groups, group_heads;
    unsigned long long* timeouts;
};

// Key tile number n of share r: to and fro, so that under a causal mask the shares get like amounts of work.
__device__ __forceinline__ uint32_t share_tile(uint32_t r, uint32_t n, uint32_t shares)
{
    return n * shares + (n & 1 ? shares - 1 - r : r);
}
// First query tile that sees key tile j, and the number of query tiles that see any key.
__device__ __forceinline__ uint32_t first_query_tile(uint32_t j, uint32_t lq, uint32_t lk, uint32_t causal)
{
    if (!causal) return 0;
    const int32_t i = (int32_t)(j * 128 + lq) - (int32_t)lk;            // first query that sees key 128 j
    return i > 0 ? (uint32_t)i / 128 : 0;
}

// ---- rows ------------------------------------------------------------------------------------------------------------
// A block takes one tile of 128 rows, a warp 16 of them: eight lanes a row, 16 bytes a load, four rows a thread with their loads
// in front (200 heads of 1024 x 64, caches cold: 7 % less time than one row a thread).
template <typename T>
__global__ void __launch_bounds__(256)
k_grad_rows(Heads o, Heads go, const float* __restrict__ lse, float* __restrict__ rows, AttnShape s, uint32_t q_tiles)
{
    constexpr int R = 4;
    after_start();
    const uint32_t lane = threadIdx.x & 31, h = blockIdx.y, b = blockIdx.z, lq = length_of(s.q_lens, b, s.Sq), lk = length_of(s.k_lens, b, s.Sk);
    const uint32_t in_tile = (threadIdx.x >> 5) * (4 * R) + (lane >> 3), i0 = blockIdx.x * 128 + in_tile;
    const T* po = (const T*)o.p + (int64_t)b * o.sb + (int64_t)i0 * o.st + (int64_t)h * o.sh;
    const T* pg = (const T*)go.p + (int64_t)b * go.sb + (int64_t)i0 * go.st + (int64_t)h * go.sh;
    bool live[R];
    float d[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        live[r] = keys_of(i0 + 4 * r, lq, lk, s.causal) > 0;
        d[r] = 0.0f;
    }
    for (uint32_t c = (lane & 7) * 8; c < s.D; c += 64) {
        Vec8<T> vo[R], vg[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (live[r]) {
                vo[r].load(po + (int64_t)(4 * r) * o.st + c);
                vg[r].load(pg + (int64_t)(4 * r) * go.st + c);
            }
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (live[r]) {
                float x[8], y[8];
                vo[r].get(x);
                vg[r].get(y);
#pragma unroll
                for (int t = 0; t < 8; ++t) d[r] += x[t] * y[t];
            }
    }
    float* dst = rows + (((uint64_t)b * s.Hq + h) * q_tiles + blockIdx.x) * 256 + in_tile;
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int t = 4; t; t >>= 1) d[r] += __shfl_xor_sync(0xFFFFFFFFu, d[r], t);
        if ((lane & 7) == 0) {
            // rows that see nothing, or nothing but scores of -infinity: 2^(s - infinity) = 0
            const float l = live[r] ? lse[((uint64_t)b * s.Hq + h) * s.Sq + i0 + 4 * r] : -INFINITY;
            dst[4 * r] = l == -INFINITY ? l : l * -1.4426950408889634f;
            dst[128 + 4 * r] = l == -INFINITY ? 0.0f : -d[r];
        }
    }
}

// ---- main ------------------------------------------------------------------------------------------------------------
template <int DP> struct GradSmem {
    static constexpr int NS = DP / 64, TILE = NS * (int)kBlockBytes;
    // stages of q (with its row values), of dout, of ds; dq leaves in pieces of 32 queries x 16 columns in fp32, CH
    // at a time for each of its warps.  (With three stages of q the products waited for it in every pair.)
    static constexpr int NQ = DP == 64 ? 4 : 2, NG = DP == 64 ? 2 : 1, ND = DP == 64 ? 2 : 1;
    static constexpr int K = 0, V = TILE, Q = 2 * TILE, G = Q + NQ * TILE, DS = G + NG * TILE, STAGE = DS + ND * 2 * (int)kBlockBytes;
    static constexpr int CH = DP == 64 ? 2 : 4, ROWS = STAGE + 4 * CH * 2048, BARS = ROWS + NQ * 1024, kBytes = BARS + 320;
};
static_assert(GradSmem<64>::kBytes <= 232448 && GradSmem<128>::kBytes <= 232448, "");

struct GradBars {
    uint64_t kv_full, q_full[4], q_empty[4], g_full[4], g_empty[4], cut_full;
    uint64_t s_full[2], p_ready[2], dp_full[2], ds_ready[2], ds_free[2], dq_full, dq_free, acc_full, acc_free, idle;
    uint32_t tmem_slot, dead;
};
static_assert(sizeof(GradBars) <= 320, "");

template <typename T, int DP>
__global__ void __launch_bounds__(kGradThreads, 1) k_grad(const __grid_constant__ GradArgs a)
{
    using L = GradSmem<DP>;
    constexpr int NS = L::NS, NQ = L::NQ, NG = L::NG, ND = L::ND;
    constexpr int NE = DP == 64 ? 2 : 1;                       // groups that the queries of a pair are split into
    constexpr bool kOwnDq = DP == 64;                          // dq has columns of its own; else it takes those of dp
    extern __shared__ __align__(1024) uint8_t smem[];          // the whole of the block's shared memory, so at an even kilobyte
    GradBars& s = *reinterpret_cast<GradBars*>(smem + L::BARS);

    const uint32_t tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    const uint32_t share = blockIdx.x % a.shares, group = blockIdx.x / a.shares, hk = blockIdx.y, b = blockIdx.z;
    const uint32_t heads = a.group_heads, h0 = hk * a.s.rep + group * heads;        // this block's query heads
    const uint32_t lq = uniform(length_of(a.s.q_lens, b, a.s.Sq)), lk = uniform(length_of(a.s.k_lens, b, a.s.Sk));
    const uint32_t nq = (lq + 127) / 128, nk = lq ? (lk + 127) / 128 : 0;
    // query tiles per head that key tile j meets
    auto meets = [&](uint32_t j) -> uint32_t {
        if (j >= nk) return 0;
        const uint32_t i0 = first_query_tile(j, lq, lk, a.s.causal);
        return i0 < nq ? nq - i0 : 0;
    };

    if (tid == 0) {
        s.dead = 0;
        for (uint64_t* p : {&s.kv_full, &s.cut_full, &s.dq_full, &s.acc_full, &s.idle}) bar_init(p, 1);
        for (int i = 0; i < NQ; ++i) { bar_init(&s.q_full[i], 1); bar_init(&s.q_empty[i], 1); }
        for (int i = 0; i < NG; ++i) { bar_init(&s.g_full[i], 1); bar_init(&s.g_empty[i], 1); }
        for (int i = 0; i < 2; ++i) {
            bar_init(&s.s_full[i], 1);
            bar_init(&s.dp_full[i], 1);
            bar_init(&s.ds_free[i], 1);
            bar_init(&s.p_ready[i], kPairWarps / NE);
            bar_init(&s.ds_ready[i], kPairWarps / NE);
        }
        bar_init(&s.acc_free, kPairWarps);
        bar_init(&s.dq_free, 4);
        fence_bar_init();
    }
    if (warp == kMmaWarp) tmem_alloc<512>(&s.tmem_slot);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(s.tmem_slot), t_s = tmem, t_dp = tmem + 128, t_dv = tmem + 256, t_dk = tmem + 256 + DP;
    const uint32_t t_dq = kOwnDq ? tmem + 384 : t_dp;
    const Guard g{&s.dead, a.timeouts};
    after_start();
    wait_before();                                              // the rows' values; what is above ran beside their kernel

    if (warp == kTmaWarp) {                                       // ---- TMA
        uint32_t n = 0, w = 0, cuts = 0;                        // pairs, key tiles with work, tiles that were cleared
        const uint32_t unseeing = a.s.causal && lq > lk ? lq - lk : 0;          // queries before this one see no key
        bool ok = true;
        // a tile of which only the rows of tokens from .. to - 1 count and the others may hold anything
        auto load_cut = [&](uint8_t* dst, const TileSource& src, uint32_t token, uint32_t head, uint32_t from, uint32_t to) -> bool {
            if (lane == 0) {
                bar_expect(&s.cut_full, L::TILE);
                load_tile<NS>(dst, src, &s.cut_full, token, head, b);
            }
            if (!warp_wait(&s.cut_full, cuts++ & 1, g)) return false;
            if (from > token) clear_rows<NS>(dst, 0, from - token);
            if (to < token + 128) clear_rows<NS>(dst, to - token, 128);
            __syncwarp();
            return true;
        };
        for (uint32_t m = 0; ok; ++m) {
            const uint32_t j = share_tile(share, m, a.shares);
            if (m * a.shares >= a.k_tiles) break;
            const uint32_t per_head = meets(j);
            if (per_head == 0) continue;
            if (w) ok = warp_wait(&s.acc_full, (w - 1) & 1, g);   // products of the tile before are done
            if (!ok) break;
            const bool kcut = j * 128 + 128 > lk && lk < a.s.Sk;
            if (kcut) ok = load_cut(smem + L::K, a.k, j * 128, hk, 0, lk);
            if (!ok) break;
            if (lane == 0) {
                bar_expect(&s.kv_full, kcut ? L::TILE : 2 * L::TILE);
                if (!kcut) load_tile<NS>(smem + L::K, a.k, &s.kv_full, j * 128, hk, b);
                load_tile<NS>(smem + L::V, a.v, &s.kv_full, j * 128, hk, b);
            }
            ++w;
            for (uint32_t t = 0; t < per_head * heads && ok; ++t, ++n) {
                const uint32_t h = h0 + t / per_head, i = nq - per_head + t % per_head;
                const bool cut = (i * 128 + 128 > lq && lq < a.s.Sq) || i * 128 < unseeing;
                const uint32_t sq = n % NQ, sg = n % NG;
                if (n >= NQ) ok = warp_wait(&s.q_empty[sq], (n / NQ - 1) & 1, g);
                if (!ok) break;
                uint8_t *dq_ = smem + L::Q + sq * L::TILE, *dg = smem + L::G + sg * L::TILE;
                if (cut) ok = load_cut(dq_, a.q, i * 128, h, unseeing, lq);
                if (!ok) break;
                if (lane == 0) {
                    bar_expect(&s.q_full[sq], (cut ? 0 : L::TILE) + 1024);
                    if (!cut) load_tile<NS>(dq_, a.q, &s.q_full[sq], i * 128, h, b);
                    bulk_load(smem + L::ROWS + sq * 1024, a.rows + (((uint64_t)b * a.s.Hq + h) * a.q_tiles + i) * 256, 1024, &s.q_full[sq]);
                }
                if (n >= NG) ok = warp_wait(&s.g_empty[sg], (n / NG - 1) & 1, g);
                if (ok && cut) ok = load_cut(dg, a.go, i * 128, h, unseeing, lq);
                if (!ok) { if (lane == 0) bar_drain(&s.q_full[sq], (n / NQ) & 1); break; }
                if (lane == 0) {
                    if (cut) {
                        bar_arrive(&s.g_full[sg]);
                    } else {
                        bar_expect(&s.g_full[sg], L::TILE);
                        load_tile<NS>(dg, a.go, &s.g_full[sg], i * 128, h, b);
                    }
                }
                __syncwarp();
            }
        }
        if (lane == 0) {                                        // every copy lands before the block may end
            if (w) bar_drain(&s.kv_full, (w - 1) & 1);
            if (cuts) bar_drain(&s.cut_full, (cuts - 1) & 1);
            for (uint32_t x = n > NQ ? n - NQ : 0; x < n; ++x) bar_drain(&s.q_full[x % NQ], (x / NQ) & 1);
            for (uint32_t x = n > NG ? n - NG : 0; x < n; ++x) bar_drain(&s.g_full[x % NG], (x / NG) & 1);
        }
    } else if (warp == kMmaWarp) {                              // ---- products
        // head_dim up to 64: each pair is done in two halves of 64 queries by two groups of warps that work half a step apart,
        // one computes p while the other computes ds.  The order below follows them: p of the first half, ds of the second
        // half of the pair before, ds of the first half, p of the second.  With 128 there is no room for that: dq takes the
        // columns of dp, so that dp of the next pair waits for dq in any case, and all warps take the whole pair together (8192
        // tokens, 16 heads on 4, causal: halves took 21 % longer).
        constexpr uint32_t id_kk = mma_desc<T>(128, 128 / NE, false, false);    // s, dp of a group
        constexpr uint32_t id_kv = mma_desc<T>(128, DP, false, true);           // dv, dk: right operand across its rows
        constexpr uint32_t id_dq = mma_desc<T>(128, DP, true, true);            // dq: both across their rows
        const uint32_t base = smem_addr(smem);
        uint32_t n = 0, w = 0;
        bool ok = true;
        // s (left k, right q) or dp (left v, right dout) of group e
        auto half_scores = [&](uint32_t to, uint32_t left, uint32_t right, uint32_t e, uint64_t* done) {
#pragma unroll
            for (int kk = 0; kk < DP / 16; ++kk) {
                const uint32_t off = (kk / 4) * kBlockBytes + (kk % 4) * 32;
                mma_ss(to + e * 64, desc_k(left + off), desc_k(right + e * (kBlockBytes / 2) + off), id_kk, kk > 0);
            }
            mma_commit(done);
        };
        auto q_at = [&](uint32_t x) { return base + L::Q + (x % NQ) * L::TILE; };
        auto g_at = [&](uint32_t x) { return base + L::G + (x % NG) * L::TILE; };
        auto ds_at = [&](uint32_t x) { return base + L::DS + (x % ND) * 2 * kBlockBytes; };
        auto scores = [&](uint32_t x, uint32_t e) { half_scores(t_s, base + L::K, q_at(x), e, &s.s_full[e]); };
        auto dprobs = [&](uint32_t x, uint32_t e) { half_scores(t_dp, base + L::V, g_at(x), e, &s.dp_full[e]); };
        auto add_dv = [&](uint32_t x, uint32_t e, bool acc) {
#pragma unroll
            for (int kk = 0; kk < 8 / NE; ++kk)                 // p of queries 32 g .. 32 g + 31 in columns 32 g .. 32 g + 15
                mma_ts(t_dv, t_s + e * 64 + (kk / 2) * 32 + (kk % 2) * 8, desc_mn(g_at(x) + e * (kBlockBytes / 2) + kk * 2048, kBlockBytes), id_kv,
                       acc || kk > 0);
        };
        auto add_dk = [&](uint32_t x, uint32_t e, bool acc) {
#pragma unroll
            for (int kk = 0; kk < 8 / NE; ++kk)
                mma_ss(t_dk, desc_k(ds_at(x) + (e + kk / 4) * kBlockBytes + kk % 4 * 32), desc_mn(q_at(x) + e * (kBlockBytes / 2) + kk * 2048, kBlockBytes), id_kv,
                       acc || kk > 0);
        };
        // last group of pair x: its ds is there, so dk and dq can be completed; `more`: another pair of this key tile follows
        auto finish = [&](uint32_t x, bool more, bool acc) {
            ok = ok && warp_wait(&s.ds_ready[NE - 1], x & 1, g);
            if (ok && kOwnDq && x) ok = warp_wait(&s.dq_free, (x - 1) & 1, g);
            if (!ok) return;
            tc_fence_after();
            if (kOwnDq && more) dprobs(x + 1, 1);
#pragma unroll
            for (int kk = 0; kk < 8; ++kk)
                mma_ss(t_dq, desc_mn(ds_at(x) + kk * 2048, kBlockBytes), desc_mn(base + L::K + kk * 2048, kBlockBytes), id_dq, kk > 0);
            mma_commit(&s.dq_full);
            add_dk(x, NE - 1, acc);
            mma_commit(&s.q_empty[x % NQ]);
            mma_commit(&s.ds_free[x % ND]);
            if (!kOwnDq && more) {                              // dp of the next pair comes where dq is
                ok = warp_wait(&s.g_full[(x + 1) % NG], ((x + 1) / NG) & 1, g) && warp_wait(&s.dq_free, x & 1, g);
                if (!ok) return;
                tc_fence_after();
                dprobs(x + 1, 0);
            }
        };
        for (uint32_t m = 0; ok && m * a.shares < a.k_tiles; ++m) {
            const uint32_t pairs = meets(share_tile(share, m, a.shares)) * heads;
            if (pairs == 0) continue;
            ok = warp_wait(&s.kv_full, w & 1, g) && warp_wait(&s.q_full[n % NQ], (n / NQ) & 1, g);
            if (!ok) break;
            tc_fence_after();
            for (int e = 0; e < NE; ++e) scores(n, e);
            ok = warp_wait(&s.g_full[n % NG], (n / NG) & 1, g);
            if (ok && !kOwnDq && n) ok = warp_wait(&s.dq_free, (n - 1) & 1, g);
            if (!ok) break;
            tc_fence_after();
            for (int e = 0; e < NE; ++e) dprobs(n, e);
            for (uint32_t t = 0; t < pairs && ok; ++t, ++n) {
                const bool more = t + 1 < pairs;
                ok = warp_wait(&s.p_ready[0], n & 1, g);
                if (ok && t == 0 && w) ok = warp_wait(&s.acc_free, (w - 1) & 1, g);
                if (!ok) break;
                tc_fence_after();
                add_dv(n, 0, t > 0);
                if (NE == 1) mma_commit(&s.g_empty[n % NG]);
                if (more) {
                    ok = warp_wait(&s.q_full[(n + 1) % NQ], ((n + 1) / NQ) & 1, g);
                    if (!ok) break;
                    tc_fence_after();
                    scores(n + 1, 0);                           // over p, which the product before has read by then
                }
                if (NE == 1) {
                    finish(n, more, t > 0);
                } else {
                    if (t > 0) finish(n - 1, true, true);
                    ok = ok && warp_wait(&s.ds_ready[0], n & 1, g);
                    if (ok && more) ok = warp_wait(&s.g_full[(n + 1) % NG], ((n + 1) / NG) & 1, g);
                    if (!ok) break;
                    tc_fence_after();
                    if (more) dprobs(n + 1, 0);
                    add_dk(n, 0, t > 0);
                    ok = warp_wait(&s.p_ready[1], n & 1, g);
                    if (!ok) break;
                    tc_fence_after();
                    add_dv(n, 1, true);
                    mma_commit(&s.g_empty[n % NG]);
                    if (more) scores(n + 1, 1);
                }
            }
            if (NE == 2) finish(n - 1, false, true);
            if (ok) mma_commit(&s.acc_full);
            ++w;
        }
        __syncwarp();
        mma_commit(&s.idle);                                    // products in flight end before the memory is freed, whoever gave up
        bar_drain(&s.idle, 0);
        __syncwarp();
    } else if (warp >= kDqWarp) {                               // ---- dq: tensor memory -> this share's buffer
        // Each warp takes 32 queries.  Pieces go through shared memory and are added by the memory system: adding from
        // registers kept the load/store unit busy and stalled every other warp behind it.
        constexpr int CH = L::CH, PER = DP / 16;
        const uint32_t quarter = warp & 3, lane_base = quarter << 21;
        float4* stage = reinterpret_cast<float4*>(smem + L::STAGE + quarter * CH * 2048);
        uint32_t n = 0;
        bool ok = true;
        for (uint32_t m = 0; ok && m * a.shares < a.k_tiles; ++m) {
            const uint32_t per_head = meets(share_tile(share, m, a.shares)), pairs = per_head * heads;
            for (uint32_t t = 0, i = nq - per_head, h = h0; t < pairs; ++t, ++n) {
                float* dst = a.dq + (((((uint64_t)share * a.s.B + b) * a.s.Hq + h) * a.q_tiles + i) * 4 + quarter) * (32 * DP);
                if (++i == nq) { i = nq - per_head; ++h; }
                ok = warp_wait(&s.dq_full, n & 1, g);
                if (!ok) break;
                tc_fence_after();
                // the additions of the last visit to this query tile are done before those of this one begin: all but those of
                // the pair before are complete, and with one pair a key tile those too
                if (lane == 0) {
                    if (pairs > 1) bulk_wait<PER>();
                    else bulk_wait<0>();
                }
#pragma unroll
                for (int c = 0; c < PER; ++c) {
                    uint32_t x[16];
                    __syncwarp();                               // lane 0 alone waited or sent: together again for the load
                    tmem_ld16(t_dq + lane_base + c * 16, x);
                    if (lane == 0) bulk_wait_read<CH - 1>();    // the piece that was here has left
                    __syncwarp();
                    tmem_wait_ld<16>(x);
                    if (c + 1 == PER) {
                        tc_fence_before();
                        warp_arrive(&s.dq_free);
                    }
                    float4* to = stage + (c % CH) * 128 + lane;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        to[e * 32] = make_float4(__uint_as_float(x[4 * e]), __uint_as_float(x[4 * e + 1]), __uint_as_float(x[4 * e + 2]), __uint_as_float(x[4 * e + 3]));
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        // the share's first key tile is the first to meet every query tile it meets at all
                        if (m == 0) bulk_store(dst + c * 512, stage + (c % CH) * 128, 2048);
                        else bulk_add_f32(dst + c * 512, stage + (c % CH) * 128, 2048);
                        bulk_commit();
                    }
                }
            }
        }
        if (lane == 0) bulk_wait<0>();
    } else {                                                    // ---- p and ds: thread = key (lane of the tile), 32 queries
        const uint32_t grp = warp >> 2, e2 = NE == 2 ? warp >> 3 : 0, lane_base = (warp & 3) << 21, row = (warp & 3) * 32 + lane;
        const uint32_t my_s = t_s + lane_base + grp * 32, my_dp = t_dp + lane_base + grp * 32;
        uint8_t* ds_row = smem + L::DS + (grp >> 1) * kBlockBytes + row * 128;
        const float2 c2 = make_float2(a.scale_log2, a.scale_log2);
        uint32_t n = 0, w = 0;
        bool ok = true;
        for (uint32_t m = 0; ok && m * a.shares < a.k_tiles; ++m) {
            const uint32_t j = share_tile(share, m, a.shares), per_head = meets(j), pairs = per_head * heads;
            if (j >= a.k_tiles) continue;
            const uint32_t key = j * 128 + row;
            for (uint32_t t = 0, i = nq - per_head; t < pairs; ++t, ++n, i = i + 1 < nq ? i + 1 : nq - per_head) {
                // queries [from, 32) of this thread's columns see the key
                int32_t from = key < lk ? 0 : 32;
                if (a.s.causal) from = max(from, (int32_t)(key + lq) - (int32_t)lk - (int32_t)(i * 128 + grp * 32));
                const bool cut = __any_sync(0xFFFFFFFFu, from > 0);
                ok = warp_wait(&s.s_full[e2], n & 1, g) && warp_wait(&s.q_full[n % NQ], (n / NQ) & 1, g);
                if (!ok) break;
                tc_fence_after();
                uint32_t p[32];
                tmem_ld32(my_s, p);
                const float4* l4 = reinterpret_cast<const float4*>(smem + L::ROWS + (n % NQ) * 1024) + grp * 8;
                tmem_wait_ld<32>(p);
#pragma unroll
                for (int part = 0; part < 32; part += 16) {
                    uint32_t w8[8];
#pragma unroll
                    for (int e = part; e < part + 16; e += 4) {
                        const float4 l = l4[e / 4];
                        const float2 u = fma2(pair(p[e], p[e + 1]), c2, make_float2(l.x, l.y)), v = fma2(pair(p[e + 2], p[e + 3]), c2, make_float2(l.z, l.w));
                        float2 y = make_float2(exp2_fast(u.x), exp2_fast(u.y)), z;
                        if (DP == 64 && e % 8 == 4) z = exp2_pair(v);           // a quarter off the special function unit
                        else z = make_float2(exp2_fast(v.x), exp2_fast(v.y));
                        p[e] = __float_as_uint(y.x);
                        p[e + 1] = __float_as_uint(y.y);
                        p[e + 2] = __float_as_uint(z.x);
                        p[e + 3] = __float_as_uint(z.y);
                    }
                    if (cut) {
#pragma unroll
                        for (int e = part; e < part + 16; ++e)
                            if (e < from) p[e] = 0;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) w8[e] = pack2<T>(__uint_as_float(p[part + 2 * e]), __uint_as_float(p[part + 2 * e + 1]));
                    tmem_st8(my_s + part / 2, w8);
                }
                tmem_wait_st();
                tc_fence_before();
                warp_arrive(&s.p_ready[e2]);

                ok = warp_wait(&s.dp_full[e2], n & 1, g);
                if (ok && n >= ND) ok = warp_wait(&s.ds_free[n % ND], (n / ND - 1) & 1, g);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int part = 0; part < 32; part += 16) {     // 16 columns at a time, for the sake of registers
                    uint32_t x[16];
                    tmem_ld16(my_dp + part, x);
                    tmem_wait_ld<16>(x);
#pragma unroll
                    for (int e = 0; e < 16; e += 8) {
                        uint32_t w[4];
#pragma unroll
                        for (int f = 0; f < 8; f += 4) {
                            const int at = part + e + f;
                            const float4 d = l4[32 + at / 4];
                            float2 u = mul2(pair(p[at], p[at + 1]), add2(pair(x[e + f], x[e + f + 1]), make_float2(d.x, d.y)));
                            float2 v = mul2(pair(p[at + 2], p[at + 3]), add2(pair(x[e + f + 2], x[e + f + 3]), make_float2(d.z, d.w)));
                            if (cut) {                          // 0 * (dp of a row that does not count) may be NaN
                                u = make_float2(at < from ? 0.0f : u.x, at + 1 < from ? 0.0f : u.y);
                                v = make_float2(at + 2 < from ? 0.0f : v.x, at + 3 < from ? 0.0f : v.y);
                            }
                            w[f / 2] = pack2<T>(u.x, u.y);
                            w[f / 2 + 1] = pack2<T>(v.x, v.y);
                        }
                        *reinterpret_cast<uint4*>(ds_row + (n % ND) * 2 * kBlockBytes + ((((grp & 1) * 4 + (part + e) / 8) ^ (row & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
                fence_async_smem();
                tc_fence_before();
                warp_arrive(&s.ds_ready[e2]);
            }
            if (!ok) break;
            // this key tile's gradients: two groups dv, two dk, half of the columns each
            const bool is_dk = grp >= 2;
            const Heads& hd = is_dk ? a.dk : a.dv;
            T* dst = (T*)hd.p + (int64_t)b * hd.sb + (int64_t)key * hd.st + (int64_t)hk * hd.sh;
            float* part = a.dkv + ((((uint64_t)(group * 2 + is_dk) * a.s.B + b) * a.s.Hkv + hk) * a.k_tiles * 128 + key) * DP;
            const float f = is_dk ? a.scale : 1.0f;
            const int c0 = (grp & 1) * (DP / 2);
            if (pairs) {
                ok = warp_wait(&s.acc_full, w & 1, g);
                if (!ok) break;
                tc_fence_after();
            }
#pragma unroll
            for (int cc = 0; cc < DP / 2; cc += 16) {
                const int c = c0 + cc;
                uint32_t x[16];
                if (pairs) {
                    __syncwarp();                               // the stores before went by the lane
                    tmem_ld16((is_dk ? t_dk : t_dv) + lane_base + c, x);
                    tmem_wait_ld<16>(x);
                }
#pragma unroll
                for (int e = 0; e < 16; e += 8) {
                    float y[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u) y[u] = pairs ? __uint_as_float(x[e + u]) * f : 0.0f;
                    if (a.dkv) {
                        Vec8<float> o;
                        o.set(y);
                        o.store(part + c + e);
                    } else if (key < a.s.Sk && (uint32_t)(c + e) < a.s.D) {
                        Vec8<T> o;
                        o.set(y);
                        o.store(dst + c + e);
                    }
                }
            }
            if (pairs) {
                tc_fence_before();
                warp_arrive(&s.acc_free);
                ++w;
            }
        }
    }
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_free<512>(tmem);
    }
}

// ---- dq --------------------------------------------------------------------------------------------------------------
// Thread: one query, 32 of its columns at a time (200 heads of 1024 x 64, two shares, caches cold: 12 % less time than 8 columns).  Share r
// has a part of query tile i iff its first key tile, r, meets it.
template <typename T, int DP>
__global__ void __launch_bounds__(256) k_grad_dq(const float4* __restrict__ part, Heads dq, AttnShape s, float scale, uint32_t q_tiles, uint32_t shares)
{
    wait_before();
    const uint32_t i = blockIdx.x, h = blockIdx.y, b = blockIdx.z, row = threadIdx.x & 127, token = i * 128 + row;
    const uint32_t lq = length_of(s.q_lens, b, s.Sq), lk = length_of(s.k_lens, b, s.Sk);
    const uint32_t most = i * 128 < lq ? keys_of(min(lq, i * 128 + 128) - 1, lq, lk, s.causal) : 0, parts = min(shares, (most + 127) / 128);
    if (token >= s.Sq) return;
    T* dst = (T*)dq.p + (int64_t)b * dq.sb + (int64_t)token * dq.st + (int64_t)h * dq.sh;
    const uint64_t stride = (uint64_t)s.B * s.Hq * q_tiles * (DP / 4) * 128;
    const float4* src = part + (((uint64_t)b * s.Hq + h) * q_tiles + i) * (DP / 4) * 128 + row / 32 * (DP / 4) * 32 + row % 32;
    // 32 columns at a time, all loads of a share before their additions
#pragma unroll
    for (int c0 = 0; c0 < DP; c0 += 64) {
        const int first = c0 + (threadIdx.x >> 7) * 32;
        if ((uint32_t)first >= s.D) break;
        float y[32] = {};
        for (uint32_t r = 0; r < parts; ++r) {
            float4 u[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = src[r * stride + (first / 4 + e) * 32];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[4 * e] += u[e].x; y[4 * e + 1] += u[e].y; y[4 * e + 2] += u[e].z; y[4 * e + 3] += u[e].w;
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            Vec8<T> o;
            float z[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) z[t] = y[8 * e + t] * scale;
            o.set(z);
            if ((uint32_t)(first + 8 * e) < s.D) o.store(dst + first + 8 * e);
        }
    }
}

// dk and dv of shared key heads from their head groups, added in order.  Thread: 8 columns of one key; grid.z: batch, dv or dk.
template <typename T, int DP>
__global__ void __launch_bounds__(256) k_grad_dkv(const float* __restrict__ part, Heads dk, Heads dv, AttnShape s, uint32_t k_rows, uint32_t groups)
{
    after_start();
    wait_before();
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, c = at % (DP / 8) * 8, key = at / (DP / 8), hk = blockIdx.y, b = blockIdx.z >> 1, is_dk = blockIdx.z & 1;
    if (key >= s.Sk || c >= s.D) return;
    const uint64_t stride = 2ull * s.B * s.Hkv * k_rows * DP;
    const float* src = part + ((((uint64_t)is_dk * s.B + b) * s.Hkv + hk) * k_rows + key) * DP + c;
    float y[8] = {};
    for (uint32_t g = 0; g < groups; ++g) {
        Vec8<float> v;
        float x[8];
        v.load(src + g * stride);
        v.get(x);
#pragma unroll
        for (int t = 0; t < 8; ++t) y[t] += x[t];
    }
    const Heads& hd = is_dk ? dk : dv;
    Vec8<T> o;
    o.set(y);
    o.store((T*)hd.p + (int64_t)b * hd.sb + (int64_t)key * hd.st + (int64_t)hk * hd.sh + c);
}

// How the work of one (sequence, key head) is cut: into R shares of its key tiles and, where query heads share it, G groups
// of them.  Blocks run one to an SM, so time is about rounds x pairs a block; every share costs a pass over q's size in
// fp32 (written, added to and read again), several groups one over k's and v's.  Microseconds from the measured 2.2 (head_dim
// up to 64) and 3.5 a pair, and about 4 bytes a nanosecond.
struct GradCut {
    uint32_t shares, groups;
};
static GradCut cut_of(const dblp_attention_t* a)
{
    const uint64_t bk = (uint64_t)a->batch * a->kv_heads, kt = (a->k_tokens + 127) / 128, qt = (a->q_tokens + 127) / 128, sms = kSms;
    const uint32_t rep = a->q_heads / a->kv_heads;
    const double dp = a->head_dim <= 64 ? 64 : 128, pair_us = a->head_dim <= 64 ? 2.2 : 3.5, half = a->flags & DBLP_ATTENTION_CAUSAL ? 0.5 : 1.0;
    const double q_us = (double)a->batch * a->q_heads * qt * 128 * dp * 4 / 4e6, k_us = 2.0 * bk * kt * 128 * dp * 4 / 4e6;
    GradCut best{1, 1};
    double least = 1e300;
    for (uint32_t g = 1; g <= rep; ++g) {
        if (rep % g || (g > 1 && a->batch > 32767)) continue;      // (grid limit of the final sum)
        for (uint32_t r = 1; r <= 32 && r <= kt; ++r) {
            const double rounds = (double)((bk * r * g + sms - 1) / sms);
            const double us = rounds * (double)((kt + r - 1) / r) * (1.0 + qt * (rep / g) * half * pair_us) + r * half * 2 * q_us + (g > 1 ? g * k_us : 0.0);
            if (us < least) { least = us; best = {r, g}; }
        }
    }
    return best;
}

struct GradSpaceA {
    static constexpr uint64_t kTooLarge = ~0ull;
    uint64_t rows, dq, dkv, bytes;
    GradCut cut;
    explicit GradSpaceA(const dblp_attention_t* a) : cut{0, 1}
    {
        const uint64_t tiles = (uint64_t)a->batch * a->q_heads * ((a->q_tokens + 127) / 128), dp = a->head_dim <= 64 ? 64 : 128;
        rows = 0;
        dq = tiles * 1024;
        dkv = dq;
        bytes = tiles >= 1ull << 40 ? kTooLarge : dq;           // sizes that no tensor has can pass 64 bits
        if (!a->k_tokens) return;
        cut = cut_of(a);
        dkv = dq + cut.shares * tiles * 128 * dp * 4;
        const uint64_t kv = cut.groups > 1 ? cut.groups * 2ull * a->batch * a->kv_heads * ((a->k_tokens + 127) / 128) : 0;
        if (bytes != kTooLarge) bytes = kv >= 1ull << 40 ? kTooLarge : dkv + kv * 128 * dp * 4;
    }
};

size_t attention_backward_space(const dblp_attention_t* a) { return few_grad_rows(a) ? grad_rows_space(a) : GradSpaceA(a).bytes; }

template <typename T, int DP>
static int launch_backward(const GradArgs& r, Heads o, Heads go, const float* lse, Heads dq, cudaStream_t s)
{
    const AttnShape& sh = r.s;
    if (sh.Sq) {
        k_grad_rows<T><<<dim3(r.q_tiles, sh.Hq, sh.B), 256, 0, s>>>(o, go, lse, (float*)r.rows, sh, r.q_tiles);
        DBLP_LAUNCHED();
    }
    if (sh.Sk) {
        const cudaError_t e = allow_shared<k_grad<T, DP>>(GradSmem<DP>::kBytes);
        DBLP_CUDA(e);
        const dim3 grid(r.shares * r.groups, sh.Hkv, sh.B);
        if (sh.Sq) {
            DBLP_NEXT(launch_next(k_grad<T, DP>, grid, kGradThreads, GradSmem<DP>::kBytes, s, r));
        } else {                                                // the call's first kernel: it reads the lengths before it waits
            k_grad<T, DP><<<grid, kGradThreads, GradSmem<DP>::kBytes, s>>>(r);
            DBLP_LAUNCHED();
        }
        if (r.dkv)
            DBLP_NEXT(launch_next(k_grad_dkv<T, DP>, dim3((sh.Sk * (DP / 8) + 255) / 256, sh.Hkv, sh.B * 2), 256, 0, s, r.dkv, r.dk, r.dv, sh,
                                  r.k_tiles * 128, r.groups));
    }
    if (sh.Sq)
        DBLP_NEXT(launch_next(k_grad_dq<T, DP>, dim3(r.q_tiles, sh.Hq, sh.B), 256, 0, s, (const float4*)r.dq, dq, sh, r.scale, r.q_tiles, r.shares));
    return DBLP_OK;
}

int attention_backward(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                       const dblp_heads_t* out, const dblp_heads_t* dout, const float* lse, const dblp_heads_t* dq,
                       const dblp_heads_t* dk, const dblp_heads_t* dv, void* ws, cudaStream_t s)
{
    if (few_grad_rows(a)) return attention_grad_rows(a, q, k, v, out, dout, lse, dq, dk, dv, ws, s);
    GradArgs r{};
    int rc = DBLP_OK;
    if (a->q_tokens) rc = make_source(&r.q, a, q, a->q_tokens, a->q_heads);
    if (rc == DBLP_OK && a->q_tokens) rc = make_source(&r.go, a, dout, a->q_tokens, a->q_heads);
    if (rc == DBLP_OK && a->k_tokens) rc = make_source(&r.k, a, k, a->k_tokens, a->kv_heads);
    if (rc == DBLP_OK && a->k_tokens) rc = make_source(&r.v, a, v, a->k_tokens, a->kv_heads);
    if (rc != DBLP_OK) return rc;
    const GradSpaceA sp(a);
    r.dk = heads(dk);
    r.dv = heads(dv);
    r.rows = (const float*)((uint8_t*)ws + sp.rows);
    r.dq = (float*)((uint8_t*)ws + sp.dq);
    r.s = shape_of(a);
    r.scale = a->scale;
    r.scale_log2 = (float)(a->scale * 1.4426950408889634);
    r.q_tiles = (a->q_tokens + 127) / 128;
    r.k_tiles = (a->k_tokens + 127) / 128;
    r.shares = sp.cut.shares;
    r.groups = sp.cut.groups;
    r.group_heads = r.s.rep / r.groups;
    r.dkv = r.groups > 1 ? (float*)((uint8_t*)ws + sp.dkv) : nullptr;
    r.timeouts = timeout_counter();
    DBLP_REQUIRE(r.timeouts, DBLP_ECUDA, "attention_grad: device setup failed: %s", cudaGetErrorString(cudaGetLastError()));
    const Heads o = heads(out), go = heads(dout), hq = heads(dq);
    if (a->dtype == DBLP_BF16)
        return a->head_dim <= 64 ? launch_backward<__nv_bfloat16, 64>(r, o, go, lse, hq, s) : launch_backward<__nv_bfloat16, 128>(r, o, go, lse, hq, s);
    return a->head_dim <= 64 ? launch_backward<__half, 64>(r, o, go, lse, hq, s) : launch_backward<__half, 128>(r, o, go, lse, hq, s);
}

}  // namespace dblp
