// dblp_attention on the tensor cores.
//
// A work item is 128 queries of one head; a block walks over the item's keys in half tiles of 64: s = q k^T into one of two
// buffers in tensor memory, one thread a row for the softmax, p back over s as the left operand of out += p v.  The products
// of one buffer run while the softmax works on the other.  The running maximum and sum of a row stay in its thread's
// registers, so nothing of size queries x keys exists.
//   scores     x = scale * log2(e) * s, p = 2^(x - m), m any value near the row's maximum so far: out and the sum use the
//              same m, so it cancels.  m moves only when the maximum has grown by more than 2^8, and only then is the
//              accumulator rescaled; p stays below 2^8, exact enough in 16 bits and far from overflow.  x - m is one fused
//              multiply-add with m rounded, off by up to 2^-24 |m| for the whole row alike; from |m| = kFar on, where that would show
//              when m moves and in the end overflow, scores are taken relative to m before the scale, which is exact where
//              it matters (a half tile in which m then moves is read twice; having the case costs others 0 to 1.5 %).
//   warps      0-3 softmax and epilogue, 4 TMA, 5 products.  Two blocks share an SM (96 KB of shared memory and 256 columns
//              of tensor memory each), so that one's products run beside the other's exponentials.  The blocks are persistent:
//              q and the first k and v of the next item are loaded, and its first scores computed, while the last item's
//              softmax and output are still under way.
//   memory     k and v tiles pass through one ring, in the order in which the products use them.
//   bound      with head_dim 64 no unit: special function unit 41 % busy, issue 49 %, tensor pipe 26 % (8 x 1024 tokens, 25 heads,
//              causal).  128 x 128 scores cost 1024 cycles of the special function unit, 768 with a quarter taken off it, and 512
//              of the tensor cores; what takes longer is the one softmax warp group a block, which waits, loads, reduces,
//              exponentiates, stores and writes the output in turn.  With 128 columns both units are half busy.
//   measured   8 x 1024 tokens, 25 heads of 64, causal: 58 us (461 TFLOP/s of what is not masked); 8192 x 8192, 16 heads of 64:
//              375 to 386 us (712 to 733 TFLOP/s); 8192 tokens, 16 heads on 4 of 128, causal: 269 to 298 us (920 to 1020 TFLOP/s, by
//              the clock that power allows).  When half tiles in two buffers replaced whole tiles in one, the first took 12 % less.
#include <math.h>

#include "attention.cuh"

namespace dblp {

constexpr int kFwdThreads = 192;

struct FwdArgs {
    TileSource q, k, v;
    Heads o;
    float* lse;
    AttnShape s;
    float scale_log2;
    uint32_t q_tiles, items, heads_together;
    unsigned long long* timeouts;
};

// Items in the order in which they are handed out: heads in groups whose k and v stay in L2
// together, within a group by query tile; under a causal mask the last tiles, which see the most keys,
// first.  Block x takes them to and fro, x, 2 grid - 1 - x, 2 grid + x, ...: like amounts of work for all.
struct Item {
    uint32_t qt, h, b;
};
__device__ __forceinline__ uint32_t item_number(uint32_t round) { return round * gridDim.x + (round & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x); }
__device__ __forceinline__ Item item_of(const FwdArgs& a, uint32_t x)
{
    const uint32_t heads = a.s.Hq * a.s.B, per = a.heads_together * a.q_tiles, g = x / per, first = g * a.heads_together;
    const uint32_t n = min(a.heads_together, heads - first), y = x - g * per, t = y / n, hb = first + y - t * n;
    return {a.s.causal ? a.q_tiles - 1 - t : t, hb % a.s.Hq, hb / a.s.Hq};
}
// Half tiles of 64 keys that a query tile's last query sees.
__device__ __forceinline__ uint32_t key_halves(const FwdArgs& a, uint32_t q0, uint32_t lq, uint32_t lk)
{
    return q0 < lq ? (keys_of(min(lq, q0 + 128) - 1, lq, lk, a.s.causal) + 63) / 64 : 0;
}

template <int DP> struct FwdSmem {
    static constexpr int NS = DP / 64, TILE = NS * (int)kBlockBytes, STAGES = DP == 64 ? 5 : 2;
    static constexpr int kBytes = 1024 + TILE * (1 + STAGES);
};

// Scores from place `left` on become -infinity.
template <int N> __device__ __forceinline__ void hide_from(uint32_t* x, uint32_t left)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        if ((uint32_t)i >= left) x[i] = 0xFF800000u;
}

constexpr float kFar = 4096.0f;

// Scores relative to m, unless that is -infinity.
template <int N> __device__ __forceinline__ void take_from(uint32_t* x, float m)
{
    const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) - base);
}

template <int N> __device__ __forceinline__ float largest(const uint32_t* x)
{
    float m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = __uint_as_float(x[i]);
#pragma unroll
    for (int i = 4; i < N; i += 8)
#pragma unroll
        for (int u = 0; u < 4; ++u)
            m[u] = i + 4 + u < N ? max3(m[u], __uint_as_float(x[i + u]), __uint_as_float(x[i + 4 + u])) : fmaxf(m[u], __uint_as_float(x[i + u]));
    return max3(fmaxf(m[0], m[1]), m[2], m[3]);
}

// 32 scores -> 16 words of probabilities in tensor memory; their fp32 sum is added to `sum`.  Rounded to 16 bits because
// that is the type of the product with v.  With head_dim up to 64 a quarter of them is computed off the special function unit
// (8192 x 8192, 16 heads, measured when it came: none 10 % slower, an eighth 4 %, half 13 %); with 128 that unit has time while the
// products run, and the extra instructions cost 2 % (causal, on 4 key heads).
template <typename T, int DP>
__device__ __forceinline__ void probabilities(const uint32_t* x, float2 c2, float2 mc2, float2& sum, uint32_t dst)
{
    uint32_t p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float2 y = fma2(make_float2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), c2, mc2);
        if (DP == 64 && i % 4 == 3) {
            y = exp2_pair(y);
        } else {
            y.x = exp2_fast(y.x);
            y.y = exp2_fast(y.y);
        }
        sum = add2(sum, y);
        p[i] = pack2<T>(y.x, y.y);
    }
    tmem_st16(dst, p);
}

template <typename T, int DP>
__global__ void __launch_bounds__(kFwdThreads, 2) k_attention(const __grid_constant__ FwdArgs a)
{
    using L = FwdSmem<DP>;
    constexpr int NS = L::NS, STAGES = L::STAGES;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t q_full, q_empty, cut_full, full[STAGES], empty[STAGES], s_full[2], p_ready[2], pv_done, o_full, o_free, idle;
    __shared__ uint32_t tmem_slot, dead;
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* sq = smem;
    uint8_t* ring = smem + L::TILE;
    const uint32_t tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;

    if (tid == 0) {
        dead = 0;
        bar_init(&q_full, 1);
        bar_init(&q_empty, 1);
        bar_init(&o_full, 1);
        bar_init(&o_free, 4);
        bar_init(&cut_full, 1);
        bar_init(&idle, 1);
        for (int i = 0; i < STAGES; ++i) { bar_init(&full[i], 1); bar_init(&empty[i], 1); }
        for (int i = 0; i < 2; ++i) { bar_init(&s_full[i], 1); bar_init(&p_ready[i], 4); }
        bar_init(&pv_done, 1);
        fence_bar_init();
    }
    if (warp == 5) tmem_alloc<256>(&tmem_slot);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(tmem_slot), t_s = tmem, t_o = tmem + 128;
    const Guard g{&dead, a.timeouts};

    if (warp == 4) {                                            // ---- TMA: q, k(0), v(0), k(1), ...
        uint32_t n = 0, w = 0, cuts = 0;                        // tiles through the ring, items with work, tiles that were cleared
        bool ok = true;
        for (uint32_t round = 0, x; (x = item_number(round)) < a.items && ok; ++round) {
            const Item it = item_of(a, x);
            const uint32_t lq = uniform(length_of(a.s.q_lens, it.b, a.s.Sq)), lk = uniform(length_of(a.s.k_lens, it.b, a.s.Sk)), hk = it.h / a.s.rep;
            const uint32_t nk = (key_halves(a, it.qt * 128, lq, lk) + 1) / 2;
            if (nk == 0) continue;
            if (w) ok = warp_wait(&q_empty, (w - 1) & 1, g);
            if (!ok) break;
            if (lane == 0) {
                bar_expect(&q_full, L::TILE);
                load_tile<NS>(sq, a.q, &q_full, it.qt * 128, it.h, it.b);
            }
            ++w;
            for (uint32_t t = 0; t < 2 * nk; ++t, ++n) {
                const uint32_t st = n % STAGES, use = n / STAGES, j = t >> 1;
                if (use) ok = warp_wait(&empty[st], (use - 1) & 1, g);
                if (!ok) break;
                const bool is_v = t & 1, cut = is_v && j * 128 + 128 > lk && lk < a.s.Sk;
                uint8_t* dst = ring + st * L::TILE;
                if (!cut) {
                    if (lane == 0) {
                        bar_expect(&full[st], L::TILE);
                        load_tile<NS>(dst, is_v ? a.v : a.k, &full[st], j * 128, hk, it.b);
                    }
                } else {                                        // a v tile whose last rows do not count: clear them first
                    if (lane == 0) {
                        bar_expect(&cut_full, L::TILE);
                        load_tile<NS>(dst, a.v, &cut_full, j * 128, hk, it.b);
                    }
                    ok = warp_wait(&cut_full, cuts++ & 1, g);
                    if (!ok) break;
                    clear_rows<NS>(dst, lk & 127, 128);
                    __syncwarp();
                    if (lane == 0) bar_arrive(&full[st]);
                }
                __syncwarp();
            }
        }
        if (lane == 0) {                                        // every copy lands before the block may end
            if (w) bar_drain(&q_full, (w - 1) & 1);
            if (cuts) bar_drain(&cut_full, (cuts - 1) & 1);
            for (uint32_t x = n > (uint32_t)STAGES ? n - STAGES : 0; x < n; ++x) bar_drain(&full[x % STAGES], (x / STAGES) & 1);
        }
    } else if (warp == 5) {                                     // ---- products
        constexpr uint32_t id_s = mma_desc<T>(128, 64, false, false), id_o = mma_desc<T>(128, DP, false, true);
        const uint32_t qa = smem_addr(sq), ra = smem_addr(ring);
        uint32_t n = 0, w = 0, count = 0;                       // ring tiles and items before this one, halves in all
        bool ok = true;
        // scores of half tile h of an item of nh: 64 of the k tile's 128 rows, into buffer (count + h) % 2
        auto scores = [&](uint32_t h, uint32_t nh) {
            const uint32_t at = n + (h & ~1u), st = at % STAGES, to = (count + h) & 1;
            ok = ok && warp_wait(&full[st], (at / STAGES) & 1, g);
            if (!ok) return;
            tc_fence_after();
            const uint32_t ka = ra + st * L::TILE + (h & 1) * (kBlockBytes / 2);
#pragma unroll
            for (int kk = 0; kk < DP / 16; ++kk) {
                const uint32_t off = (kk / 4) * kBlockBytes + (kk % 4) * 32;
                mma_ss(t_s + to * 64, desc_k(qa + off), desc_k(ka + off), id_s, kk > 0);
            }
            if ((h & 1) || h + 1 == nh) mma_commit(&empty[st]);
            mma_commit(&s_full[to]);
            if (h + 1 == nh) mma_commit(&q_empty);
        };
        for (uint32_t round = 0, x; (x = item_number(round)) < a.items && ok; ++round) {
            const Item it = item_of(a, x);
            const uint32_t lq = uniform(length_of(a.s.q_lens, it.b, a.s.Sq)), lk = uniform(length_of(a.s.k_lens, it.b, a.s.Sk));
            const uint32_t nh = key_halves(a, it.qt * 128, lq, lk);
            if (nh == 0) continue;
            ok = warp_wait(&q_full, w & 1, g);
            scores(0, nh);
            if (nh > 1) scores(1, nh);
            for (uint32_t h = 0; h < nh && ok; ++h) {
                const uint32_t at = n + (h | 1), st = at % STAGES, from = (count + h) & 1;
                ok = warp_wait(&p_ready[from], ((count + h) >> 1) & 1, g) && warp_wait(&full[st], (at / STAGES) & 1, g);
                if (ok && h == 0 && w) ok = warp_wait(&o_free, (w - 1) & 1, g);
                if (!ok) break;
                tc_fence_after();
                const uint32_t va = ra + st * L::TILE + (h & 1) * (kBlockBytes / 2);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    mma_ts(t_o, t_s + from * 64 + kk * 8, desc_mn(va + kk * 2048, kBlockBytes), id_o, h > 0 || kk > 0);
                if ((h & 1) || h + 1 == nh) mma_commit(&empty[st]);
                mma_commit(&pv_done);
                if (h + 1 == nh) mma_commit(&o_full);
                if (h + 2 < nh) scores(h + 2, nh);              // over p(h), which the product before has read by then
            }
            n += (nh + 1) / 2 * 2;
            count += nh;
            ++w;
        }
        __syncwarp();
        mma_commit(&idle);                                      // products in flight end before the memory is freed, whoever gave up
        bar_drain(&idle, 0);
        __syncwarp();
    } else {                                                    // ---- softmax: one thread a row
        const uint32_t lane_base = warp << 21;                  // lane 32 * warp
        const float c = a.scale_log2, grow = fminf(8.0f / c, 3e38f);
        uint32_t w = 0, count = 0;
        bool ok = true;
        for (uint32_t round = 0, x; (x = item_number(round)) < a.items && ok; ++round) {
        const Item it = item_of(a, x);
        const uint32_t q0 = it.qt * 128, lq = uniform(length_of(a.s.q_lens, it.b, a.s.Sq)), lk = uniform(length_of(a.s.k_lens, it.b, a.s.Sk));
        const uint32_t nh = key_halves(a, q0, lq, lk);
        const uint32_t row = q0 + tid, seen = keys_of(row, lq, lk, a.s.causal);
        // m: the row's reference.  Once far, the same in all lanes, scores are taken relative to it: it then counts as 0 (ref) and
        // nothing is left to subtract (mc).
        float m = -INFINITY, l = 0.0f, ref = -INFINITY, mc = 0.0f;
        bool far = false;
        for (uint32_t h = 0; h < nh;) {
            const uint32_t buf = count & 1, my_s = t_s + lane_base + buf * 64;
            ok = warp_wait(&s_full[buf], (count >> 1) & 1, g);
            if (!ok) break;
            tc_fence_after();
            uint32_t s[64];
            tmem_ld32(my_s, s);
            tmem_ld32(my_s + 32, s + 32);
            tmem_wait_ld<64>(s);
            const uint32_t left = seen > h * 64 ? seen - h * 64 : 0;
            if (__any_sync(0xFFFFFFFFu, left < 64 || far)) {
                hide_from<64>(s, left);
                if (far) take_from<64>(s, m);
            }
            const float top = largest<64>(s);
            const bool move = top > ref + grow;                 // also from -infinity
            if (__any_sync(0xFFFFFFFFu, move)) {
                const float before = m;
                if (move) m = far && m != -INFINITY ? m + top : top;
                const float alpha = move ? exp2_fast((before - m) * c) : 1.0f;                      // before = -infinity: 0
                far = far || __any_sync(0xFFFFFFFFu, m != -INFINITY && fabsf(m * c) > kFar);
                ref = far && m != -INFINITY ? 0.0f : m;
                mc = far || m == -INFINITY ? 0.0f : -m * c;
                l *= alpha;
                if (h > 0) {                                    // the product of the half before still adds to the accumulator
                    ok = warp_wait(&pv_done, (count - 1) & 1, g);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int i = 0; i < DP / 16; ++i) {
                        uint32_t o[16];
                        tmem_ld16(t_o + lane_base + i * 16, o);
                        tmem_wait_ld<16>(o);
#pragma unroll
                        for (int t = 0; t < 16; ++t) o[t] = __float_as_uint(__uint_as_float(o[t]) * alpha);
                        tmem_st16(t_o + lane_base + i * 16, o);
                    }
                }
                if (far) {                                      // this half again, relative to the new m (m only grows, to the largest score
                    tmem_wait_st();                             // at the latest with the third reading)
                    continue;
                }
            }
            const float2 c2 = make_float2(c, c), mc2 = make_float2(mc, mc);
            float2 sum = make_float2(0.0f, 0.0f);
            probabilities<T, DP>(s, c2, mc2, sum, my_s);            // p(h) over s(h), which is in registers by now
            probabilities<T, DP>(s + 32, c2, mc2, sum, my_s + 16);
            l += sum.x + sum.y;
            tmem_wait_st();
            tc_fence_before();
            warp_arrive(&p_ready[buf]);
            ++h;
            ++count;
        }
        if (!ok) break;
        if (nh) {
            ok = warp_wait(&o_full, w & 1, g);
            if (!ok) break;
            tc_fence_after();
            ++w;
        }
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;                  // l = NaN: so is the row
        T* o = (T*)a.o.p + (int64_t)it.b * a.o.sb + (int64_t)row * a.o.st + (int64_t)it.h * a.o.sh;
#pragma unroll
        for (int i = 0; i < DP / 32; ++i) {
            uint32_t y32[32];
            if (nh) {
                __syncwarp();                                   // the stores before went by the lane
                tmem_ld32(t_o + lane_base + i * 32, y32);
                tmem_wait_ld<32>(y32);
                if (i + 1 == DP / 32) {
                    tc_fence_before();
                    warp_arrive(&o_free);
                }
            }
#pragma unroll
            for (int t = 0; t < 32; t += 8) {
                Vec8<T> v;
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = seen ? __uint_as_float(y32[t + e]) * inv : 0.0f;
                v.set(y);
                if (row < a.s.Sq && (uint32_t)(i * 32 + t) < a.s.D) v.store(o + i * 32 + t);
            }
        }
        if (a.lse && row < a.s.Sq)
            a.lse[((uint64_t)it.b * a.s.Hq + it.h) * a.s.Sq + row] = seen ? (m * c + log2f(l)) * 0.693147180559945309f : -INFINITY;
        }
    }
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        tmem_free<256>(tmem);
    }
}

template <typename T, int DP> static int launch_forward(const FwdArgs& r, cudaStream_t s)
{
    const cudaError_t e = allow_shared<k_attention<T, DP>>(FwdSmem<DP>::kBytes);
    DBLP_CUDA(e);
    const unsigned grid = r.items < 2 * kSms ? r.items : 2 * kSms;       // two blocks an SM
    k_attention<T, DP><<<grid, kFwdThreads, FwdSmem<DP>::kBytes, s>>>(r);
    DBLP_LAUNCHED();
    return DBLP_OK;
}

size_t attention_forward_space(const dblp_attention_t* a) { return few_rows(a) ? rows_space(a) : 0; }

int attention_forward(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                      const dblp_heads_t* out, float* lse, void* ws, cudaStream_t s)
{
    if (few_rows(a)) return attention_rows(a, q, k, v, out, lse, ws, s);
    FwdArgs r{};
    int rc = make_source(&r.q, a, q, a->q_tokens, a->q_heads);
    if (rc == DBLP_OK && a->k_tokens) rc = make_source(&r.k, a, k, a->k_tokens, a->kv_heads);
    if (rc == DBLP_OK && a->k_tokens) rc = make_source(&r.v, a, v, a->k_tokens, a->kv_heads);
    if (rc != DBLP_OK) return rc;
    r.o = heads(out);
    r.lse = lse;
    r.s = shape_of(a);
    r.scale_log2 = (float)(a->scale * 1.4426950408889634);
    r.q_tiles = (a->q_tokens + 127) / 128;
    const uint64_t items = (uint64_t)r.q_tiles * a->q_heads * a->batch, kv_bytes = (uint64_t)a->k_tokens * a->head_dim * 4 + 1;
    DBLP_REQUIRE(items < (1ull << 31), DBLP_ECAPACITY, "attention: 2^31 query tiles or more");
    r.items = (uint32_t)items;
    // heads that walk together: their k and v take at most 32 MB of the L2 (query heads that share one count it each)
    const uint64_t heads = (uint64_t)a->q_heads * a->batch, fit = (32ull << 20) / kv_bytes;
    r.heads_together = (uint32_t)(fit < 1 ? 1 : fit < heads ? fit : heads);
    r.timeouts = timeout_counter();
    DBLP_REQUIRE(r.timeouts, DBLP_ECUDA, "attention: device setup failed: %s", cudaGetErrorString(cudaGetLastError()));
    if (a->dtype == DBLP_BF16)
        return a->head_dim <= 64 ? launch_forward<__nv_bfloat16, 64>(r, s) : launch_forward<__nv_bfloat16, 128>(r, s);
    return a->head_dim <= 64 ? launch_forward<__half, 64>(r, s) : launch_forward<__half, 128>(r, s);
}

}  // namespace dblp
