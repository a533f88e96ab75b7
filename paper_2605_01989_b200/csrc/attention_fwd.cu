// dblp_attention on the tensor cores.
//
// One block takes 128 queries of one head and walks over its keys in tiles of 128: s = q k^T into tensor memory, one thread
// a row for the softmax, p back into tensor memory as the left operand of out += p v.  The running maximum and sum of a row
// stay in its thread's registers, so nothing of size queries x keys exists.
//   scores     x = scale * log2(e) * s, p = 2^(x - m), m any value near the row's maximum so far: out and the sum use the
//              same m, so it cancels.  m moves only when the maximum has grown by more than 2^8, and only then is the
//              accumulator rescaled; p stays below 2^8, exact enough in 16 bits and far from overflow.
//   warps      0-3 softmax and epilogue, 4 TMA, 5 products.  Two blocks share an SM (96 KB of shared memory and 256 columns
//              of tensor memory each), so that one's products run beside the other's exponentials and a block's start and
//              end are hidden.
//   memory     k and v tiles pass through one ring, in the order in which the products use them.
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
    unsigned long long* timeouts;
};

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
// that is the type of the product with v.
template <typename T>
__device__ __forceinline__ void probabilities(const uint32_t* x, float2 c2, float2 mc2, float2& sum, uint32_t dst)
{
    uint32_t p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float2 y = fma2(make_float2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), c2, mc2);
        y.x = exp2_fast(y.x);
        y.y = exp2_fast(y.y);
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
    __shared__ uint64_t q_full, cut_full, full[STAGES], empty[STAGES], s_full, p_ready, idle;
    __shared__ uint32_t tmem_slot, dead;
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* sq = smem;
    uint8_t* ring = smem + L::TILE;

    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // a causal head's last queries see the most keys: start with them
    const uint32_t qt = a.s.causal ? gridDim.x - 1 - blockIdx.x : blockIdx.x, h = blockIdx.y, b = blockIdx.z, hk = h / a.s.rep;
    const uint32_t q0 = qt * 128, lq = length_of(a.s.q_lens, b, a.s.Sq), lk = length_of(a.s.k_lens, b, a.s.Sk);
    const uint32_t most = q0 < lq ? keys_of(min(lq, q0 + 128) - 1, lq, lk, a.s.causal) : 0;      // of the tile's last query
    const uint32_t nk = (most + 127) / 128;

    if (nk == 0) {                                              // nothing to see: zeros
        if (tid < 128 && q0 + tid < a.s.Sq) {
            T* o = (T*)a.o.p + (int64_t)b * a.o.sb + (int64_t)(q0 + tid) * a.o.st + (int64_t)h * a.o.sh;
            for (uint32_t c = 0; c < a.s.D; c += 8) *reinterpret_cast<uint4*>(o + c) = make_uint4(0, 0, 0, 0);
            if (a.lse) a.lse[((uint64_t)b * a.s.Hq + h) * a.s.Sq + q0 + tid] = -INFINITY;
        }
        return;
    }

    if (tid == 0) {
        dead = 0;
        bar_init(&q_full, 1);
        bar_init(&cut_full, 1);
        bar_init(&idle, 1);
        for (int i = 0; i < STAGES; ++i) { bar_init(&full[i], 1); bar_init(&empty[i], 1); }
        bar_init(&s_full, 1);
        bar_init(&p_ready, 4);
        fence_bar_init();
    }
    if (warp == 5) tmem_alloc<256>(&tmem_slot);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, t_s = tmem, t_o = tmem + 128;
    const Guard g{&dead, a.timeouts};

    if (warp == 4) {                                            // ---- TMA: k(0), v(0), k(1), ...
        if (lane == 0) {
            bar_expect(&q_full, L::TILE);
            load_tile<NS>(sq, a.q, &q_full, q0, h, b);
        }
        const uint32_t tail = lk & 127;                         // rows of the last tile that count, if not all
        uint32_t issued = 0;
        bool ok = true;
        for (uint32_t n = 0; n < 2 * nk && ok; ++n) {
            const uint32_t st = n % STAGES, use = n / STAGES, j = n >> 1;
            if (use) ok = warp_wait(&empty[st], (use - 1) & 1, g);
            if (!ok) break;
            const bool is_v = n & 1, cut = is_v && j * 128 + 128 > lk && lk < a.s.Sk;
            uint8_t* dst = ring + st * L::TILE;
            if (!cut) {
                if (lane == 0) {
                    bar_expect(&full[st], L::TILE);
                    load_tile<NS>(dst, is_v ? a.v : a.k, &full[st], j * 128, hk, b);
                }
                issued = n + 1;
            } else {                                            // a v tile whose last rows do not count: clear them first
                if (lane == 0) {
                    bar_expect(&cut_full, L::TILE);
                    load_tile<NS>(dst, a.v, &cut_full, j * 128, hk, b);
                }
                bar_drain(&cut_full, 0);                        // one such tile a block, the last
                __syncwarp();
                clear_rows<NS>(dst, tail);
                __syncwarp();
                if (lane == 0) bar_arrive(&full[st]);
                issued = n + 1;
            }
            __syncwarp();
        }
        if (lane == 0) {                                        // every copy lands before the block may end
            bar_drain(&q_full, 0);
            for (uint32_t n = issued > (uint32_t)STAGES ? issued - STAGES : 0; n < issued; ++n) bar_drain(&full[n % STAGES], (n / STAGES) & 1);
        }
    } else if (warp == 5) {                                     // ---- products
        {
            const uint32_t leader = elect_leader();
            constexpr uint32_t id_s = mma_desc<T>(128, 128, false, false), id_o = mma_desc<T>(128, DP, false, true);
            const uint32_t qa = smem_addr(sq), ra = smem_addr(ring);
            bool ok = warp_wait(&q_full, 0, g);
            auto scores = [&](uint32_t j) {
                const uint32_t n = 2 * j, st = n % STAGES;
                ok = ok && warp_wait(&full[st], (n / STAGES) & 1, g);
                if (!ok) return;
                tc_fence_after();
#pragma unroll
                for (int kk = 0; kk < DP / 16; ++kk) {
                    const uint32_t off = (kk / 4) * kBlockBytes + (kk % 4) * 32;
                    mma_ss(leader, t_s, desc_k(qa + off), desc_k(ra + st * L::TILE + off), id_s, kk > 0);
                }
                mma_commit(leader, &empty[st]);
                mma_commit(leader, &s_full);
            };
            scores(0);
            for (uint32_t j = 0; j < nk && ok; ++j) {
                const uint32_t n = 2 * j + 1, st = n % STAGES;
                ok = warp_wait(&p_ready, j & 1, g) && warp_wait(&full[st], (n / STAGES) & 1, g);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                    mma_ts(leader, t_o, t_s + 64 + kk * 8, desc_mn(ra + st * L::TILE + kk * 2048, kBlockBytes), id_o, j > 0 || kk > 0);
                mma_commit(leader, &empty[st]);
                if (j + 1 < nk) scores(j + 1);                  // overwrites p(j), which the product before has read by then
                else mma_commit(leader, &s_full);
            }
            if (!ok) {                                          // products in flight end before the memory is freed
                mma_commit(leader, &idle);
                bar_drain(&idle, 0);
            }
        }
        __syncwarp();
    } else {                                                    // ---- softmax: one thread a row
        const uint32_t row = q0 + tid, seen = keys_of(row, lq, lk, a.s.causal), lane_base = warp << 21;      // lane 32 * warp
        const float c = a.scale_log2, grow = 8.0f / c;
        float m = -INFINITY, l = 0.0f;
        bool ok = true;
        for (uint32_t j = 0; j < nk; ++j) {
            ok = warp_wait(&s_full, j & 1, g);
            if (!ok) break;
            tc_fence_after();
            // All 128 scores for the maximum; the first 64 are then dropped and read again chunk by chunk, which keeps the
            // thread below 168 registers.  p(j) goes to columns 64 .. 127 of s(j): those are in registers by then.
            const uint32_t left = seen > j * 128 ? seen - j * 128 : 0;
            const bool cut = __any_sync(0xFFFFFFFFu, left < 128);
            uint32_t lo[64], hi[64];
            tmem_ld32(t_s + lane_base, lo);
            tmem_ld32(t_s + lane_base + 32, lo + 32);
            tmem_ld32(t_s + lane_base + 64, hi);
            tmem_ld32(t_s + lane_base + 96, hi + 32);
            tmem_wait_ld<64>(lo);
            tmem_loaded<64>(hi);
            if (cut) {
                hide_from<64>(lo, left);
                hide_from<64>(hi, left > 64 ? left - 64 : 0);
            }
            const float top = fmaxf(largest<64>(lo), largest<64>(hi));
            const bool move = top > m + grow;                   // also from -infinity
            if (__any_sync(0xFFFFFFFFu, move)) {
                const float alpha = move ? exp2_fast((m - top) * c) : 1.0f;                         // m = -infinity: 0
                if (move) m = top;
                l *= alpha;
                if (j > 0) {
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
            }
            const float mc = m == -INFINITY ? 0.0f : -m * c;
            const float2 c2 = make_float2(c, c), mc2 = make_float2(mc, mc);
            float2 sum = make_float2(0.0f, 0.0f);
            uint32_t again[32];
            tmem_ld32(t_s + lane_base, again);
            probabilities<T>(hi, c2, mc2, sum, t_s + lane_base + 96);
            probabilities<T>(hi + 32, c2, mc2, sum, t_s + lane_base + 112);
            tmem_wait_ld<32>(again);
            uint32_t again2[32];
            tmem_ld32(t_s + lane_base + 32, again2);
            if (cut) hide_from<32>(again, left);
            probabilities<T>(again, c2, mc2, sum, t_s + lane_base + 64);
            tmem_wait_ld<32>(again2);
            if (cut) hide_from<32>(again2, left > 32 ? left - 32 : 0);
            probabilities<T>(again2, c2, mc2, sum, t_s + lane_base + 80);
            l += sum.x + sum.y;
            tmem_wait_st();
            tc_fence_before();
            warp_arrive(&p_ready);
        }
        if (ok) ok = warp_wait(&s_full, nk & 1, g);
        if (ok) {
            tc_fence_after();
            const float inv = l > 0.0f ? 1.0f / l : 0.0f;
            T* o = (T*)a.o.p + (int64_t)b * a.o.sb + (int64_t)row * a.o.st + (int64_t)h * a.o.sh;
#pragma unroll
            for (int i = 0; i < DP / 32; ++i) {
                uint32_t x[32];
                tmem_ld32(t_o + lane_base + i * 32, x);
                tmem_wait_ld<32>(x);
#pragma unroll
                for (int t = 0; t < 32; t += 8) {
                    Vec8<T> w;
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = seen ? __uint_as_float(x[t + e]) * inv : 0.0f;
                    w.set(y);
                    if (row < a.s.Sq && (uint32_t)(i * 32 + t) < a.s.D) w.store(o + i * 32 + t);
                }
            }
            if (a.lse && row < a.s.Sq)
                a.lse[((uint64_t)b * a.s.Hq + h) * a.s.Sq + row] = seen ? (m * c + log2f(l)) * 0.693147180559945309f : -INFINITY;
            tc_fence_before();
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
    const dim3 grid((r.s.Sq + 127) / 128, r.s.Hq, r.s.B);
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
    r.timeouts = timeout_counter();
    DBLP_REQUIRE(r.timeouts, DBLP_ECUDA, "attention: device setup failed: %s", cudaGetErrorString(cudaGetLastError()));
    if (a->dtype == DBLP_BF16)
        return a->head_dim <= 64 ? launch_forward<__nv_bfloat16, 64>(r, s) : launch_forward<__nv_bfloat16, 128>(r, s);
    return a->head_dim <= 64 ? launch_forward<__half, 64>(r, s) : launch_forward<__half, 128>(r, s);
}

}  // namespace dblp
