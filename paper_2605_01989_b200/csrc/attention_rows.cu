// dblp_attention and dblp_attention_grad for few queries: generation, one or a few new tokens against a long list of keys.
//
// Each key and value is used for NR = q_tokens x (query heads per key head) <= 8 rows only, so the time is that of reading k
// and v once; tensor-core tiles of 128 queries would be nearly empty and walk the keys one tile after the other.  Here a
// group of LPK = 8 (or 16) lanes holds one key, 8 elements a lane, and serves all NR rows with it; a block's groups take
// the keys in turn, each with its own running maximum and sum per row, several keys in flight.  The keys are cut into splits,
// one block each, so that few heads fill the machine too; partial results are joined in a fixed order, first the lanes',
// then the warps', then (k_attention_join) the splits'.
//
// The gradient goes the same way with up to 4 rows: everything about a key (p, ds, and with them its dk and dv) is known to
// the lanes that hold it, so dk and dv are written once and only dq is joined (k_grad_few_join).
//
// Measured: 8 sequences x 25 heads of 64, 1 query, 1024 keys (52 MB): 16 us, 3.3 TB/s; one wave of blocks whose 8 dependent
// loads are the time.  The tensor-core kernel took 27 us there, and 135 us for 8192 keys, 16 heads on 4 of 128 (here 13).  The gradient
// of 4 sequences, 16 heads on 4 of 128, 1 query, 4096 keys: 32 us, 90 in tiles.
#include <math.h>

#include "attention.cuh"

namespace dblp {

constexpr int kRowsWarps = 4;

struct RowsArgs {
    Heads q, k, v, o;
    float* lse;
    float* part;               // [splits][B][Hkv][NR][DP + 2]: sums of p v, then m (log2 units) and l; null with one split
    AttnShape s;
    float scale_log2;
    uint32_t splits, per_split;
};

// (m, l, acc) <- the softmax sums of both; either may be empty (m = -infinity, l = 0)
template <int N> __device__ __forceinline__ void join_sums(float& m, float& l, float* acc, float m2, float l2, const float* acc2)
{
    const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top, f = exp2_fast(m - base), f2 = exp2_fast(m2 - base);
    l = l * f + l2 * f2;
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = acc[i] * f + acc2[i] * f2;
    m = top;
}

template <typename T>
__device__ __forceinline__ void finish_query(const RowsArgs& a, uint32_t b, uint32_t i, uint32_t h, uint32_t c, const float* acc, float m, float l)
{
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    if (c < a.s.D) {
        float y[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) y[t] = acc[t] * inv;
        Vec8<T> w;
        w.set(y);
        w.store((T*)a.o.p + (int64_t)b * a.o.sb + (int64_t)i * a.o.st + (int64_t)h * a.o.sh + c);
    }
    if (c == 0 && a.lse) a.lse[((uint64_t)b * a.s.Hq + h) * a.s.Sq + i] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.693147180559945309f;  // NaN stays
}

template <typename T, int LPK, int NR>
__global__ void __launch_bounds__(kRowsWarps * 32) k_attention_rows(const __grid_constant__ RowsArgs a)
{
    constexpr int GROUPS = 32 / LPK, STEP = kRowsWarps * GROUPS, DP = LPK * 8;
    constexpr int kRowsAhead = NR <= 4 ? 4 : 2;                 // keys a group takes at a time, with as many more in flight
    __shared__ float s_acc[kRowsWarps][NR][DP + 2];
    after_start();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, in_key = lane % LPK, group = warp * GROUPS + lane / LPK, c = in_key * 8;
    const uint32_t hk = blockIdx.x, split = blockIdx.y, b = blockIdx.z, rows = a.s.Sq * a.s.rep;
    const uint32_t lq = length_of(a.s.q_lens, b, a.s.Sq), lk = length_of(a.s.k_lens, b, a.s.Sk);
    const bool live = c < a.s.D;

    float q[NR][8], acc[NR][8], m[NR], l[NR];
    uint32_t sees[NR], most = 0;
#pragma unroll
    for (int r = 0; r < NR; ++r) {                              // row r: query r / rep of head hk * rep + r % rep
        const uint32_t i = r / a.s.rep, h = hk * a.s.rep + r % a.s.rep;
        sees[r] = (uint32_t)r < rows ? keys_of(i, lq, lk, a.s.causal) : 0;
        most = max(most, sees[r]);
        m[r] = -INFINITY;
        l[r] = 0.0f;
#pragma unroll
        for (int t = 0; t < 8; ++t) q[r][t] = acc[r][t] = 0.0f;
        if (sees[r] && live) {
            Vec8<T> w;
            w.load((const T*)a.q.p + (int64_t)b * a.q.sb + (int64_t)i * a.q.st + (int64_t)h * a.q.sh + c);
            w.get(q[r]);
#pragma unroll
            for (int t = 0; t < 8; ++t) q[r][t] *= a.scale_log2;
        }
    }
    const uint32_t first = split * a.per_split, last = min(most, first + a.per_split);
    const T* kp = (const T*)a.k.p + (int64_t)b * a.k.sb + (int64_t)hk * a.k.sh + c;
    const T* vp = (const T*)a.v.p + (int64_t)b * a.v.sb + (int64_t)hk * a.v.sh + c;
    Vec8<T> vk[kRowsAhead], vv[kRowsAhead], nk[kRowsAhead], nv[kRowsAhead];
    auto load = [&](uint32_t j0, Vec8<T>* kk, Vec8<T>* vals) {
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            const uint32_t j = j0 + u * STEP + group;
            if (j < last && live) {
                kk[u].load(kp + (int64_t)j * a.k.st);
                vals[u].load(vp + (int64_t)j * a.v.st);
            } else {
                kk[u].w = vals[u].w = make_uint4(0, 0, 0, 0);
            }
        }
    };
    load(first, nk, nv);
    for (uint32_t j0 = first; j0 < last; j0 += STEP * kRowsAhead) {             // the same trip count for all lanes
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) { vk[u] = nk[u]; vv[u] = nv[u]; }
        load(j0 + STEP * kRowsAhead, nk, nv);
        float x[NR][kRowsAhead];
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            float y[8];
            vk[u].get(y);
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                float s = q[r][0] * y[0];
#pragma unroll
                for (int t = 1; t < 8; ++t) s = fmaf(q[r][t], y[t], s);
#pragma unroll
                for (int o = LPK / 2; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
                x[r][u] = j0 + u * STEP + group < min(last, sees[r]) ? s : -INFINITY;
            }
        }
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float top = m[r];
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u) top = fmaxf(top, x[r][u]);
            const float base = top == -INFINITY ? 0.0f : top, f = exp2_fast(m[r] - base);
            m[r] = top;
            l[r] *= f;
#pragma unroll
            for (int t = 0; t < 8; ++t) acc[r][t] *= f;
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u) {
                x[r][u] = exp2_fast(x[r][u] - base);
                l[r] += x[r][u];
            }
        }
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            float y[8];
            vv[u].get(y);
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int t = 0; t < 8; ++t) acc[r][t] = fmaf(x[r][u], y[t], acc[r][t]);
        }
    }
    // the warp's groups, then the block's warps in order
#pragma unroll
    for (int r = 0; r < NR; ++r) {
#pragma unroll
        for (int o = LPK; o < 32; o <<= 1) {
            float other[8];
            const float m2 = __shfl_xor_sync(0xFFFFFFFFu, m[r], o), l2 = __shfl_xor_sync(0xFFFFFFFFu, l[r], o);
#pragma unroll
            for (int t = 0; t < 8; ++t) other[t] = __shfl_xor_sync(0xFFFFFFFFu, acc[r][t], o);
            join_sums<8>(m[r], l[r], acc[r], m2, l2, other);
        }
        if (lane < LPK) {
#pragma unroll
            for (int t = 0; t < 8; ++t) s_acc[warp][r][c + t] = acc[r][t];
            if (lane == 0) { s_acc[warp][r][DP] = m[r]; s_acc[warp][r][DP + 1] = l[r]; }
        }
    }
    __syncthreads();
    for (uint32_t w = threadIdx.x; w < rows * LPK; w += kRowsWarps * 32) {
        const uint32_t r = w / LPK, cc = w % LPK * 8;
        float y[8], mm = s_acc[0][r][DP], ll = s_acc[0][r][DP + 1];
#pragma unroll
        for (int t = 0; t < 8; ++t) y[t] = s_acc[0][r][cc + t];
        for (int p = 1; p < kRowsWarps; ++p) join_sums<8>(mm, ll, y, s_acc[p][r][DP], s_acc[p][r][DP + 1], &s_acc[p][r][cc]);
        if (a.part) {
            float* dst = a.part + ((((uint64_t)split * a.s.B + b) * a.s.Hkv + hk) * rows + r) * (DP + 2);
#pragma unroll
            for (int t = 0; t < 8; ++t) dst[cc + t] = y[t];
            if (cc == 0) { dst[DP] = mm; dst[DP + 1] = ll; }
        } else {
            finish_query<T>(a, b, r / a.s.rep, hk * a.s.rep + r % a.s.rep, cc, y, mm, ll);
        }
    }
}

// A block joins one row: its 128 / LPK groups of lanes take contiguous parts of the splits, then the first joins the parts in
// order.
template <typename T, int LPK>
__global__ void __launch_bounds__(128) k_attention_join(const __grid_constant__ RowsArgs a)
{
    constexpr int DP = LPK * 8, GROUPS = 128 / LPK;
    __shared__ float s_acc[GROUPS][DP + 2];
    wait_before();
    const uint32_t rows = a.s.Sq * a.s.rep, row = blockIdx.x, group = threadIdx.x / LPK, c = threadIdx.x % LPK * 8;
    const uint64_t total = (uint64_t)a.s.B * a.s.Hkv * rows;
    const uint32_t per = (a.splits + GROUPS - 1) / GROUPS, lo = min(a.splits, group * per), hi = min(a.splits, lo + per);
    float y[8] = {}, m = -INFINITY, l = 0.0f;
#pragma unroll 4
    for (uint32_t p = lo; p < hi; ++p) {
        const float* src = a.part + (p * total + row) * (DP + 2);
        float z[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) z[t] = src[c + t];
        join_sums<8>(m, l, y, src[DP], src[DP + 1], z);
    }
#pragma unroll
    for (int t = 0; t < 8; ++t) s_acc[group][c + t] = y[t];
    if (c == 0) { s_acc[group][DP] = m; s_acc[group][DP + 1] = l; }
    __syncthreads();
    if (group) return;
    for (uint32_t p = 1; p < GROUPS && p * per < a.splits; ++p) join_sums<8>(m, l, y, s_acc[p][DP], s_acc[p][DP + 1], &s_acc[p][c]);
    const uint32_t r = row % rows, hk = row / rows % a.s.Hkv, b = row / rows / a.s.Hkv;
    finish_query<T>(a, b, r / a.s.rep, hk * a.s.rep + r % a.s.rep, c, y, m, l);
}

// Rows per key head up to 8: the arithmetic of one key (about 10 instructions a warp and row) still hides behind its bytes.
bool few_rows(const dblp_attention_t* a)
{
    return (uint64_t)a->q_tokens * (a->q_heads / a->kv_heads) <= 8 && (uint64_t)a->batch * a->q_heads * a->q_tokens < (1ull << 31);
}

// Splits: enough blocks for about four to an SM, at least 128 keys each.
static uint32_t splits_of(const dblp_attention_t* a)
{
    const uint64_t heads = (uint64_t)a->batch * a->kv_heads, most = (a->k_tokens + 127) / 128, want = kSms * 4 / heads;
    const uint64_t n = want < most ? want : most;
    return n < 1 ? 1 : (uint32_t)n;
}

size_t rows_space(const dblp_attention_t* a)
{
    const uint64_t splits = splits_of(a), dp = a->head_dim <= 64 ? 64 : 128;
    return splits > 1 ? splits * a->batch * a->q_heads * a->q_tokens * (dp + 2) * 4 : 0;
}

// ---- gradient --------------------------------------------------------------------------------------------------------
struct FewArgs {
    Heads q, k, v, o, go, dq, dk, dv;
    const float* lse;
    float* part;               // [splits][B][Hkv][rows][DP]: dq before scaling; null with one split
    AttnShape s;
    float scale, scale_log2;
    uint32_t splits, per_split;
};

template <typename T, int LPK> __device__ __forceinline__ float group_sum(float x)
{
#pragma unroll
    for (int o = LPK / 2; o; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

template <typename T>
__device__ __forceinline__ void store_dq(const FewArgs& a, uint32_t b, uint32_t hk, uint32_t r, uint32_t c, float* y)
{
    if (c >= a.s.D) return;
#pragma unroll
    for (int t = 0; t < 8; ++t) y[t] *= a.scale;
    Vec8<T> w;
    w.set(y);
    w.store((T*)a.dq.p + (int64_t)b * a.dq.sb + (int64_t)(r / a.s.rep) * a.dq.st + (int64_t)(hk * a.s.rep + r % a.s.rep) * a.dq.sh + c);
}

template <typename T, int LPK, int NR>
__global__ void __launch_bounds__(kRowsWarps * 32) k_grad_few(const __grid_constant__ FewArgs a)
{
    constexpr int GROUPS = 32 / LPK, STEP = kRowsWarps * GROUPS, DP = LPK * 8, AHEAD = 2;
    __shared__ float s_acc[kRowsWarps][NR][DP];
    after_start();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = warp * GROUPS + lane / LPK, c = lane % LPK * 8;
    const uint32_t hk = blockIdx.x, split = blockIdx.y, b = blockIdx.z, rows = a.s.Sq * a.s.rep;
    const uint32_t lq = length_of(a.s.q_lens, b, a.s.Sq), lk = length_of(a.s.k_lens, b, a.s.Sk);
    const bool live = c < a.s.D;
    float q[NR][8], g[NR][8], dq[NR][8], lse[NR], delta[NR];
    uint32_t sees[NR], most = 0;
#pragma unroll
    for (int r = 0; r < NR; ++r) {                              // row r: query r / rep of head hk * rep + r % rep
        const uint32_t i = r / a.s.rep, h = hk * a.s.rep + r % a.s.rep;
        sees[r] = (uint32_t)r < rows ? keys_of(i, lq, lk, a.s.causal) : 0;
        lse[r] = 0.0f;
        float d = 0.0f;
#pragma unroll
        for (int t = 0; t < 8; ++t) q[r][t] = g[r][t] = dq[r][t] = 0.0f;
        if (sees[r]) lse[r] = a.lse[((uint64_t)b * a.s.Hq + h) * a.s.Sq + i] * 1.4426950408889634f;
        if (lse[r] == -INFINITY) sees[r] = 0;                   // nothing but scores of -infinity: as a row that sees no key
        most = max(most, sees[r]);
        if (sees[r] && live) {
            Vec8<T> w;
            float o[8];
            w.load((const T*)a.q.p + (int64_t)b * a.q.sb + (int64_t)i * a.q.st + (int64_t)h * a.q.sh + c);
            w.get(q[r]);
            w.load((const T*)a.go.p + (int64_t)b * a.go.sb + (int64_t)i * a.go.st + (int64_t)h * a.go.sh + c);
            w.get(g[r]);
            w.load((const T*)a.o.p + (int64_t)b * a.o.sb + (int64_t)i * a.o.st + (int64_t)h * a.o.sh + c);
            w.get(o);
#pragma unroll
            for (int t = 0; t < 8; ++t) d = fmaf(g[r][t], o[t], d);
        }
        delta[r] = group_sum<T, LPK>(d);
    }
    const uint32_t first = split * a.per_split, last = min(a.s.Sk, first + a.per_split);
    const T* kp = (const T*)a.k.p + (int64_t)b * a.k.sb + (int64_t)hk * a.k.sh + c;
    const T* vp = (const T*)a.v.p + (int64_t)b * a.v.sb + (int64_t)hk * a.v.sh + c;
    T* dkp = (T*)a.dk.p + (int64_t)b * a.dk.sb + (int64_t)hk * a.dk.sh + c;
    T* dvp = (T*)a.dv.p + (int64_t)b * a.dv.sb + (int64_t)hk * a.dv.sh + c;
    Vec8<T> vk[AHEAD], vv[AHEAD], nk[AHEAD], nv[AHEAD];
    auto load = [&](uint32_t j0, Vec8<T>* kk, Vec8<T>* vals) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const uint32_t j = j0 + u * STEP + group;
            if (j < min(last, most) && live) {                  // what no row sees is never read
                kk[u].load(kp + (int64_t)j * a.k.st);
                vals[u].load(vp + (int64_t)j * a.v.st);
            } else {
                kk[u].w = vals[u].w = make_uint4(0, 0, 0, 0);
            }
        }
    };
    load(first, nk, nv);
    for (uint32_t j0 = first; j0 < last; j0 += STEP * AHEAD) {                  // the same trip count for all lanes
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) { vk[u] = nk[u]; vv[u] = nv[u]; }
        load(j0 + STEP * AHEAD, nk, nv);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const uint32_t j = j0 + u * STEP + group;
            float y[8], z[8], dk[8] = {}, dv[8] = {};
            vk[u].get(y);
            vv[u].get(z);
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                float s = 0.0f, dp = 0.0f;
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    s = fmaf(q[r][t], y[t], s);
                    dp = fmaf(g[r][t], z[t], dp);
                }
                s = group_sum<T, LPK>(s);
                dp = group_sum<T, LPK>(dp);
                const bool visible = j < min(last, sees[r]);
                const float p = visible ? exp2_fast(fmaf(s, a.scale_log2, -lse[r])) : 0.0f, ds = visible ? p * (dp - delta[r]) : 0.0f;
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    dv[t] = fmaf(p, g[r][t], dv[t]);
                    dk[t] = fmaf(ds, q[r][t], dk[t]);
                    dq[r][t] = fmaf(ds, y[t], dq[r][t]);
                }
            }
            if (j < last && live) {
                Vec8<T> w;
                w.set(dv);
                w.store(dvp + (int64_t)j * a.dv.st);
#pragma unroll
                for (int t = 0; t < 8; ++t) dk[t] *= a.scale;
                w.set(dk);
                w.store(dkp + (int64_t)j * a.dk.st);
            }
        }
    }
    // the warp's groups, then the block's warps in order
#pragma unroll
    for (int r = 0; r < NR; ++r) {
#pragma unroll
        for (int o = LPK; o < 32; o <<= 1)
#pragma unroll
            for (int t = 0; t < 8; ++t) dq[r][t] += __shfl_xor_sync(0xFFFFFFFFu, dq[r][t], o);
        if (lane < LPK)
#pragma unroll
            for (int t = 0; t < 8; ++t) s_acc[warp][r][c + t] = dq[r][t];
    }
    __syncthreads();
    for (uint32_t w = threadIdx.x; w < rows * LPK; w += kRowsWarps * 32) {
        const uint32_t r = w / LPK, cc = w % LPK * 8;
        float y[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            y[t] = s_acc[0][r][cc + t];
            for (int p = 1; p < kRowsWarps; ++p) y[t] += s_acc[p][r][cc + t];
        }
        if (a.part) {
            float* dst = a.part + ((((uint64_t)split * a.s.B + b) * a.s.Hkv + hk) * rows + r) * DP + cc;
#pragma unroll
            for (int t = 0; t < 8; ++t) dst[t] = y[t];
        } else {
            store_dq<T>(a, b, hk, r, cc, y);
        }
    }
}

// A block joins one row's dq: contiguous parts of the splits, then the parts in order.
template <typename T, int LPK>
__global__ void __launch_bounds__(128) k_grad_few_join(const __grid_constant__ FewArgs a)
{
    constexpr int DP = LPK * 8, GROUPS = 128 / LPK;
    __shared__ float s_acc[GROUPS][DP];
    wait_before();
    const uint32_t rows = a.s.Sq * a.s.rep, row = blockIdx.x, group = threadIdx.x / LPK, c = threadIdx.x % LPK * 8;
    const uint64_t total = (uint64_t)a.s.B * a.s.Hkv * rows;
    const uint32_t per = (a.splits + GROUPS - 1) / GROUPS, lo = min(a.splits, group * per), hi = min(a.splits, lo + per);
    float y[8] = {};
#pragma unroll 4
    for (uint32_t p = lo; p < hi; ++p)
#pragma unroll
        for (int t = 0; t < 8; ++t) y[t] += a.part[(p * total + row) * DP + c + t];
#pragma unroll
    for (int t = 0; t < 8; ++t) s_acc[group][c + t] = y[t];
    __syncthreads();
    if (group) return;
    for (uint32_t p = 1; p < GROUPS && p * per < a.splits; ++p)
#pragma unroll
        for (int t = 0; t < 8; ++t) y[t] += s_acc[p][c + t];
    store_dq<T>(a, row / rows / a.s.Hkv, row / rows % a.s.Hkv, row % rows, c, y);
}

bool few_grad_rows(const dblp_attention_t* a)
{
    return a->q_tokens > 0 && (uint64_t)a->q_tokens * (a->q_heads / a->kv_heads) <= 4 && (uint64_t)a->batch * a->q_heads * a->q_tokens < (1ull << 31);
}

size_t grad_rows_space(const dblp_attention_t* a)
{
    const uint64_t splits = splits_of(a), dp = a->head_dim <= 64 ? 64 : 128;
    return splits > 1 ? splits * a->batch * a->q_heads * a->q_tokens * dp * 4 : 0;
}

template <typename T, int LPK> static int launch_few(const FewArgs& r, cudaStream_t s)
{
    const uint32_t rows = r.s.Sq * r.s.rep;
    const dim3 grid(r.s.Hkv, r.splits, r.s.B);
    if (rows == 1) k_grad_few<T, LPK, 1><<<grid, kRowsWarps * 32, 0, s>>>(r);
    else if (rows == 2) k_grad_few<T, LPK, 2><<<grid, kRowsWarps * 32, 0, s>>>(r);
    else k_grad_few<T, LPK, 4><<<grid, kRowsWarps * 32, 0, s>>>(r);
    DBLP_LAUNCHED();
    if (r.part) DBLP_NEXT(launch_next(k_grad_few_join<T, LPK>, r.s.B * r.s.Hkv * rows, 128, 0, s, r));
    return DBLP_OK;
}

int attention_grad_rows(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                        const dblp_heads_t* out, const dblp_heads_t* dout, const float* lse, const dblp_heads_t* dq, const dblp_heads_t* dk,
                        const dblp_heads_t* dv, void* ws, cudaStream_t s)
{
    FewArgs r{};
    r.q = heads(q); r.k = heads(k); r.v = heads(v); r.o = heads(out); r.go = heads(dout);
    r.dq = heads(dq); r.dk = heads(dk); r.dv = heads(dv);
    r.lse = lse;
    r.s = shape_of(a);
    r.scale = a->scale;
    r.scale_log2 = (float)(a->scale * 1.4426950408889634);
    r.splits = splits_of(a);
    r.per_split = (a->k_tokens + r.splits - 1) / r.splits;
    r.part = r.splits > 1 ? (float*)ws : nullptr;
    if (a->dtype == DBLP_BF16) return a->head_dim <= 64 ? launch_few<__nv_bfloat16, 8>(r, s) : launch_few<__nv_bfloat16, 16>(r, s);
    return a->head_dim <= 64 ? launch_few<__half, 8>(r, s) : launch_few<__half, 16>(r, s);
}

// ---- forward: host ---------------------------------------------------------------------------------------------------
template <typename T, int LPK> static int launch_rows(const RowsArgs& r, cudaStream_t s)
{
    const uint32_t rows = r.s.Sq * r.s.rep;
    const dim3 grid(r.s.Hkv, r.splits, r.s.B);                          // neighbouring heads, whose rows lie side by side, together
    if (rows == 1) k_attention_rows<T, LPK, 1><<<grid, kRowsWarps * 32, 0, s>>>(r);
    else if (rows == 2) k_attention_rows<T, LPK, 2><<<grid, kRowsWarps * 32, 0, s>>>(r);
    else if (rows <= 4) k_attention_rows<T, LPK, 4><<<grid, kRowsWarps * 32, 0, s>>>(r);
    else k_attention_rows<T, LPK, 8><<<grid, kRowsWarps * 32, 0, s>>>(r);
    DBLP_LAUNCHED();
    if (r.part) {
        DBLP_NEXT(launch_next(k_attention_join<T, LPK>, r.s.B * r.s.Hkv * rows, 128, 0, s, r));
    }
    return DBLP_OK;
}

int attention_rows(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v, const dblp_heads_t* out,
                   float* lse, void* ws, cudaStream_t s)
{
    RowsArgs r{};
    r.q = heads(q); r.k = heads(k); r.v = heads(v); r.o = heads(out);
    r.lse = lse;
    r.s = shape_of(a);
    r.scale_log2 = (float)(a->scale * 1.4426950408889634);
    r.splits = splits_of(a);
    r.per_split = (a->k_tokens + r.splits - 1) / r.splits;
    r.part = r.splits > 1 ? (float*)ws : nullptr;
    if (a->dtype == DBLP_BF16) return a->head_dim <= 64 ? launch_rows<__nv_bfloat16, 8>(r, s) : launch_rows<__nv_bfloat16, 16>(r, s);
    return a->head_dim <= 64 ? launch_rows<__half, 8>(r, s) : launch_rows<__half, 16>(r, s);
}

}  // namespace dblp
