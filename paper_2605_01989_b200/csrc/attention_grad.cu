// dblp_attention_grad, one warp a row: the plain arrangement, fp32 throughout.
#include <math.h>

#include "attention.cuh"

namespace dblp {

constexpr int kAttnWarps = 8;
constexpr int kPerLane = 4;                 // head_dim <= 128

struct AttnArgs {
    Heads q, k, v, o, go, dq, dk, dv;
    float *lse, *delta;
    uint32_t B, Sq, Sk, Hq, Hkv, D, causal;
    float scale;
    const int32_t *q_lens, *k_lens;
};

template <typename T>
__device__ __forceinline__ const T* row_of(const Heads& h, uint32_t b, uint32_t t, uint32_t head)
{
    return (const T*)h.p + (int64_t)b * h.sb + (int64_t)t * h.st + (int64_t)head * h.sh;
}

template <typename T>
__device__ __forceinline__ void load_row(const T* p, uint32_t D, uint32_t lane, float* x)
{
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) x[i] = lane + 32 * i < D ? to_f32(p[lane + 32 * i]) : 0.0f;
}

template <typename T>
__device__ __forceinline__ void store_row(const Heads& h, uint32_t b, uint32_t t, uint32_t head, uint32_t D, uint32_t lane, const float* x)
{
    T* p = const_cast<T*>(row_of<T>(h, b, t, head));
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
        if (lane + 32 * i < D) p[lane + 32 * i] = from_f32<T>(x[i]);
}

__device__ __forceinline__ float dot_rows(const float* a, const float* b)
{
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) s += a[i] * b[i];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    return s;
}

template <typename T>
__global__ void __launch_bounds__(kAttnWarps * 32) k_attention_dq(AttnArgs a)
{
    const uint32_t lane = threadIdx.x & 31, i = blockIdx.x * kAttnWarps + (threadIdx.x >> 5), h = blockIdx.y, b = blockIdx.z;
    if (i >= a.Sq) return;
    const uint32_t hk = h / (a.Hq / a.Hkv), n = keys_of(i, length_of(a.q_lens, b, a.Sq), length_of(a.k_lens, b, a.Sk), a.causal);
    const uint64_t at = ((uint64_t)b * a.Hq + h) * a.Sq + i;
    float q[kPerLane], x[kPerLane], g[kPerLane], dq[kPerLane] = {};
    load_row(row_of<T>(a.q, b, i, h), a.D, lane, q);
    load_row(row_of<T>(a.go, b, i, h), a.D, lane, g);
    load_row(row_of<T>(a.o, b, i, h), a.D, lane, x);
    const float delta = dot_rows(g, x), lse = a.lse[at];
    if (lane == 0) a.delta[at] = delta;
    for (uint32_t j = 0; j < n; ++j) {
        load_row(row_of<T>(a.v, b, j, hk), a.D, lane, x);
        const float dp = dot_rows(g, x);
        load_row(row_of<T>(a.k, b, j, hk), a.D, lane, x);
        const float ds = expf(dot_rows(q, x) * a.scale - lse) * (dp - delta);
#pragma unroll
        for (int t = 0; t < kPerLane; ++t) dq[t] += ds * x[t];
    }
#pragma unroll
    for (int t = 0; t < kPerLane; ++t) dq[t] *= a.scale;
    store_row<T>(a.dq, b, i, h, a.D, lane, dq);
}

template <typename T>
__global__ void __launch_bounds__(kAttnWarps * 32) k_attention_dkv(AttnArgs a)
{
    const uint32_t lane = threadIdx.x & 31, j = blockIdx.x * kAttnWarps + (threadIdx.x >> 5), hk = blockIdx.y, b = blockIdx.z;
    if (j >= a.Sk) return;
    const uint32_t rep = a.Hq / a.Hkv, lq = length_of(a.q_lens, b, a.Sq), lk = length_of(a.k_lens, b, a.Sk);
    float k[kPerLane], v[kPerLane], x[kPerLane], g[kPerLane], dk[kPerLane] = {}, dv[kPerLane] = {};
    if (j < lk) {
        load_row(row_of<T>(a.k, b, j, hk), a.D, lane, k);
        load_row(row_of<T>(a.v, b, j, hk), a.D, lane, v);
        const int64_t first = a.causal ? max((int64_t)0, (int64_t)j + lq - lk) : 0;
        for (uint32_t h = hk * rep; h < hk * rep + rep; ++h)
            for (uint32_t i = (uint32_t)first; i < lq; ++i) {
                const uint64_t at = ((uint64_t)b * a.Hq + h) * a.Sq + i;
                load_row(row_of<T>(a.q, b, i, h), a.D, lane, x);
                load_row(row_of<T>(a.go, b, i, h), a.D, lane, g);
                const float p = expf(dot_rows(x, k) * a.scale - a.lse[at]), ds = p * (dot_rows(g, v) - a.delta[at]) * a.scale;
#pragma unroll
                for (int t = 0; t < kPerLane; ++t) { dv[t] += p * g[t]; dk[t] += ds * x[t]; }
            }
    }
    store_row<T>(a.dk, b, j, hk, a.D, lane, dk);
    store_row<T>(a.dv, b, j, hk, a.D, lane, dv);
}

size_t attention_backward_space(const dblp_attention_t* a) { return (size_t)a->batch * a->q_heads * a->q_tokens * 4; }

int attention_backward(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                       const dblp_heads_t* out, const dblp_heads_t* dout, const float* lse, const dblp_heads_t* dq,
                       const dblp_heads_t* dk, const dblp_heads_t* dv, void* ws, cudaStream_t s)
{
    AttnArgs r{};
    r.B = a->batch; r.Sq = a->q_tokens; r.Sk = a->k_tokens; r.Hq = a->q_heads; r.Hkv = a->kv_heads; r.D = a->head_dim;
    r.causal = a->flags & DBLP_ATTENTION_CAUSAL; r.scale = a->scale; r.q_lens = a->q_lens; r.k_lens = a->k_lens;
    r.q = heads(q); r.k = heads(k); r.v = heads(v); r.o = heads(out); r.go = heads(dout);
    r.dq = heads(dq); r.dk = heads(dk); r.dv = heads(dv); r.lse = const_cast<float*>(lse);
    r.delta = (float*)ws;
    const dim3 gq((a->q_tokens + kAttnWarps - 1) / kAttnWarps, a->q_heads, a->batch), gk((a->k_tokens + kAttnWarps - 1) / kAttnWarps, a->kv_heads, a->batch);
    const bool bf = a->dtype == DBLP_BF16;
    if (a->q_tokens) {
        if (bf) k_attention_dq<__nv_bfloat16><<<gq, kAttnWarps * 32, 0, s>>>(r);
        else k_attention_dq<__half><<<gq, kAttnWarps * 32, 0, s>>>(r);
        DBLP_LAUNCHED();
    }
    if (a->k_tokens) {
        if (bf) k_attention_dkv<__nv_bfloat16><<<gk, kAttnWarps * 32, 0, s>>>(r);
        else k_attention_dkv<__half><<<gk, kAttnWarps * 32, 0, s>>>(r);
        DBLP_LAUNCHED();
    }
    return DBLP_OK;
}

}  // namespace dblp
