// dblp_attention and dblp_attention_grad, one warp a row: the plain arrangement, fp32 throughout.
#include <math.h>

#include "types.cuh"

namespace dblp {

constexpr int kAttnWarps = 8;
constexpr int kPerLane = 4;                 // head_dim <= 128

struct Heads {
    void* p;
    int64_t sb, st, sh;
};

struct AttnArgs {
    Heads q, k, v, o, go, dq, dk, dv;
    float *lse, *delta;
    uint32_t B, Sq, Sk, Hq, Hkv, D, causal;
    float scale;
    const int32_t *q_lens, *k_lens;
};

__device__ __forceinline__ uint32_t length_of(const int32_t* lens, uint32_t b, uint32_t extent)
{
    return lens ? (uint32_t)min(max(lens[b], 0), (int32_t)extent) : extent;
}

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

// keys that query i sees: 0 .. result - 1
__device__ __forceinline__ uint32_t keys_of(uint32_t i, uint32_t lq, uint32_t lk, uint32_t causal)
{
    if (i >= lq) return 0;
    if (!causal) return lk;
    const int64_t e = (int64_t)i + lk - lq + 1;
    return e < 0 ? 0 : (uint32_t)e;
}

template <typename T>
__global__ void __launch_bounds__(kAttnWarps * 32) k_attention(AttnArgs a)
{
    const uint32_t lane = threadIdx.x & 31, i = blockIdx.x * kAttnWarps + (threadIdx.x >> 5), h = blockIdx.y, b = blockIdx.z;
    if (i >= a.Sq) return;
    const uint32_t hk = h / (a.Hq / a.Hkv), n = keys_of(i, length_of(a.q_lens, b, a.Sq), length_of(a.k_lens, b, a.Sk), a.causal);
    float q[kPerLane], x[kPerLane], o[kPerLane] = {}, m = -INFINITY, l = 0.0f;
    load_row(row_of<T>(a.q, b, i, h), a.D, lane, q);
    for (uint32_t j = 0; j < n; ++j) {
        load_row(row_of<T>(a.k, b, j, hk), a.D, lane, x);
        const float s = dot_rows(q, x) * a.scale, mn = fmaxf(m, s), c = expf(m - mn), p = expf(s - mn);
        load_row(row_of<T>(a.v, b, j, hk), a.D, lane, x);
        l = l * c + p;
        m = mn;
#pragma unroll
        for (int t = 0; t < kPerLane; ++t) o[t] = o[t] * c + p * x[t];
    }
#pragma unroll
    for (int t = 0; t < kPerLane; ++t) o[t] = n ? o[t] / l : 0.0f;
    store_row<T>(a.o, b, i, h, a.D, lane, o);
    if (a.lse && lane == 0) a.lse[((uint64_t)b * a.Hq + h) * a.Sq + i] = n ? m + logf(l) : -INFINITY;
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

static Heads heads(const dblp_heads_t* h) { return Heads{h->data, h->batch_stride, h->token_stride, h->head_stride}; }

static int check_shape(const char* who, const dblp_attention_t* a)
{
    DBLP_REQUIRE(a, DBLP_EINVAL, "%s: null argument", who);
    DBLP_REQUIRE(a->dtype == DBLP_BF16 || a->dtype == DBLP_F16, DBLP_EINVAL, "%s: dtype %d (bf16 or f16)", who, a->dtype);
    DBLP_REQUIRE(a->head_dim >= 8 && a->head_dim <= 128 && a->head_dim % 8 == 0, DBLP_EINVAL,
                 "%s: head_dim %u is not a multiple of 8 up to 128", who, a->head_dim);
    DBLP_REQUIRE(a->q_heads > 0 && a->kv_heads > 0 && a->q_heads % a->kv_heads == 0, DBLP_EINVAL,
                 "%s: %u key heads do not divide %u query heads", who, a->kv_heads, a->q_heads);
    DBLP_REQUIRE((a->flags & ~(uint32_t)DBLP_ATTENTION_CAUSAL) == 0, DBLP_EINVAL, "%s: unknown flags %u", who, a->flags);
    DBLP_REQUIRE(a->scale > 0.0f && a->scale < INFINITY, DBLP_EINVAL, "%s: scale %g is not finite and positive", who, a->scale);
    DBLP_REQUIRE(a->batch < 65536 && a->q_heads < 65536 && a->q_tokens < (1u << 30) && a->k_tokens < (1u << 30), DBLP_ECAPACITY,
                 "%s: batch and heads below 65536, tokens below 2^30", who);
    return DBLP_OK;
}

// Data and the strides that are used: multiples of 16 bytes; outputs: no two elements in one place.
static int check_heads(const char* who, const char* name, const dblp_attention_t* a, const dblp_heads_t* h, uint32_t tokens, uint32_t nheads,
                       bool output)
{
    DBLP_REQUIRE(h && h->data, DBLP_EINVAL, "%s: %s is null", who, name);
    const struct { int64_t stride; uint64_t extent; } dim[3] = {{h->batch_stride, a->batch}, {h->token_stride, tokens}, {h->head_stride, nheads}};
    bool aligned = aligned16(h->data);
    for (auto& d : dim) {
        if (d.extent <= 1) continue;
        aligned = aligned && d.stride % 8 == 0;
        DBLP_REQUIRE(d.stride >= 0 && d.stride < (1ll << 39), DBLP_EINVAL, "%s: %s has a stride of %lld", who, name, (long long)d.stride);
    }
    DBLP_REQUIRE(aligned, DBLP_EALIGN, "%s: %s has data or a stride that is not a multiple of 16 bytes", who, name);
    if (output) {                                   // sorted by stride, each dimension must clear the ones below it
        uint64_t reach = a->head_dim;
        bool used[3] = {false, false, false};
        for (int r = 0; r < 3; ++r) {
            int best = -1;
            for (int i = 0; i < 3; ++i)
                if (!used[i] && dim[i].extent > 1 && (best < 0 || dim[i].stride < dim[best].stride)) best = i;
            if (best < 0) break;
            used[best] = true;
            DBLP_REQUIRE((uint64_t)dim[best].stride >= reach, DBLP_EINVAL, "%s: sections of %s overlap", who, name);
            reach = (uint64_t)dim[best].stride * (dim[best].extent - 1) + reach;
        }
    }
    return DBLP_OK;
}

static AttnArgs make_args(const dblp_attention_t* a)
{
    AttnArgs r{};
    r.B = a->batch; r.Sq = a->q_tokens; r.Sk = a->k_tokens; r.Hq = a->q_heads; r.Hkv = a->kv_heads; r.D = a->head_dim;
    r.causal = a->flags & DBLP_ATTENTION_CAUSAL; r.scale = a->scale; r.q_lens = a->q_lens; r.k_lens = a->k_lens;
    return r;
}

}  // namespace dblp

using namespace dblp;

extern "C" int dblp_attention_workspace_bytes(const dblp_attention_t* a, size_t* fwd_bytes, size_t* grad_bytes)
{
    const int rc = check_shape("attention_workspace_bytes", a);
    if (rc != DBLP_OK) return rc;
    if (fwd_bytes) *fwd_bytes = 0;
    if (grad_bytes) *grad_bytes = (size_t)a->batch * a->q_heads * a->q_tokens * 4;
    return DBLP_OK;
}

#define DBLP_TRY(call)                      \
    do {                                    \
        const int rc_ = (call);             \
        if (rc_ != DBLP_OK) return rc_;     \
    } while (0)

extern "C" int dblp_attention(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                              const dblp_heads_t* out, float* lse, void* ws, size_t ws_bytes, void* stream)
{
    (void)ws; (void)ws_bytes;
    DBLP_TRY(check_shape("attention", a));
    if (a->batch == 0 || a->q_tokens == 0) return DBLP_OK;
    DBLP_TRY(check_heads("attention", "q", a, q, a->q_tokens, a->q_heads, false));
    DBLP_TRY(check_heads("attention", "out", a, out, a->q_tokens, a->q_heads, true));
    AttnArgs r = make_args(a);
    r.q = heads(q); r.o = heads(out); r.lse = lse;
    if (a->k_tokens) {
        DBLP_TRY(check_heads("attention", "k", a, k, a->k_tokens, a->kv_heads, false));
        DBLP_TRY(check_heads("attention", "v", a, v, a->k_tokens, a->kv_heads, false));
        r.k = heads(k); r.v = heads(v);
    }
    const dim3 grid((a->q_tokens + kAttnWarps - 1) / kAttnWarps, a->q_heads, a->batch);
    if (a->dtype == DBLP_BF16) k_attention<__nv_bfloat16><<<grid, kAttnWarps * 32, 0, (cudaStream_t)stream>>>(r);
    else k_attention<__half><<<grid, kAttnWarps * 32, 0, (cudaStream_t)stream>>>(r);
    DBLP_LAUNCHED();
    return DBLP_OK;
}

extern "C" int dblp_attention_grad(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                                   const dblp_heads_t* out, const dblp_heads_t* dout, const float* lse, const dblp_heads_t* dq,
                                   const dblp_heads_t* dk, const dblp_heads_t* dv, void* ws, size_t ws_bytes, void* stream)
{
    DBLP_TRY(check_shape("attention_grad", a));
    if (a->batch == 0) return DBLP_OK;
    AttnArgs r = make_args(a);
    if (a->q_tokens) {
        DBLP_TRY(check_heads("attention_grad", "q", a, q, a->q_tokens, a->q_heads, false));
        DBLP_TRY(check_heads("attention_grad", "out", a, out, a->q_tokens, a->q_heads, false));
        DBLP_TRY(check_heads("attention_grad", "dout", a, dout, a->q_tokens, a->q_heads, false));
        DBLP_TRY(check_heads("attention_grad", "dq", a, dq, a->q_tokens, a->q_heads, true));
        DBLP_REQUIRE(lse, DBLP_EINVAL, "attention_grad: lse is null");
        r.q = heads(q); r.o = heads(out); r.go = heads(dout); r.dq = heads(dq); r.lse = const_cast<float*>(lse);
    }
    if (a->k_tokens) {
        DBLP_TRY(check_heads("attention_grad", "k", a, k, a->k_tokens, a->kv_heads, false));
        DBLP_TRY(check_heads("attention_grad", "v", a, v, a->k_tokens, a->kv_heads, false));
        DBLP_TRY(check_heads("attention_grad", "dk", a, dk, a->k_tokens, a->kv_heads, true));
        DBLP_TRY(check_heads("attention_grad", "dv", a, dv, a->k_tokens, a->kv_heads, true));
        r.k = heads(k); r.v = heads(v); r.dk = heads(dk); r.dv = heads(dv);
    }
    size_t need = 0;
    DBLP_TRY(dblp_attention_workspace_bytes(a, nullptr, &need));
    DBLP_REQUIRE(need == 0 || (ws && ((uintptr_t)ws & 255) == 0), ws ? DBLP_EALIGN : DBLP_EINVAL,
                 "attention_grad: the workspace is null or not 256-byte aligned");
    DBLP_REQUIRE(ws_bytes >= need, DBLP_ECAPACITY, "attention_grad: workspace of %zu bytes, needs %zu", ws_bytes, need);
    r.delta = (float*)ws;
    cudaStream_t s = (cudaStream_t)stream;
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
