// Shared by the attention kernels: argument block, index rules, host-side checks and tensor maps.
#pragma once

#include "tc.cuh"

namespace dblp {

struct Heads {
    void* p;
    int64_t sb, st, sh;
};

// A tensor as TMA sees it: dimensions (column, token, head, batch).  A dimension of stride 0 is entered with extent 1 and
// its coordinate multiplied by 0.
struct TileSource {
    CUtensorMap map;
    int mh, mb;
};

struct AttnShape {
    uint32_t B, Sq, Sk, Hq, Hkv, D, causal, rep;
    const int32_t *q_lens, *k_lens;
};

__device__ __forceinline__ uint32_t length_of(const int32_t* lens, uint32_t b, uint32_t extent)
{
    return lens ? (uint32_t)min(max(lens[b], 0), (int32_t)extent) : extent;
}

// Keys that query i of a sequence sees: 0 .. result - 1.
__device__ __forceinline__ uint32_t keys_of(uint32_t i, uint32_t lq, uint32_t lk, uint32_t causal)
{
    if (i >= lq) return 0;
    return causal ? (uint32_t)max(0, (int32_t)(i + 1 + lk) - (int32_t)lq) : lk;
}

template <int NS>
__device__ __forceinline__ void load_tile(uint8_t* dst, const TileSource& src, uint64_t* bar, uint32_t token, uint32_t head, uint32_t b)
{
#pragma unroll
    for (int s = 0; s < NS; ++s)
        tma_tile(dst + s * kBlockBytes, &src.map, bar, s * 64, (int)token, (int)head * src.mh, (int)b * src.mb);
}

// Rows first .. last - 1 of a 128-row tile become zero: what lies beyond a sequence, or sees nothing, may hold anything, and
// 0 * NaN is NaN inside a product.  Called by one whole warp, for tiles that hold such a boundary only.
template <int NS>
__device__ __forceinline__ void clear_rows(uint8_t* tile, uint32_t first, uint32_t last)
{
    const uint32_t lane = threadIdx.x & 31;
    for (uint32_t i = first * 8 + lane; i < last * 8; i += 32)
#pragma unroll
        for (int s = 0; s < NS; ++s) *reinterpret_cast<uint4*>(tile + s * kBlockBytes + i * 16) = make_uint4(0, 0, 0, 0);
    fence_async_smem();
}

// dblp_attention for few queries a key head (attention_rows.cu)
bool few_rows(const dblp_attention_t* a);
size_t rows_space(const dblp_attention_t* a);
int attention_rows(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                   const dblp_heads_t* out, float* lse, void* ws, cudaStream_t s);
// dblp_attention_grad for few queries a key head (attention_rows.cu)
bool few_grad_rows(const dblp_attention_t* a);
size_t grad_rows_space(const dblp_attention_t* a);
int attention_grad_rows(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                        const dblp_heads_t* out, const dblp_heads_t* dout, const float* lse, const dblp_heads_t* dq,
                        const dblp_heads_t* dk, const dblp_heads_t* dv, void* ws, cudaStream_t s);
int attention_forward(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                      const dblp_heads_t* out, float* lse, void* ws, cudaStream_t s);
size_t attention_forward_space(const dblp_attention_t* a);
int attention_backward(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                       const dblp_heads_t* out, const dblp_heads_t* dout, const float* lse, const dblp_heads_t* dq,
                       const dblp_heads_t* dk, const dblp_heads_t* dv, void* ws, cudaStream_t s);
size_t attention_backward_space(const dblp_attention_t* a);

// Lets kernel K use `bytes` of shared memory on the current device; asked of the runtime once per kernel and device.
template <auto K> inline cudaError_t allow_shared(int bytes)
{
    static std::atomic<unsigned long long> done{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 64 && (done.load(std::memory_order_acquire) >> dev & 1)) return cudaSuccess;
    e = cudaFuncSetAttribute(K, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_acq_rel);
    return e;
}

unsigned long long* timeout_counter();     // of the current device; null after a CUDA error
int make_source(TileSource* t, const dblp_attention_t* a, const dblp_heads_t* h, uint32_t tokens, uint32_t nheads);
inline Heads heads(const dblp_heads_t* h) { return h ? Heads{h->data, h->batch_stride, h->token_stride, h->head_stride} : Heads{}; }
inline AttnShape shape_of(const dblp_attention_t* a)
{
    return AttnShape{a->batch, a->q_tokens, a->k_tokens, a->q_heads, a->kv_heads, a->head_dim,
                     a->flags & (uint32_t)DBLP_ATTENTION_CAUSAL, a->q_heads / a->kv_heads, a->q_lens, a->k_lens};
}

}  // namespace dblp
