// dblp_attention, dblp_attention_grad: argument checks, tensor maps and the entry points.
#include <math.h>

#include "attention.cuh"

namespace dblp {

static __device__ unsigned long long d_wait_timeouts;

constexpr int kMaxDevices = 64;

unsigned long long* timeout_counter()
{
    static std::atomic<void*> at[kMaxDevices];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev >= kMaxDevices) return nullptr;
    void* p = at[dev].load(std::memory_order_acquire);
    if (!p) {
        if (cudaGetSymbolAddress(&p, d_wait_timeouts) != cudaSuccess) return nullptr;
        at[dev].store(p, std::memory_order_release);
    }
    return (unsigned long long*)p;
}

EncodeTiled map_encoder()
{
    static std::atomic<void*> fn{nullptr};
    void* f = fn.load(std::memory_order_acquire);
    if (!f) {
        cudaDriverEntryPointQueryResult st;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &st) != cudaSuccess ||
            st != cudaDriverEntryPointSuccess)
            return nullptr;
        fn.store(f, std::memory_order_release);
    }
    return (EncodeTiled)f;
}

// Boxes of 128 tokens x 64 columns; what lies outside the tensor reads as zero.
int make_source(TileSource* t, const dblp_attention_t* a, const dblp_heads_t* h, uint32_t tokens, uint32_t nheads)
{
    const EncodeTiled encode = map_encoder();
    DBLP_REQUIRE(encode, DBLP_ECUDA, "attention: the driver has no cuTensorMapEncodeTiled");
    const cuuint64_t unused = (cuuint64_t)a->head_dim * 2;
    const bool hb = nheads > 1 && h->head_stride == 0, bb = a->batch > 1 && h->batch_stride == 0;
    const cuuint64_t dims[4] = {a->head_dim, tokens, hb ? 1u : nheads, bb ? 1u : a->batch};
    const cuuint64_t strides[3] = {tokens > 1 ? (cuuint64_t)h->token_stride * 2 : unused, dims[2] > 1 ? (cuuint64_t)h->head_stride * 2 : unused,
                                   dims[3] > 1 ? (cuuint64_t)h->batch_stride * 2 : unused};
    const cuuint32_t box[4] = {64, 128, 1, 1}, step[4] = {1, 1, 1, 1};
    const CUresult rc = encode(&t->map, a->dtype == DBLP_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
                               h->data, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    DBLP_REQUIRE(rc == CUDA_SUCCESS, DBLP_ECUDA, "attention: tensor map refused (driver error %d)", (int)rc);
    t->mh = hb ? 0 : 1;
    t->mb = bb ? 0 : 1;
    return DBLP_OK;
}

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
    DBLP_REQUIRE(((uintptr_t)a->q_lens & 3) == 0 && ((uintptr_t)a->k_lens & 3) == 0, DBLP_EALIGN, "%s: lengths are not aligned to their type", who);
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
        DBLP_REQUIRE(d.stride >= (&d == &dim[1] && !output ? 1 : 0) && d.stride < (1ll << 39), DBLP_EINVAL, "%s: %s has a stride of %lld", who, name, (long long)d.stride);
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

}  // namespace dblp

using namespace dblp;

#define DBLP_TRY(call)                      \
    do {                                    \
        const int rc_ = (call);             \
        if (rc_ != DBLP_OK) return rc_;     \
    } while (0)

extern "C" int dblp_attention_workspace_bytes(const dblp_attention_t* a, size_t* fwd_bytes, size_t* grad_bytes)
{
    DBLP_TRY(check_shape("attention_workspace_bytes", a));
    const size_t grad = a->batch ? attention_backward_space(a) : 0;            // the rules that cut the work divide by the batch
    DBLP_REQUIRE(grad < 1ull << 62, DBLP_ECAPACITY, "attention_workspace_bytes: the gradient's workspace passes 2^62 bytes");
    if (fwd_bytes) *fwd_bytes = a->batch ? attention_forward_space(a) : 0;
    if (grad_bytes) *grad_bytes = grad;
    return DBLP_OK;
}

static int check_space(const char* who, const void* ws, size_t ws_bytes, size_t need)
{
    DBLP_REQUIRE(need == 0 || ws, DBLP_EINVAL, "%s: the workspace is null", who);
    DBLP_REQUIRE(need == 0 || ((uintptr_t)ws & 255) == 0, DBLP_EALIGN, "%s: the workspace is not 256-byte aligned", who);
    DBLP_REQUIRE(ws_bytes >= need, DBLP_ECAPACITY, "%s: workspace of %zu bytes, needs %zu", who, ws_bytes, need);
    return DBLP_OK;
}

extern "C" int dblp_attention(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                              const dblp_heads_t* out, float* lse, void* ws, size_t ws_bytes, void* stream)
{
    DBLP_TRY(check_shape("attention", a));
    if (a->batch == 0 || a->q_tokens == 0) return DBLP_OK;
    DBLP_TRY(check_heads("attention", "q", a, q, a->q_tokens, a->q_heads, false));
    DBLP_TRY(check_heads("attention", "out", a, out, a->q_tokens, a->q_heads, true));
    if (a->k_tokens) {
        DBLP_TRY(check_heads("attention", "k", a, k, a->k_tokens, a->kv_heads, false));
        DBLP_TRY(check_heads("attention", "v", a, v, a->k_tokens, a->kv_heads, false));
    }
    DBLP_REQUIRE(((uintptr_t)lse & 3) == 0, DBLP_EALIGN, "attention: lse is not aligned to its type");
    DBLP_TRY(check_space("attention", ws, ws_bytes, attention_forward_space(a)));
    return attention_forward(a, q, k, v, out, lse, ws, (cudaStream_t)stream);
}

extern "C" int dblp_attention_grad(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                                   const dblp_heads_t* out, const dblp_heads_t* dout, const float* lse, const dblp_heads_t* dq,
                                   const dblp_heads_t* dk, const dblp_heads_t* dv, void* ws, size_t ws_bytes, void* stream)
{
    DBLP_TRY(check_shape("attention_grad", a));
    if (a->batch == 0 || (a->q_tokens == 0 && a->k_tokens == 0)) return DBLP_OK;
    if (a->q_tokens) {
        DBLP_TRY(check_heads("attention_grad", "q", a, q, a->q_tokens, a->q_heads, false));
        DBLP_TRY(check_heads("attention_grad", "out", a, out, a->q_tokens, a->q_heads, false));
        DBLP_TRY(check_heads("attention_grad", "dout", a, dout, a->q_tokens, a->q_heads, false));
        DBLP_TRY(check_heads("attention_grad", "dq", a, dq, a->q_tokens, a->q_heads, true));
        DBLP_REQUIRE(lse, DBLP_EINVAL, "attention_grad: lse is null");
        DBLP_REQUIRE(((uintptr_t)lse & 3) == 0, DBLP_EALIGN, "attention_grad: lse is not aligned to its type");
    }
    if (a->k_tokens) {
        DBLP_TRY(check_heads("attention_grad", "k", a, k, a->k_tokens, a->kv_heads, false));
        DBLP_TRY(check_heads("attention_grad", "v", a, v, a->k_tokens, a->kv_heads, false));
        DBLP_TRY(check_heads("attention_grad", "dk", a, dk, a->k_tokens, a->kv_heads, true));
        DBLP_TRY(check_heads("attention_grad", "dv", a, dv, a->k_tokens, a->kv_heads, true));
    }
    DBLP_TRY(check_space("attention_grad", ws, ws_bytes, attention_backward_space(a)));
    return attention_backward(a, q, k, v, out, dout, lse, dq, dk, dv, ws, (cudaStream_t)stream);
}

extern "C" int dblp_wait_timeouts(uint64_t* count)
{
    DBLP_REQUIRE(count, DBLP_EINVAL, "wait_timeouts: null output");
    unsigned long long* p = timeout_counter(), v = 0;
    DBLP_REQUIRE(p, DBLP_ECUDA, "wait_timeouts: no device counter: %s", cudaGetErrorString(cudaGetLastError()));
    DBLP_CUDA(cudaMemcpy(&v, p, sizeof(v), cudaMemcpyDeviceToHost));
    *count = v;
    return DBLP_OK;
}
