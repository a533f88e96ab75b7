// Matrix products C[m, n] = sum over k of A[m, k] B[k, n], for the linear layer, its gradients and the orthogonalised update.
#pragma once

#include "epilogue.cuh"
#include "product_plan.h"

namespace dblp {

// A row-major matrix that the kernels around the products read, eight elements at a time.
struct Source {
    const void* p;
    int64_t stride;
    int dtype;
    bool vec;                   // data and stride allow 16-byte accesses
};
inline Source source_of(const void* p, int64_t stride, uint64_t rows, int dtype)
{
    if (rows <= 1) stride = 0;
    return Source{p, stride, dtype, ((uintptr_t)p | (uint64_t)stride * element_bytes(dtype)) % 16 == 0};
}
__device__ __forceinline__ void load8(const Source& r, uint32_t m, uint32_t n, uint32_t left, float* x)
{
    const int64_t at = (int64_t)m * r.stride + n;
    auto go = [&](auto tag) {
        using T = decltype(tag);
        const T* p = (const T*)r.p + at;
        if (r.vec && left >= 8) {
            Vec8<T> v;
            v.load(p);
            v.get(x);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) x[i] = i < left ? to_f32(p[i]) : 0.0f;
        }
    };
    if (r.dtype == DBLP_F32) go(float());
    else if (r.dtype == DBLP_BF16) go(__nv_bfloat16());
    else go(__half());
}

size_t product_space(const Product& p);          // bytes of workspace
// chained: the kernels before it on the stream belong to the same call and let this one be set up while they run
// RUNS: the result is wanted to fp32's precision (the tensor cores' own sums truncate); without it long sums alone are taken in runs.
template <bool RUNS, typename E> int run_product(const Product& p, const E& epilogue, void* ws, bool chained, cudaStream_t s);

// parts of it that are the same for every epilogue
int make_map(CUtensorMap* map, const void* data, int64_t stride, const Operand& o, uint32_t rows, uint32_t K, uint32_t batch, uint32_t box, int dtype);
int make_store_map(CUtensorMap* map, const Output& o, const Product& p);
int repack(const Operand& o, void* to, uint32_t stride, uint32_t outer, uint32_t inner, cudaStream_t s);

}  // namespace dblp
