// Matrix products C[m, n] = sum over k of A[m, k] B[k, n], for the linear layer, its gradients and the orthogonalised update.
#pragma once

#include "epilogue.cuh"

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

// A 16-bit operand: its rows (m of A, n of B) and the summed dimension, one of which is contiguous.
struct Operand {
    const void* p;
    const void* lo;             // second word of each element (terms = 3), or null
    int64_t stride;             // of the other dimension, in elements
    int64_t each;               // from one product of a batch to the next
    bool mn;                    // the rows are contiguous, not the summed dimension
};

struct Product {
    Operand a, b;
    uint32_t M, N, K, batch;
    int dtype;                  // of both operands
    int terms;                  // 1, or 3: hi hi + hi lo + lo hi
    bool few;                   // few rows (M) may be computed as columns
    bool symmetric;             // M = N and the result equals its transpose: computed once, written twice
};

size_t product_space(const Product& p);          // bytes of workspace
// chained: the kernels before it on the stream belong to the same call and let this one be set up while they run
// RUNS: the result is wanted to fp32's precision (the tensor cores' own sums truncate).
template <bool RUNS, typename E> int run_product(const Product& p, const E& epilogue, void* ws, bool chained, cudaStream_t s);

}  // namespace dblp
