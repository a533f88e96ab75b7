// Matrix products C[m, n] = sum over k of A[m, k] B[k, n], for the linear layer, its gradients and the orthogonalised update.
#pragma once

#include "epilogue.cuh"

namespace dblp {

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
    bool runs;                  // the result is wanted to fp32's precision: the tensor cores' sums, which truncate, are taken in short runs
    bool symmetric;             // M = N and the result equals its transpose: computed once, written twice
};

size_t product_space(const Product& p);          // bytes of workspace
// chained: the kernels before it on the stream belong to the same call and let this one be set up while they run
template <typename E> int run_product(const Product& p, const E& epilogue, void* ws, bool chained, cudaStream_t s);

}  // namespace dblp
