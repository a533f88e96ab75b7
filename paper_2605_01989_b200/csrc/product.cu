// Matrix products, first form: one thread a row and eight columns, fp32.
#include "product.cuh"

namespace dblp {

template <typename T> __device__ __forceinline__ float word(const Operand& o, uint32_t b, uint32_t r, uint32_t k)
{
    const int64_t at = b * o.each + (o.mn ? (int64_t)k * o.stride + r : (int64_t)r * o.stride + k);
    return to_f32(((const T*)o.p)[at]) + (o.lo ? to_f32(((const T*)o.lo)[at]) : 0.0f);
}

template <typename T, typename E> __global__ void __launch_bounds__(256) k_product(const __grid_constant__ Product p, const __grid_constant__ E e)
{
    const uint32_t n = (blockIdx.x * 32 + threadIdx.x) * 8, m = blockIdx.y * 8 + threadIdx.y, b = blockIdx.z;
    if (m >= p.M || n >= p.N) return;
    const uint32_t left = min(8u, p.N - n);
    float v[8] = {};
    for (uint32_t k = 0; k < p.K; ++k) {
        const float x = word<T>(p.a, b, m, k);
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < left) v[i] = fmaf(x, word<T>(p.b, b, n + i, k), v[i]);
    }
    e.apply(b, m, n, left, v);
}

size_t product_space(const Product&) { return 0; }

template <typename E> int run_product(const Product& p, const E& e, void*, cudaStream_t s)
{
    const dim3 grid((p.N + 255) / 256, (p.M + 7) / 8, p.batch), block(32, 8);
    if (p.dtype == DBLP_BF16) k_product<__nv_bfloat16, E><<<grid, block, 0, s>>>(p, e);
    else k_product<__half, E><<<grid, block, 0, s>>>(p, e);
    DBLP_LAUNCHED();
    return DBLP_OK;
}

template int run_product(const Product&, const EpiLinear&, void*, cudaStream_t);
template int run_product(const Product&, const EpiGradX&, void*, cudaStream_t);
template int run_product(const Product&, const EpiStore&, void*, cudaStream_t);
template int run_product(const Product&, const EpiPoly&, void*, cudaStream_t);
template int run_product(const Product&, const EpiLast&, void*, cudaStream_t);

}  // namespace dblp
