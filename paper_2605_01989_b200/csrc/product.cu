// Matrix products: workspace, tensor maps and the copies of operands that TMA cannot address.  The kernels are in product_kernels.cuh,
// built for their epilogues by product_linear_*.cu, product_dx.cu, product_dw.cu, product_poly.cu and product_last.cu.
#include "product.cuh"

namespace dblp {

// Rows of any stride and alignment -> rows of `to` elements, a multiple of eight.
__global__ void __launch_bounds__(256) k_repack(const uint16_t* src, int64_t stride, uint16_t* dst, uint32_t to, uint32_t rows, uint32_t cols)
{
    after_start();
    const uint32_t per_row = to / 8;
    const uint64_t x = (uint64_t)blockIdx.x * 256 + threadIdx.x, r = x / per_row;
    if (r >= rows) return;
    const uint32_t c = (uint32_t)(x - r * per_row) * 8;
    const uint16_t* p = src + (int64_t)r * stride + c;
    uint32_t w[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
        w[i] = (c + 2 * i < cols ? p[2 * i] : 0u) | (c + 2 * i + 1 < cols ? (uint32_t)p[2 * i + 1] << 16 : 0u);
    *reinterpret_cast<uint4*>(dst + r * to + c) = make_uint4(w[0], w[1], w[2], w[3]);
}

size_t product_space(const Product& p)
{
    if (rows_take(p)) return 0;
    const ProductPlan r = plan_product(p);
    return r.a_bytes + r.b_bytes + r.partial_bytes;
}

// Boxes of `box` rows x 64 of the summed dimension, or of 64 rows x 64 where the rows are contiguous; zero outside.
int make_map(CUtensorMap* map, const void* data, int64_t stride, const Operand& o, uint32_t rows, uint32_t K, uint32_t batch, uint32_t box, int dtype)
{
    const EncodeTiled encode = map_encoder();
    DBLP_REQUIRE(encode, DBLP_ECUDA, "product: the driver has no cuTensorMapEncodeTiled");
    const uint32_t inner = o.mn ? rows : K, outer = o.mn ? K : rows;
    const cuuint64_t unused = ((cuuint64_t)inner + 7) / 8 * 16;
    const cuuint64_t dims[3] = {inner, outer, batch}, strides[2] = {outer > 1 ? (cuuint64_t)stride * 2 : unused, batch > 1 ? (cuuint64_t)o.each * 2 : unused};
    const cuuint32_t boxes[3] = {64, o.mn ? 64 : box, 1}, ones[3] = {1, 1, 1};
    const CUresult rc = encode(map, dtype == DBLP_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, (void*)data, dims, strides,
                               boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    DBLP_REQUIRE(rc == CUDA_SUCCESS, DBLP_ECUDA, "product: tensor map refused (driver error %d)", (int)rc);
    return DBLP_OK;
}

// Pieces of 32 x 32 of a result.
int make_store_map(CUtensorMap* map, const Output& o, const Product& p)
{
    const EncodeTiled encode = map_encoder();
    DBLP_REQUIRE(encode, DBLP_ECUDA, "product: the driver has no cuTensorMapEncodeTiled");
    const cuuint64_t unused = ((cuuint64_t)p.N * o.bytes + 15) / 16 * 16;
    const cuuint64_t dims[3] = {p.N, p.M, p.batch}, strides[2] = {p.M > 1 ? (cuuint64_t)o.stride * o.bytes : unused, p.batch > 1 ? (cuuint64_t)o.each * o.bytes : unused};
    const cuuint32_t boxes[3] = {32, 32, 1}, ones[3] = {1, 1, 1};
    const CUresult rc = encode(map, o.bytes == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, o.p, dims, strides, boxes, ones,
                               CU_TENSOR_MAP_INTERLEAVE_NONE, o.bytes == 4 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                               CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    DBLP_REQUIRE(rc == CUDA_SUCCESS, DBLP_ECUDA, "product: tensor map of a result refused (driver error %d)", (int)rc);
    return DBLP_OK;
}

int repack(const Operand& o, void* to, uint32_t stride, uint32_t outer, uint32_t inner, cudaStream_t s)
{
    const uint64_t blocks = ((uint64_t)outer * (stride / 8) + 255) / 256;
    DBLP_REQUIRE(blocks < 1ull << 31, DBLP_ECAPACITY, "product: an operand of 2^42 elements or more");
    k_repack<<<(unsigned)blocks, 256, 0, s>>>((const uint16_t*)o.p, o.stride, (uint16_t*)to, stride, outer, inner);
    DBLP_LAUNCHED();
    return DBLP_OK;
}

}  // namespace dblp
