// The products of dblp_linear, operands in bf16.
#include "product_kernels.cuh"

namespace dblp {

DBLP_PRODUCT(false, EpiLinear<__nv_bfloat16, __nv_bfloat16>);
DBLP_PRODUCT(true, EpiLinear<__nv_bfloat16, float>);

}  // namespace dblp
