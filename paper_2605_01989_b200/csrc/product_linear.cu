// The products of dblp_linear.
#include "product_kernels.cuh"

namespace dblp {

DBLP_PRODUCT(false, EpiLinear<__nv_bfloat16, __nv_bfloat16>);
DBLP_PRODUCT(false, EpiLinear<__half, __half>);
DBLP_PRODUCT(true, EpiLinear<__nv_bfloat16, float>);
DBLP_PRODUCT(true, EpiLinear<__half, float>);

}  // namespace dblp
