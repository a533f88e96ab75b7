// The products of dblp_linear_grad for dx.
#include "product_kernels.cuh"

namespace dblp {

DBLP_PRODUCT(false, EpiGradX<__nv_bfloat16>);
DBLP_PRODUCT(false, EpiGradX<__half>);

}  // namespace dblp
