// The products of dblp_linear_grad.
#include "product_kernels.cuh"

namespace dblp {

DBLP_PRODUCT(false, EpiGradX<__nv_bfloat16>);
DBLP_PRODUCT(false, EpiGradX<__half>);
DBLP_PRODUCT(false, EpiStore<__nv_bfloat16>);
DBLP_PRODUCT(false, EpiStore<__half>);
DBLP_PRODUCT(true, EpiStore<float>);

}  // namespace dblp
