// The products of dblp_linear_grad for dw.
#include "product_kernels.cuh"

namespace dblp {

DBLP_PRODUCT(false, EpiStore<__nv_bfloat16>);
DBLP_PRODUCT(false, EpiStore<__half>);
DBLP_PRODUCT(true, EpiStore<float>);

}  // namespace dblp
