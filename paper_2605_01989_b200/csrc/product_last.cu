// The last product of dblp_orthogonalize.
#include "product_kernels.cuh"

namespace dblp {

DBLP_PRODUCT(false, EpiLast<__nv_bfloat16>);
DBLP_PRODUCT(true, EpiLast<__nv_bfloat16>);
DBLP_PRODUCT(true, EpiLast<__half>);
DBLP_PRODUCT(true, EpiLast<float>);

}  // namespace dblp
