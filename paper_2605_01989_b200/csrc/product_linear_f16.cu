// The products of dblp_linear, operands in f16.
#include "product_kernels.cuh"

namespace dblp {

DBLP_PRODUCT(false, EpiLinear<__half, __half>);
DBLP_PRODUCT(true, EpiLinear<__half, float>);

}  // namespace dblp
