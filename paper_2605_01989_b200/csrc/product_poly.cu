// The products of dblp_orthogonalize but the last.
#include "product_kernels.cuh"

namespace dblp {

DBLP_PRODUCT(false, EpiPoly<true>);
DBLP_PRODUCT(true, EpiPoly<true>);
DBLP_PRODUCT(false, EpiPoly<false>);
DBLP_PRODUCT(true, EpiPoly<false>);

}  // namespace dblp
