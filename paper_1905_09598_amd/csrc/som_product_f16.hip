// The products of som_product.h on _Float16.
#include "som_product.h"

namespace som {

hipError_t launch_product_f16(ProductArgs a, const ProductPlan &p, hipStream_t stream) {
    return launch_product<_Float16>(a, p, stream);
}

}  // namespace som
