// The products of som_product.h on float.
#include "som_product.h"

namespace som {

hipError_t launch_product_f32(ProductArgs a, const ProductPlan &p, hipStream_t stream) {
    return launch_product<float>(a, p, stream);
}

}  // namespace som
