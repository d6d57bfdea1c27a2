// The products of som_product.h on __bf16.
#include "som_product.h"

namespace som {

hipError_t launch_product_bf16(ProductArgs a, const ProductPlan &p, hipStream_t stream) {
    return launch_product<__bf16>(a, p, stream);
}

}  // namespace som
