// Products of the cross entropy: fp16 operands.
#include "tf_product.h"

namespace tf {
int launch_product_f16(const ProductLaunch &a, void *stream) { return product<TF_F16>(a, stream); }
}  // namespace tf
