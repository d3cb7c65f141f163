// Products of the cross entropy: fp32 operands.
#include "tf_product.h"

namespace tf {
int launch_product_f32(const ProductLaunch &a, void *stream) { return product<TF_F32>(a, stream); }
}  // namespace tf
