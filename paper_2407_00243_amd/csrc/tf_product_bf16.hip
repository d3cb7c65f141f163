// Products of the cross entropy: bf16 operands (and fp32 ones, as three of them).
#include "tf_product.h"

namespace tf {
int launch_product_bf16(const ProductLaunch &a, void *stream) { return product<TF_BF16>(a, stream); }
}  // namespace tf
