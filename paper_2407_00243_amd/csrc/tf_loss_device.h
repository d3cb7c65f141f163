// Sums of exponentials and what a row's loss is made of them, for the kernels of the cross entropy.
#pragma once
#include <hip/hip_runtime.h>

#include "tf_loss.h"

namespace tf {
namespace {

// Sums of exponentials over their largest argument: x holds that and the sum.
__device__ __forceinline__ Float2 add_sums(Float2 x, Float2 y) {
    constexpr float LOW = -__builtin_inff();
    const float m = fmaxf(x[0], y[0]);
    return Float2{m, (x[0] == LOW ? x[1] : x[1] * expf(x[0] - m)) + (y[0] == LOW ? y[1] : y[1] * expf(y[0] - m))};
}
// x: largest logit of all classes and the sum of the others than the label's over it; hit: the label's logit.  A small loss keeps its precision as
// log(1 + sum / exp(label's logit)).
__device__ __forceinline__ void write_loss(Float2 x, float hit, float *loss, float *lse) {
    const float top = x[0], sum = x[1], all = top + logf(sum + expf(hit - top));
    *lse = all;
    *loss = top - hit < 40.0f ? log1pf(sum * expf(top - hit)) : all - hit;
}

}  // namespace
}  // namespace tf
