// Experts' products in bf16.
#include "tf_experts.h"

namespace tf {
int launch_experts_bf16(const ExpertLaunch &a, void *stream) { return launch_experts_el<TF_BF16>(a, stream); }
}  // namespace tf
