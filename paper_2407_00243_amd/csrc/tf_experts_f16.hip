// Experts' products in f16.
#include "tf_experts.h"

namespace tf {
int launch_experts_f16(const ExpertLaunch &a, void *stream) { return launch_experts_el<TF_F16>(a, stream); }
}  // namespace tf
