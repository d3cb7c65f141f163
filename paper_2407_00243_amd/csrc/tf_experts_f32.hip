// Experts' products in f32.
#include "tf_experts.h"

namespace tf {
int launch_experts_f32(const ExpertLaunch &a, void *stream) { return launch_experts_el<TF_F32>(a, stream); }
}  // namespace tf
