// libnomad: routing by scores of f32 logits.
#include "scored_launch.h"

namespace nomad_router {

void scored_f32(const ScoredArgs& p, bool vec, hipStream_t st) { launch_scored<float>(p, vec, st); }
void scored_gradient_f32(const ScoredGradientArgs& p, bool vec, hipStream_t st) { launch_scored_gradient_type<float>(p, vec, st); }

}  // namespace nomad_router
