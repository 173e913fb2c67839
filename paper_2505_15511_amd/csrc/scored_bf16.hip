// libnomad: routing by scores of bf16 logits.
#include "scored_launch.h"

namespace nomad_router {

void scored_bf16(const ScoredArgs& p, bool vec, hipStream_t st) { launch_scored<__bf16>(p, vec, st); }
void scored_gradient_bf16(const ScoredGradientArgs& p, bool vec, hipStream_t st) { launch_scored_gradient_type<__bf16>(p, vec, st); }

}  // namespace nomad_router
