// libnomad: routing by scores of f16 logits.
#include "scored_launch.h"

namespace nomad_router {

void scored_f16(const ScoredArgs& p, bool vec, hipStream_t st) { launch_scored<_Float16>(p, vec, st); }
void scored_gradient_f16(const ScoredGradientArgs& p, bool vec, hipStream_t st) { launch_scored_gradient_type<_Float16>(p, vec, st); }

}  // namespace nomad_router
