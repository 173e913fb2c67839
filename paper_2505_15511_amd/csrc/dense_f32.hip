// libnomad: dense products of f32 operands.
#include "dense_launch.h"

namespace nomad_dense {

void dense_f32(const DenseArgs& p, const Launch& l, hipStream_t st) { launch_type<float>(p, l, st); }
void slope_f32(const SlopeArgs& p, int64_t parts, bool vec, hipStream_t st) { launch_slope<float>(p, parts, vec, st); }

}  // namespace nomad_dense
