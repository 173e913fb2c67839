// libnomad: dense products of f16 operands.
#include "dense_launch.h"

namespace nomad_dense {

void dense_f16(const DenseArgs& p, const Launch& l, hipStream_t st) { launch_type<_Float16>(p, l, st); }
void slope_f16(const SlopeArgs& p, int64_t parts, bool vec, hipStream_t st) { launch_slope<_Float16>(p, parts, vec, st); }

}  // namespace nomad_dense
