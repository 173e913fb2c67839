// libnomad: dense products of bf16 operands.
#include "dense_launch.h"

namespace nomad_dense {

void dense_bf16(const DenseArgs& p, const Launch& l, hipStream_t st) { launch_type<__bf16>(p, l, st); }
void slope_bf16(const SlopeArgs& p, int64_t parts, bool vec, hipStream_t st) { launch_slope<__bf16>(p, parts, vec, st); }

}  // namespace nomad_dense
