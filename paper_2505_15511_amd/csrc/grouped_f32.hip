// libnomad: grouped products of float32 operands.
#include "grouped_launch.h"

namespace nomad_grouped {

void product_f32(const ProductArgs& p, ProductTile tile, bool, bool w_kc, bool loads, bool stores, int units, hipStream_t st) {
    launch_product_type<float, float>(p, tile, w_kc, loads, stores, units, st);
}
void gradient_f32(const GradientArgs& p, const GradientPlan& plan, bool, bool loads, bool stores, int units, hipStream_t st) {
    launch_gradient_type<float, float>(p, plan, loads, stores, units, st);
}

}  // namespace nomad_grouped
