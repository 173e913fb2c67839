// libnomad: grouped products of bf16 operands.
#include "grouped_launch.h"

namespace nomad_grouped {

void product_bf16(const ProductArgs& p, ProductTile tile, bool wide, bool w_kc, bool loads, bool stores, int units, hipStream_t st) {
    if (wide) launch_product_type<__bf16, float>(p, tile, w_kc, loads, stores, units, st);
    else launch_product_type<__bf16, __bf16>(p, tile, w_kc, loads, stores, units, st);
}
void gradient_bf16(const GradientArgs& p, const GradientPlan& plan, bool wide, bool loads, bool stores, int units, hipStream_t st) {
    if (wide) launch_gradient_type<__bf16, float>(p, plan, loads, stores, units, st);
    else launch_gradient_type<__bf16, __bf16>(p, plan, loads, stores, units, st);
}

}  // namespace nomad_grouped
