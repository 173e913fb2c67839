// libnomad: grouped products of bf16 operands.
#include "grouped_launch.h"

namespace nomad_grouped {

void product_bf16(const ProductArgs& p, ProductTile tile, bool wide, bool w_kc, bool fast, int units, hipStream_t st) {
    if (wide) launch_product_type<__bf16, float>(p, tile, w_kc, fast, units, st);
    else launch_product_type<__bf16, __bf16>(p, tile, w_kc, fast, units, st);
}
void gradient_bf16(const GradientArgs& p, const GradientPlan& plan, bool wide, bool fast, int units, hipStream_t st) {
    if (wide) launch_gradient_type<__bf16, float>(p, plan, fast, units, st);
    else launch_gradient_type<__bf16, __bf16>(p, plan, fast, units, st);
}

}  // namespace nomad_grouped
