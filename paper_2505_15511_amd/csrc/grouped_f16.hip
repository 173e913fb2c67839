// libnomad: grouped products of f16 operands.
#include "grouped_launch.h"

namespace nomad_grouped {

void product_f16(const ProductArgs& p, ProductTile tile, bool wide, bool w_kc, bool loads, bool stores, int units, hipStream_t st) {
    if (wide) launch_product_type<_Float16, float>(p, tile, w_kc, loads, stores, units, st);
    else launch_product_type<_Float16, _Float16>(p, tile, w_kc, loads, stores, units, st);
}
void gradient_f16(const GradientArgs& p, const GradientPlan& plan, bool wide, bool loads, bool stores, int units, hipStream_t st) {
    if (wide) launch_gradient_type<_Float16, float>(p, plan, loads, stores, units, st);
    else launch_gradient_type<_Float16, _Float16>(p, plan, loads, stores, units, st);
}

}  // namespace nomad_grouped
