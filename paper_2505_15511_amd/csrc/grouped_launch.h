// Launches of the grouped products for one element type (each type has a source file of its own: they compile side by side).
#pragma once
#include "grouped_kernels.h"
#include "grouped_plan.h"
#include "host_util.h"

namespace nomad_grouped {

// loads, stores: rows of whole 16-byte chunks where they are read, where they are written
void product_f32(const ProductArgs& p, ProductTile tile, bool wide, bool w_kc, bool loads, bool stores, int units, hipStream_t st);
void product_bf16(const ProductArgs& p, ProductTile tile, bool wide, bool w_kc, bool loads, bool stores, int units, hipStream_t st);
void product_f16(const ProductArgs& p, ProductTile tile, bool wide, bool w_kc, bool loads, bool stores, int units, hipStream_t st);
void gradient_f32(const GradientArgs& p, const GradientPlan& plan, bool wide, bool loads, bool stores, int units, hipStream_t st);
void gradient_bf16(const GradientArgs& p, const GradientPlan& plan, bool wide, bool loads, bool stores, int units, hipStream_t st);
void gradient_f16(const GradientArgs& p, const GradientPlan& plan, bool wide, bool loads, bool stores, int units, hipStream_t st);

// workgroups a compute unit holds at a time: what fits its 160 KB of LDS and eight wavefronts (the kernels take up to 256 registers)
template <int TA, int TB, int WAVES>
constexpr int resident() { return std::max(1, std::min(163840 / (2 * (TA + TB) * kStepBytes), 8 / WAVES)); }

template <typename T, typename O, int TA, int TB, int WA, int WB, bool W_KC, bool LOADS, bool STORES>
void launch_product(const ProductArgs& p, int units, hipStream_t st) {
    const int64_t rows = std::min<int64_t>(p.rows, p.rows / TB + p.n_groups + 1);   // tiles of them: no more than one a row, one a group beyond the whole ones
    const int64_t total = rows * tiles_of(p.out, TA), at_once = (int64_t)units * resident<TA, TB, WA * WB>();
    hipLaunchKernelGGL((k_grouped_product<T, O, TA, TB, WA, WB, W_KC, LOADS, STORES>), dim3((uint32_t)std::min(total, at_once)), dim3(64 * WA * WB), 0, st, p);
}
template <typename T, typename O, int TA, int TB, int WA, int WB, bool W_KC>
void launch_product_ends(const ProductArgs& p, bool loads, bool stores, int units, hipStream_t st) {
    if (loads && stores) launch_product<T, O, TA, TB, WA, WB, W_KC, true, true>(p, units, st);
    else if (stores) launch_product<T, O, TA, TB, WA, WB, W_KC, false, true>(p, units, st);
    else launch_product<T, O, TA, TB, WA, WB, W_KC, false, false>(p, units, st);
}
template <typename T, typename O, bool W_KC>
void launch_product_tile(const ProductArgs& p, ProductTile tile, bool loads, bool stores, int units, hipStream_t st) {
    if (tile == kProductFew) {
        const int64_t rows = std::min<int64_t>(p.rows, p.rows / 16 + p.n_groups + 1);
        hipLaunchKernelGGL((k_grouped_few<T, O>), grid_of(rows * tiles_of(p.out, 16)), dim3(64 * kFewWaves), 0, st, p);
    } else if (tile == kProduct16) {
        if (loads && !stores) launch_product<T, O, 16, 256, 1, 4, W_KC, true, false>(p, units, st);   // (results of two columns: coordinates)
        else launch_product_ends<T, O, 16, 256, 1, 4, W_KC>(p, loads, stores, units, st);
    } else if (tile == kProduct64) {
        launch_product_ends<T, O, 64, 128, 2, 2, W_KC>(p, loads, stores, units, st);
    } else if (tile == kProduct128 || !loads || !stores || sizeof(T) == 4) {
        launch_product_ends<T, O, 128, 128, 2, 2, W_KC>(p, loads, stores, units, st);
    } else if constexpr (sizeof(T) == 2) {
        launch_product<T, O, 256, 256, 4, 2, W_KC, true, true>(p, units, st);
    }
}
template <typename T, typename O>
void launch_product_type(const ProductArgs& p, ProductTile tile, bool w_kc, bool loads, bool stores, int units, hipStream_t st) {
    if (w_kc) launch_product_tile<T, O, true>(p, tile, loads, stores, units, st);
    else launch_product_tile<T, O, false>(p, tile, loads, stores, units, st);
}

template <typename T, typename O, int TA, int TB, int WA, int WB, bool LOADS, bool STORES>
void launch_gradient(const GradientArgs& p, int units, hipStream_t st) {
    const int64_t total = tiles_of(p.in, TA) * tiles_of(p.out, TB) * (p.n_groups + p.rows / p.most);   // (a group has one part and one more for every `most` rows at most)
    const int64_t at_once = (int64_t)units * resident<TA, TB, WA * WB>();
    hipLaunchKernelGGL((k_grouped_gradient<T, O, TA, TB, WA, WB, LOADS, STORES>), dim3((uint32_t)std::min(total, at_once)), dim3(64 * WA * WB), 0, st, p);
}
template <typename T, typename O, int TA, int TB, int WA, int WB>
void launch_gradient_ends(const GradientArgs& p, bool loads, bool stores, int units, hipStream_t st) {
    if (loads && stores) launch_gradient<T, O, TA, TB, WA, WB, true, true>(p, units, st);
    else if (stores) launch_gradient<T, O, TA, TB, WA, WB, false, true>(p, units, st);
    else launch_gradient<T, O, TA, TB, WA, WB, false, false>(p, units, st);
}
template <typename T, typename O>
void launch_gradient_type(const GradientArgs& p, const GradientPlan& plan, bool loads, bool stores, int units, hipStream_t st) {
    if (plan.tile == kGradient16) {
        launch_gradient_ends<T, O, 128, 16, 4, 1>(p, loads, stores, units, st);
    } else if (plan.tile == kGradient64) {
        launch_gradient_ends<T, O, 64, 64, 2, 2>(p, loads, stores, units, st);
    } else if (plan.tile == kGradient128 || !loads || !stores || sizeof(T) == 4) {
        launch_gradient_ends<T, O, 128, 128, 2, 2>(p, loads, stores, units, st);
    } else if constexpr (sizeof(T) == 2) {
        launch_gradient<T, O, 256, 256, 4, 2, true, true>(p, units, st);
    }
    if (p.slots > 0) {   // (more than `most` rows in all: some group may be long)
        const int64_t size = (int64_t)p.in * p.out, groups = p.rows / p.most;
        // few elements: one a lane, so that there are workgroups for all units (50 x 129, 400 parts: 18 us; four a lane 186, one part after
        // the other); many: four (256 x 128 in 128 groups: 12 us, 61 with one)
        if (size < 16384) hipLaunchKernelGGL((k_grouped_parts<O, 1>), grid_of(groups * tiles_of(size, 256)), dim3(256), 0, st, p);
        else hipLaunchKernelGGL((k_grouped_parts<O, 4>), grid_of(groups * tiles_of(size, 1024)), dim3(256), 0, st, p);
    }
}

}  // namespace nomad_grouped
