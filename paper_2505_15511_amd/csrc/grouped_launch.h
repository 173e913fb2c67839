// Launches of the grouped products for one element type (each type has a source file of its own: they compile side by side).
#pragma once
#include "grouped_kernels.h"
#include "grouped_plan.h"
#include "host_util.h"

namespace nomad_grouped {

// fast: whole 16-byte chunks on every side
void product_f32(const ProductArgs& p, ProductTile tile, bool wide, bool w_kc, bool fast, int units, hipStream_t st);
void product_bf16(const ProductArgs& p, ProductTile tile, bool wide, bool w_kc, bool fast, int units, hipStream_t st);
void product_f16(const ProductArgs& p, ProductTile tile, bool wide, bool w_kc, bool fast, int units, hipStream_t st);
void gradient_f32(const GradientArgs& p, const GradientPlan& plan, bool wide, bool fast, int units, hipStream_t st);
void gradient_bf16(const GradientArgs& p, const GradientPlan& plan, bool wide, bool fast, int units, hipStream_t st);
void gradient_f16(const GradientArgs& p, const GradientPlan& plan, bool wide, bool fast, int units, hipStream_t st);

// workgroups a compute unit holds at a time: what fits its 160 KB of LDS and eight wavefronts (the kernels take up to 256 registers)
template <int TA, int TB, int WAVES>
constexpr int resident() { return std::max(1, std::min(163840 / (2 * (TA + TB) * kStepBytes), 8 / WAVES)); }

template <typename T, typename O, int TA, int TB, int WA, int WB, bool W_KC, bool FAST>
void launch_product(const ProductArgs& p, int units, hipStream_t st) {
    const int64_t rows = std::min<int64_t>(p.rows, p.rows / TB + p.n_groups + 1);   // tiles of them: no more than one a row, one a group beyond the whole ones
    const int64_t total = rows * tiles_of(p.out, TA), at_once = (int64_t)units * resident<TA, TB, WA * WB>();
    hipLaunchKernelGGL((k_grouped_product<T, O, TA, TB, WA, WB, W_KC, FAST>), dim3((uint32_t)std::min(total, at_once)), dim3(64 * WA * WB), 0, st, p);
}
template <typename T, typename O, bool W_KC>
void launch_product_tile(const ProductArgs& p, ProductTile tile, bool fast, int units, hipStream_t st) {
    if (tile == kProduct16) {
        if (fast) launch_product<T, O, 16, 256, 1, 4, W_KC, true>(p, units, st);
        else launch_product<T, O, 16, 256, 1, 4, W_KC, false>(p, units, st);
    } else if (!fast) {
        launch_product<T, O, 128, 128, 2, 2, W_KC, false>(p, units, st);
    } else if (tile == kProduct64) {
        launch_product<T, O, 64, 128, 2, 2, W_KC, true>(p, units, st);
    } else if (tile == kProduct128 || sizeof(T) == 4) {
        launch_product<T, O, 128, 128, 2, 2, W_KC, true>(p, units, st);
    } else if constexpr (sizeof(T) == 2) {
        launch_product<T, O, 256, 256, 4, 2, W_KC, true>(p, units, st);
    }
}
template <typename T, typename O>
void launch_product_type(const ProductArgs& p, ProductTile tile, bool w_kc, bool fast, int units, hipStream_t st) {
    if (w_kc) launch_product_tile<T, O, true>(p, tile, fast, units, st);
    else launch_product_tile<T, O, false>(p, tile, fast, units, st);
}

template <typename T, typename O, int TA, int TB, int WA, int WB, bool FAST>
void launch_gradient(const GradientArgs& p, int units, hipStream_t st) {
    const int64_t total = tiles_of(p.in, TA) * tiles_of(p.out, TB) * (p.n_groups + p.rows / p.most);   // (a group has one part and one more for every `most` rows at most)
    const int64_t at_once = (int64_t)units * resident<TA, TB, WA * WB>();
    hipLaunchKernelGGL((k_grouped_gradient<T, O, TA, TB, WA, WB, FAST>), dim3((uint32_t)std::min(total, at_once)), dim3(64 * WA * WB), 0, st, p);
}
template <typename T, typename O>
void launch_gradient_type(const GradientArgs& p, const GradientPlan& plan, bool fast, int units, hipStream_t st) {
    if (plan.tile == kGradient16) {
        if (fast) launch_gradient<T, O, 128, 16, 4, 1, true>(p, units, st);
        else launch_gradient<T, O, 128, 16, 4, 1, false>(p, units, st);
    } else if (!fast) {
        launch_gradient<T, O, 128, 128, 2, 2, false>(p, units, st);
    } else if (plan.tile == kGradient128 || sizeof(T) == 4) {
        launch_gradient<T, O, 128, 128, 2, 2, true>(p, units, st);
    } else if constexpr (sizeof(T) == 2) {
        launch_gradient<T, O, 256, 256, 4, 2, true>(p, units, st);
    }
    if (p.slots > 0)   // (more than `most` rows in all: some group may be long)
        hipLaunchKernelGGL((k_grouped_parts<O>), grid_of(p.rows / p.most * tiles_of((int64_t)p.in * p.out, kPiece)), dim3(256), 0, st, p);
}

}  // namespace nomad_grouped
