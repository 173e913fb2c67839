// Launches of the dense products for one element type (each type has a source file of its own: they compile side by side).
#pragma once
#include "dense_kernels.h"
#include "dense_plan.h"
#include "grouped_launch.h"

namespace nomad_dense {

// Operands by where k is contiguous: both (rows of W and x), b alone (W turned), neither (columns of x and dz)
enum Turn { kForward = 0, kTurned = 1, kWeights = 2 };

struct Launch {
    Turn turn;
    Plan plan;
    bool wide;             // results in float32 of 16-bit operands
    bool loads, stores;    // rows of whole 16-byte chunks where they are read, where they are written
    int units;
};

void dense_f32(const DenseArgs& p, const Launch& l, hipStream_t st);
void dense_bf16(const DenseArgs& p, const Launch& l, hipStream_t st);
void dense_f16(const DenseArgs& p, const Launch& l, hipStream_t st);
void slope_f32(const SlopeArgs& p, int64_t parts, bool vec, hipStream_t st);
void slope_bf16(const SlopeArgs& p, int64_t parts, bool vec, hipStream_t st);
void slope_f16(const SlopeArgs& p, int64_t parts, bool vec, hipStream_t st);

inline void launch_sums(const float* part, int32_t parts, int64_t rows, float* to, hipStream_t st) {
    hipLaunchKernelGGL(k_dense_sums, dim3(blocks_of(rows, kSumColumns)), dim3(256), 0, st, part, parts, rows, to);
}

template <typename T, int TA, int TB, int WA, int WB, bool A_KC, bool B_KC, bool LOADS, bool STORES>
void launch_dense(const DenseArgs& p, const Launch& l, hipStream_t st) {
    const int64_t total = tiles_of(p.columns, TA) * tiles_of(p.rows, TB) * p.parts, at_once = (int64_t)l.units * nomad_grouped::resident<TA, TB, WA * WB>();
    hipLaunchKernelGGL((k_dense<T, TA, TB, WA, WB, A_KC, B_KC, LOADS, STORES>), dim3((uint32_t)std::min(total, at_once)), dim3(64 * WA * WB), 0, st, p);
}
template <typename T, int TA, int TB, int WA, int WB, bool A_KC, bool B_KC>
void launch_ends(const DenseArgs& p, const Launch& l, hipStream_t st) {
    if (l.loads && l.stores) launch_dense<T, TA, TB, WA, WB, A_KC, B_KC, true, true>(p, l, st);
    else if (l.stores) launch_dense<T, TA, TB, WA, WB, A_KC, B_KC, false, true>(p, l, st);
    else launch_dense<T, TA, TB, WA, WB, A_KC, B_KC, false, false>(p, l, st);
}
template <typename T, bool A_KC, bool B_KC>
void launch_tile(const DenseArgs& p, const Launch& l, hipStream_t st) {
    switch (l.plan.tile) {
        case k16: launch_ends<T, 16, 256, 1, 4, A_KC, B_KC>(p, l, st); break;
        case k64: launch_ends<T, 64, 128, 2, 2, A_KC, B_KC>(p, l, st); break;
        case k256:
            if constexpr (sizeof(T) == 2) { launch_dense<T, 256, 256, 4, 2, A_KC, B_KC, true, true>(p, l, st); break; }
            [[fallthrough]];
        default: launch_ends<T, 128, 128, 2, 2, A_KC, B_KC>(p, l, st);
    }
}
template <typename T, typename O>
void launch_few(const DenseArgs& p, const Launch& l, hipStream_t st) {
    const dim3 grid((uint32_t)l.plan.units), block(64 * nomad_grouped::kFewWaves);
    if (p.rows <= 16) hipLaunchKernelGGL((k_dense_few<T, O, 1>), grid, block, 0, st, p);
    else if (p.rows <= 32) hipLaunchKernelGGL((k_dense_few<T, O, 2>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((k_dense_few<T, O, 4>), grid, block, 0, st, p);
}
template <typename T, typename O>
void launch_parts(const DenseArgs& p, hipStream_t st) {
    if (p.columns % 4 == 0 && p.part_stride % 4 == 0 && (uintptr_t)p.part % 16 == 0) hipLaunchKernelGGL((k_dense_parts<T, O, 4>), grid_of((p.rows * (p.columns / 4) + 255) / 256), dim3(256), 0, st, p);
    else hipLaunchKernelGGL((k_dense_parts<T, O, 1>), grid_of((p.rows * p.columns + 255) / 256), dim3(256), 0, st, p);
}
template <typename T>
void launch_type(const DenseArgs& p, const Launch& l, hipStream_t st) {
    if (l.plan.tile == kFew) {
        if (l.wide) launch_few<T, float>(p, l, st);
        else launch_few<T, T>(p, l, st);
    } else if (l.turn == kForward) launch_tile<T, true, true>(p, l, st);
    else if (l.turn == kTurned) launch_tile<T, false, true>(p, l, st);
    else launch_tile<T, false, false>(p, l, st);
    // (results of one part that are where they belong: nothing is left to do)
    const Finish& f = p.f;
    const bool done = !p.part || (p.parts == 1 && (const void*)p.part == f.y && !f.bias && !f.residual && !f.slope_at && !f.z_out && f.activation == nomad_grouped::kNone && f.factor == 1.f);
    if (!done) {
        if (l.wide) launch_parts<T, float>(p, st);
        else launch_parts<T, T>(p, st);
    }
}
template <typename T>
void launch_slope(SlopeArgs p, int64_t parts, bool vec, hipStream_t st) {
    constexpr int n = 16 / (int)sizeof(T);
    const int32_t pieces = vec ? p.columns / n : p.columns;
    p.wide = 1;
    while (p.wide < pieces && p.wide < 256) p.wide *= 2;
    const dim3 grid((uint32_t)(tiles_of(pieces, p.wide) * parts));
    if (vec) hipLaunchKernelGGL((k_dense_slope<T, n>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((k_dense_slope<T, 1>), grid, dim3(256), 0, st, p);
}

}  // namespace nomad_dense
