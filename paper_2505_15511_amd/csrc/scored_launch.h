// Launches of routing by scores for one element type (each type has a source file of its own: they compile side by side).
#pragma once
#include "route_launch.h"
#include "scored_kernels.h"

namespace nomad_router {

void scored_f32(const ScoredArgs& p, bool vec, hipStream_t st);
void scored_bf16(const ScoredArgs& p, bool vec, hipStream_t st);
void scored_f16(const ScoredArgs& p, bool vec, hipStream_t st);
void scored_gradient_f32(const ScoredGradientArgs& p, bool vec, hipStream_t st);
void scored_gradient_bf16(const ScoredGradientArgs& p, bool vec, hipStream_t st);
void scored_gradient_f16(const ScoredGradientArgs& p, bool vec, hipStream_t st);

// lanes of a team where as many teams as there are groups (a power of two, at most all lanes) share the lanes of a row
inline int32_t team_of(int32_t groups, int32_t lanes) {
    int32_t teams = 1;
    while (teams < groups && teams < lanes) teams *= 2;
    return lanes / teams;
}
// experts a lane of sixteen holds, where every lane has those of one group
inline int32_t held_by_a_lane(const ScoredArgs& p, int32_t size, bool vec) {
    const int32_t epc = vec ? 16 / size : 1, team = team_of(p.groups, 16);
    return p.groups > 16 ? 1 << 30 : (p.size + team * epc - 1) / (team * epc) * epc;
}

template <typename T, int CAP, int K>
void launch_quick(const ScoredArgs& p, bool vec, hipStream_t st) {
    const dim3 grid((uint32_t)p.r.n_chunks), block(kQuickThreads);
    if (p.groups > 1 && vec) hipLaunchKernelGGL((k_scored_quick<T, CAP, K, true, true>), grid, block, 0, st, p);
    else if (p.groups > 1) hipLaunchKernelGGL((k_scored_quick<T, CAP, K, false, true>), grid, block, 0, st, p);
    else if (vec) hipLaunchKernelGGL((k_scored_quick<T, CAP, K, true, false>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((k_scored_quick<T, CAP, K, false, false>), grid, block, 0, st, p);
    if (!p.bias && sizeof(T) == 2 && (p.groups == 1 || p.best == 1)) return;   // (logits of 16 bits, which keys hold whole)
    ScoredArgs rest = p;
    rest.team = team_of(p.groups, 64);
    rest.open_team = team_of(p.top_groups, 64);
    hipLaunchKernelGGL((k_scored_rest<T>), grid, dim3(kRestThreads), 0, st, rest);
}
template <typename T>
void launch_scored(ScoredArgs p, bool vec, hipStream_t st) {
    const int32_t held = held_by_a_lane(p, (int32_t)sizeof(T), vec);
    // (the line of nomad_route. One workgroup and several kernels, us: 1, 16, 64 and 128 rows of 256 in bfloat16, k = 8 of groups, 14, 20, 36, 63 and 19, 19, 27, 27; in
    // float32, k = 2, 9, 12, 19, 32 and 15, 15, 18, 19; 1 and 32 rows of 1,024 17, 34 and 27, 89: for up to 256 experts it could lie at some 16 rows)
    const bool small = is_small(p.r.n, p.r.n_experts, p.r.k), quick = !small && held <= 16;
    const int32_t lanes = quick || (small && p.r.n > kSmallThreads / 64 && p.r.n_experts <= 512) ? 16 : 64;
    p.team = team_of(p.groups, lanes);
    p.open_team = team_of(p.top_groups, lanes);
    if (small) {
        const size_t lds = sizeof(int32_t) * (size_t)(p.r.n_experts + p.r.n * p.r.k);
        if (lanes == 16) hipLaunchKernelGGL((k_scored_small<T, 16, 8, false>), dim3(1), dim3(kSmallThreads), lds, st, p);
        else hipLaunchKernelGGL((k_scored_small<T, 64, 8, false>), dim3(1), dim3(kSmallThreads), lds, st, p);
        return;
    }
    if (quick) {
        if (held <= 8 && p.r.k <= 2) launch_quick<T, 8, 2>(p, vec, st);
        else if (held <= 8) launch_quick<T, 8, 8>(p, vec, st);
        else if (p.r.k <= 2) launch_quick<T, 16, 2>(p, vec, st);
        else launch_quick<T, 16, 8>(p, vec, st);
    } else {
        const dim3 grid((uint32_t)p.r.n_chunks), block(kPickThreads);
        const size_t lds = sizeof(int32_t) * (size_t)p.r.n_experts;
        if (vec) hipLaunchKernelGGL((k_scored_pick<T, 64, 8, true>), grid, block, lds, st, p);
        else hipLaunchKernelGGL((k_scored_pick<T, 64, 8, false>), grid, block, lds, st, p);
    }
    launch_places(p.r, st);
}

template <typename T, int K, int LANES>
void launch_scored_gradient(const ScoredGradientArgs& p, bool vec, hipStream_t st) {
    const dim3 grid = grid_of((p.r.n + 256 / LANES - 1) / (256 / LANES));
    if (vec) hipLaunchKernelGGL((k_scored_gradient<T, LANES, K, true>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((k_scored_gradient<T, LANES, K, false>), grid, dim3(256), 0, st, p);
}
template <typename T>
void launch_scored_gradient_type(const ScoredGradientArgs& p, bool vec, hipStream_t st) {
    if (p.r.n_experts <= 512 && (p.sigmoid || p.r.normalize)) {
        const dim3 grid = grid_of((p.r.n + 15) / 16);
        const size_t lds = 16 * (((size_t)p.r.n_experts * sizeof(T) + 15) / 16 * 16);
        if (vec) hipLaunchKernelGGL((k_scored_gradient_rows<T, true>), grid, dim3(256), lds, st, p);
        else hipLaunchKernelGGL((k_scored_gradient_rows<T, false>), grid, dim3(256), lds, st, p);
    } else if (p.r.n_experts <= 512) launch_scored_gradient<T, 8, 16>(p, vec, st);
    else launch_scored_gradient<T, 8, 64>(p, vec, st);
}

}  // namespace nomad_router
