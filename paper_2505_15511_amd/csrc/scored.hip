// libnomad: routing by scores behind the C ABI of include/nomad.h (host side).
#include <hip/hip_runtime.h>

#include <cmath>

#include "device_scope.h"
#include "route_launch.h"
#include "scored_kernels.h"

using namespace nomad_router;

namespace {

// lanes of a team where as many teams as there are groups (a power of two, at most all lanes) share the lanes of a row
int32_t team_of(int32_t groups, int32_t lanes) {
    int32_t teams = 1;
    while (teams < groups && teams < lanes) teams *= 2;
    return lanes / teams;
}

template <typename T, int LANES, int K>
void launch_pick(ScoredArgs p, bool small, bool vec, hipStream_t st) {
    p.team = team_of(p.groups, LANES);
    p.open_team = team_of(p.top_groups, LANES);
    if (small) {
        const size_t lds = sizeof(int32_t) * (size_t)(p.r.n_experts + p.r.n * p.r.k);
        if (vec) hipLaunchKernelGGL((k_scored_small<T, LANES, K, true>), dim3(1), dim3(kSmallThreads), lds, st, p);
        else hipLaunchKernelGGL((k_scored_small<T, LANES, K, false>), dim3(1), dim3(kSmallThreads), lds, st, p);
        return;
    }
    const dim3 grid((uint32_t)p.r.n_chunks), block(kPickThreads);
    const size_t lds = sizeof(int32_t) * (size_t)p.r.n_experts;
    if (vec) hipLaunchKernelGGL((k_scored_pick<T, LANES, K, true>), grid, block, lds, st, p);
    else hipLaunchKernelGGL((k_scored_pick<T, LANES, K, false>), grid, block, lds, st, p);
    launch_places(p.r, st);
}
template <typename T, int K>
void launch_scored(const ScoredArgs& p, bool vec, hipStream_t st) {
    const bool small = is_small(p.r.n, p.r.n_experts, p.r.k);
    // as in nomad_route
    const bool wide = p.r.n_experts > 512 || (small && p.r.n <= kSmallThreads / 64);
    if (wide) launch_pick<T, 64, K>(p, small, vec, st);
    else launch_pick<T, 16, K>(p, small, vec, st);
}
template <typename T>
void launch_scored_k(const ScoredArgs& p, bool vec, hipStream_t st) {
    if (p.r.k == 1) launch_scored<T, 1>(p, vec, st);
    else if (p.r.k == 2) launch_scored<T, 2>(p, vec, st);
    else if (p.r.k <= 4) launch_scored<T, 4>(p, vec, st);
    else launch_scored<T, 8>(p, vec, st);
}

template <typename T, int K>
void launch_gradient(const ScoredGradientArgs& p, bool vec, hipStream_t st) {
    if (p.r.n_experts <= 512) {
        const dim3 grid = grid_of((p.r.n + 15) / 16);
        if (vec) hipLaunchKernelGGL((k_scored_gradient<T, 16, K, true>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((k_scored_gradient<T, 16, K, false>), grid, dim3(256), 0, st, p);
    } else {
        const dim3 grid = grid_of((p.r.n + 3) / 4);
        if (vec) hipLaunchKernelGGL((k_scored_gradient<T, 64, K, true>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((k_scored_gradient<T, 64, K, false>), grid, dim3(256), 0, st, p);
    }
}
template <typename T>
void launch_gradient_k(const ScoredGradientArgs& p, bool vec, hipStream_t st) {
    if (p.r.k == 1) launch_gradient<T, 1>(p, vec, st);
    else if (p.r.k == 2) launch_gradient<T, 2>(p, vec, st);
    else if (p.r.k <= 4) launch_gradient<T, 4>(p, vec, st);
    else launch_gradient<T, 8>(p, vec, st);
}

bool is_scoring(const nomad_scoring* s, int32_t n_experts, int32_t k) {
    if (!s || s->struct_size != sizeof(nomad_scoring)) return false;
    if ((s->score != NOMAD_SCORE_SOFTMAX && s->score != NOMAD_SCORE_SIGMOID) || (s->normalize != 0 && s->normalize != 1)) return false;
    if (!std::isfinite(s->scale) || s->scale == 0.f) return false;
    if (s->groups < 1 || s->groups > NOMAD_ROUTE_MAX_GROUPS || n_experts % s->groups || s->top_groups < 1 || s->top_groups > s->groups) return false;
    return (s->group_best == 1 || s->group_best == 2) && k <= (int64_t)s->top_groups * (n_experts / s->groups);
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" int nomad_route_scored(const void* logits, int32_t dtype, int64_t n, int64_t stride, int32_t n_experts, int32_t k, const nomad_scoring* scoring,
                                  int32_t* experts, float* weights, int32_t* offsets, int32_t* order, int32_t* slots, void* workspace, int64_t workspace_bytes,
                                  int32_t device, void* stream) {
    if (!is_dtype(dtype) || n < 0 || stride < 0 || n_experts < 1 || k < 1 || k > kMaxK || k > n_experts || device < 0) return NOMAD_E_INVALID_ARG;
    if (n_experts > kMaxExperts || n > NOMAD_MAX_ROWS / k) return NOMAD_E_TOO_LARGE;
    if (!is_scoring(scoring, n_experts, k)) return NOMAD_E_INVALID_ARG;
    if (!offsets || (n > 0 && (!logits || !experts || !weights || !order || !slots))) return NOMAD_E_INVALID_ARG;
    const int64_t need = nomad_route_workspace(n, n_experts, k);
    if (need > 0 && (!workspace || workspace_bytes < need)) return NOMAD_E_INVALID_ARG;
    const DeviceScope on(device);
    if (!on.ok()) return NOMAD_E_HIP;
    hipStream_t st = (hipStream_t)stream;
    ScoredArgs p{};
    p.r.logits = logits;
    p.r.stride = stride;
    p.r.normalize = scoring->normalize;
    fill_places(p.r, n, n_experts, k, experts, weights, offsets, order, slots, workspace);
    p.bias = scoring->bias;
    p.scale = scoring->scale;
    p.sigmoid = scoring->score == NOMAD_SCORE_SIGMOID;
    p.top_groups = scoring->top_groups;
    p.groups = p.top_groups == scoring->groups ? 1 : scoring->groups;   // (all of them open: there is nothing to compare)
    if (p.groups == 1) p.top_groups = 1;
    p.best = scoring->group_best;
    p.size = n_experts / p.groups;
    const int64_t size = size_of(dtype);
    const bool vec = by(logits, stride, size, 16) && p.size % (16 / size) == 0;
    if (dtype == NOMAD_F32) launch_scored_k<float>(p, vec, st);
    else if (dtype == NOMAD_BF16) launch_scored_k<__bf16>(p, vec, st);
    else launch_scored_k<_Float16>(p, vec, st);
    KTRY(hipGetLastError());
    return NOMAD_OK;
}

extern "C" int nomad_route_scored_gradient(const void* logits, int32_t dtype, int64_t n, int64_t stride, int32_t n_experts, int32_t k, const nomad_scoring* scoring,
                                           const int32_t* experts, const float* weights, const float* dweights, void* dlogits, int32_t device, void* stream) {
    if (!is_dtype(dtype) || n < 0 || stride < 0 || n_experts < 1 || k < 1 || k > kMaxK || k > n_experts || device < 0) return NOMAD_E_INVALID_ARG;
    if (n_experts > kMaxExperts || n > NOMAD_MAX_ROWS / k) return NOMAD_E_TOO_LARGE;
    if (!is_scoring(scoring, n_experts, k)) return NOMAD_E_INVALID_ARG;
    if (n == 0) return NOMAD_OK;
    if (!logits || !experts || !weights || !dweights || !dlogits) return NOMAD_E_INVALID_ARG;
    const DeviceScope on(device);
    if (!on.ok()) return NOMAD_E_HIP;
    const bool over_all = scoring->score == NOMAD_SCORE_SOFTMAX && !scoring->normalize;   // (reads the logits)
    const ScoredGradientArgs p{{logits, n, stride, n_experts, k, scoring->normalize, experts, weights, dweights, dlogits},
                               scoring->scale, scoring->normalize ? 1.f / scoring->scale : 0.f, scoring->score == NOMAD_SCORE_SIGMOID};
    const int64_t size = size_of(dtype);
    const bool vec = (!over_all || by(logits, stride, size, 16)) && by(dlogits, n_experts, size, 16);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == NOMAD_F32) launch_gradient_k<float>(p, vec, st);
    else if (dtype == NOMAD_BF16) launch_gradient_k<__bf16>(p, vec, st);
    else launch_gradient_k<_Float16>(p, vec, st);
    KTRY(hipGetLastError());
    return NOMAD_OK;
}

extern "C" int nomad_balance_bias(const float* bias, const int32_t* offsets, int32_t n_experts, float rate, float* out, int32_t device, void* stream) {
    if (!bias || !offsets || !out || n_experts < 1 || !std::isfinite(rate) || device < 0) return NOMAD_E_INVALID_ARG;
    if (n_experts > kMaxExperts) return NOMAD_E_TOO_LARGE;
    const DeviceScope on(device);
    if (!on.ok()) return NOMAD_E_HIP;
    hipLaunchKernelGGL(k_balance_bias, dim3(blocks_of(n_experts, 256)), dim3(256), 0, (hipStream_t)stream, bias, offsets, n_experts, rate, out);
    KTRY(hipGetLastError());
    return NOMAD_OK;
}
#pragma GCC visibility pop
