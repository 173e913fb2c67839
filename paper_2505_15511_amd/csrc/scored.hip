// libnomad: routing by scores behind the C ABI of include/nomad.h (host side).
#include <hip/hip_runtime.h>

#include <cmath>

#include "device_scope.h"
#include "scored_launch.h"

using namespace nomad_router;

namespace {

bool is_scoring(const nomad_scoring* s, int32_t n_experts, int32_t k) {
    if (!s || s->struct_size != sizeof(nomad_scoring)) return false;
    if ((s->score != NOMAD_SCORE_SOFTMAX && s->score != NOMAD_SCORE_SIGMOID) || (s->normalize != 0 && s->normalize != 1)) return false;
    if (!std::isfinite(s->scale) || s->scale == 0.f || !std::isfinite(1.f / s->scale)) return false;
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
    if (dtype == NOMAD_F32) scored_f32(p, vec, st);
    else if (dtype == NOMAD_BF16) scored_bf16(p, vec, st);
    else scored_f16(p, vec, st);
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
                               scoring->scale, scoring->score == NOMAD_SCORE_SIGMOID};
    const int64_t size = size_of(dtype);
    const bool vec = (!over_all || by(logits, stride, size, 16)) && by(dlogits, n_experts, size, 16);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == NOMAD_F32) scored_gradient_f32(p, vec, st);
    else if (dtype == NOMAD_BF16) scored_gradient_bf16(p, vec, st);
    else scored_gradient_f16(p, vec, st);
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
