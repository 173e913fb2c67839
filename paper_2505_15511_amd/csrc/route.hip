// libnomad: the router of a learned map and the weighted sum over experts behind the C ABI of include/nomad.h (host side).
#include <hip/hip_runtime.h>

#include "device_scope.h"
#include "host_util.h"
#include "nomad.h"
#include "route_kernels.h"

using namespace nomad_router;

namespace {

bool is_dtype(int32_t dtype) { return dtype == NOMAD_F32 || dtype == NOMAD_BF16 || dtype == NOMAD_F16; }
int64_t size_of(int32_t dtype) { return dtype == NOMAD_F32 ? 4 : 2; }
bool by(const void* p, int64_t stride, int64_t size, int64_t bytes) { return ((uintptr_t)p | (uintptr_t)(stride * size)) % (uintptr_t)bytes == 0; }

// Rows a chunk of the counts: their scan walks the chunks of an expert, so there are about a thousand at most, and no fewer rows
// in one than keep the counts well below the logits
int64_t chunk_rows(int64_t n) { return std::max<int64_t>(256, (n + 1023) / 1024); }
// One workgroup does it all where the logits are few (a row of 256: 4.4 us, the three kernels of the other form 12.4; 100 rows of 50: 6.4 against 40)
// and its counters and slots fit the 64 KB of LDS that a launch has without asking
bool is_small(int64_t n, int32_t n_experts, int32_t k) { return n * n_experts <= 32768 && n <= 1024 && n_experts + n * k <= 16384; }

template <typename T, int LANES, int K>
void launch_pick(const RouteArgs& p, bool vec, hipStream_t st) {
    const dim3 grid((uint32_t)p.n_chunks), block(kPickThreads);
    const size_t lds = sizeof(int32_t) * (size_t)p.n_experts;
    if (vec) hipLaunchKernelGGL((k_route_pick<T, LANES, K, true>), grid, block, lds, st, p);
    else hipLaunchKernelGGL((k_route_pick<T, LANES, K, false>), grid, block, lds, st, p);
}
template <typename T, int LANES, int K>
void launch_small(const RouteArgs& p, bool vec, hipStream_t st) {
    const size_t lds = sizeof(int32_t) * (size_t)(p.n_experts + p.n * p.k);
    if (vec) hipLaunchKernelGGL((k_route_small<T, LANES, K, true>), dim3(1), dim3(kSmallThreads), lds, st, p);
    else hipLaunchKernelGGL((k_route_small<T, LANES, K, false>), dim3(1), dim3(kSmallThreads), lds, st, p);
}
template <typename T, int K>
void launch_route(const RouteArgs& p, bool vec, hipStream_t st) {
    if (is_small(p.n, p.n_experts, p.k)) {
        // few rows: a wavefront each; more: four a wavefront, as long as a row is a few loads of 16 lanes
        if (p.n <= kSmallThreads / 64 || p.n_experts > 512) launch_small<T, 64, K>(p, vec, st);
        else launch_small<T, 16, K>(p, vec, st);
        return;
    }
    // 16 lanes a row as long as each reads it in a few loads: the row's best are found in four exchanges, not six, four rows at once
    // (a million rows of 256: 224 us, 486 with 64 lanes; whole calls on 262,144 rows of 64, 256, 512 and 1,024 in float32: 55, 78, 137 and 237 us
    // with 16 lanes, 146, 154, 186 and 252 with 64; of 2,048, 434 and 463: the line could lie higher)
    if (p.n_experts <= 512) launch_pick<T, 16, K>(p, vec, st);
    else launch_pick<T, 64, K>(p, vec, st);
    hipLaunchKernelGGL(k_route_scan, dim3(blocks_of(p.n_experts, kScanColumns)), dim3(kScanThreads), 0, st, p);
    // (four wavefronts' counters of 2,048 experts are 32 KB of LDS; two million slots: 28 us, 44 with one wavefront a chunk; whole calls on 65,536
    // rows of 1,024 and 2,048: 178 and 282 us, 183 and 287 with one)
    if (p.n_experts <= 2048) hipLaunchKernelGGL(k_route_place<4>, dim3((uint32_t)p.n_chunks), dim3(256), sizeof(int32_t) * 4 * (size_t)p.n_experts, st, p);
    else hipLaunchKernelGGL(k_route_place<1>, dim3((uint32_t)p.n_chunks), dim3(64), sizeof(int32_t) * (size_t)p.n_experts, st, p);
}
template <typename T>
void launch_route_k(const RouteArgs& p, bool vec, hipStream_t st) {
    if (p.k == 1) launch_route<T, 1>(p, vec, st);
    else if (p.k == 2) launch_route<T, 2>(p, vec, st);
    else if (p.k <= 4) launch_route<T, 4>(p, vec, st);
    else launch_route<T, 8>(p, vec, st);
}

template <typename T, int K>
void launch_route_gradient(const RouteGradientArgs& p, bool vec, hipStream_t st) {
    // (a million rows of 256: 187 us, 304 with 64 lanes a row: a wavefront then waits for one row's experts and weights, not for four; 262,144 rows
    // of 64, 256, 512 and 1,024 in float32: 19, 55, 107 and 202 us with 16 lanes, 37, 47, 101 and 201 with 64; with weights over all experts 44, 121,
    // 285 and 670 with 16, 131, 162, 275 and 486 with 64)
    if (p.n_experts <= 512) {
        const dim3 grid = grid_of((p.n + 15) / 16);
        if (vec) hipLaunchKernelGGL((k_route_gradient<T, 16, K, true>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((k_route_gradient<T, 16, K, false>), grid, dim3(256), 0, st, p);
    } else {
        const dim3 grid = grid_of((p.n + 3) / 4);
        if (vec) hipLaunchKernelGGL((k_route_gradient<T, 64, K, true>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((k_route_gradient<T, 64, K, false>), grid, dim3(256), 0, st, p);
    }
}
template <typename T>
void launch_route_gradient_k(const RouteGradientArgs& p, bool vec, hipStream_t st) {
    if (p.k == 1) launch_route_gradient<T, 1>(p, vec, st);
    else if (p.k == 2) launch_route_gradient<T, 2>(p, vec, st);
    else if (p.k <= 4) launch_route_gradient<T, 4>(p, vec, st);
    else launch_route_gradient<T, 8>(p, vec, st);
}

template <typename T, int VEC, int LANES>
void launch_combine(const CombineArgs& p, hipStream_t st) {
    const dim3 grid = grid_of((p.n + 256 / LANES - 1) / (256 / LANES));
    if (p.dy) hipLaunchKernelGGL((k_combine_gradient<T, LANES, VEC>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((k_combine<T, LANES, VEC>), grid, dim3(256), 0, st, p);
}
template <typename T, int VEC>
void launch_combine_lanes(const CombineArgs& p, hipStream_t st) {
    const int32_t pieces = (p.d + VEC - 1) / VEC;
    if (pieces <= 1) launch_combine<T, VEC, 1>(p, st);
    else if (pieces <= 4) launch_combine<T, VEC, 4>(p, st);
    else if (pieces <= 16) launch_combine<T, VEC, 16>(p, st);
    else launch_combine<T, VEC, 64>(p, st);
}
template <typename T>
void launch_combine_vec(const CombineArgs& p, bool vec, hipStream_t st) {
    if (vec) launch_combine_lanes<T, 16 / (int)sizeof(T)>(p, st);
    else launch_combine_lanes<T, 1>(p, st);
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" int64_t nomad_route_workspace(int64_t n, int32_t n_experts, int32_t k) {
    if (n <= 0 || n_experts < 1 || k < 1 || n > NOMAD_MAX_ROWS || n_experts > kMaxExperts || is_small(n, n_experts, k)) return 0;
    return ((n + chunk_rows(n) - 1) / chunk_rows(n) + 1) * n_experts * (int64_t)sizeof(int32_t);
}

extern "C" int nomad_route(const void* logits, int32_t dtype, int64_t n, int64_t stride, int32_t n_experts, int32_t k, int32_t normalize, int32_t* experts,
                           float* weights, int32_t* offsets, int32_t* order, int32_t* slots, void* workspace, int64_t workspace_bytes, int32_t device,
                           void* stream) {
    if (!is_dtype(dtype) || n < 0 || stride < 0 || n_experts < 1 || k < 1 || k > kMaxK || k > n_experts || (normalize != 0 && normalize != 1) || device < 0)
        return NOMAD_E_INVALID_ARG;
    if (n_experts > kMaxExperts || n > NOMAD_MAX_ROWS / k) return NOMAD_E_TOO_LARGE;
    if (!offsets || (n > 0 && (!logits || !experts || !weights || !order || !slots))) return NOMAD_E_INVALID_ARG;
    const int64_t need = nomad_route_workspace(n, n_experts, k);
    if (need > 0 && (!workspace || workspace_bytes < need)) return NOMAD_E_INVALID_ARG;
    const DeviceScope on(device);
    if (!on.ok()) return NOMAD_E_HIP;
    hipStream_t st = (hipStream_t)stream;
    RouteArgs p{};
    p.logits = logits;
    p.n = n;
    p.stride = stride;
    p.n_experts = n_experts;
    p.k = k;
    p.normalize = normalize;
    p.experts = experts;
    p.weights = weights;
    p.offsets = offsets;
    p.order = order;
    p.slots = slots;
    p.chunk = (int32_t)chunk_rows(n);
    p.n_chunks = (int32_t)((n + p.chunk - 1) / p.chunk);
    p.counts = (int32_t*)workspace;
    p.totals = (int32_t*)workspace + (int64_t)p.n_chunks * n_experts;
    const int64_t size = size_of(dtype);
    const bool vec = by(logits, stride, size, 16) && n_experts % (16 / size) == 0;
    if (dtype == NOMAD_F32) launch_route_k<float>(p, vec, st);
    else if (dtype == NOMAD_BF16) launch_route_k<__bf16>(p, vec, st);
    else launch_route_k<_Float16>(p, vec, st);
    KTRY(hipGetLastError());
    return NOMAD_OK;
}

extern "C" int nomad_route_gradient(const void* logits, int32_t dtype, int64_t n, int64_t stride, int32_t n_experts, int32_t k, int32_t normalize,
                                    const int32_t* experts, const float* weights, const float* dweights, void* dlogits, int32_t device, void* stream) {
    if (!is_dtype(dtype) || n < 0 || stride < 0 || n_experts < 1 || k < 1 || k > kMaxK || k > n_experts || (normalize != 0 && normalize != 1) || device < 0)
        return NOMAD_E_INVALID_ARG;
    if (n_experts > kMaxExperts || n > NOMAD_MAX_ROWS / k) return NOMAD_E_TOO_LARGE;
    if (n == 0) return NOMAD_OK;
    if ((!normalize && !logits) || !experts || !weights || !dweights || !dlogits) return NOMAD_E_INVALID_ARG;
    const DeviceScope on(device);
    if (!on.ok()) return NOMAD_E_HIP;
    const RouteGradientArgs p{logits, n, stride, n_experts, k, normalize, experts, weights, dweights, dlogits};
    const int64_t size = size_of(dtype);
    const bool vec = (normalize || by(logits, stride, size, 16)) && by(dlogits, n_experts, size, 16);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == NOMAD_F32) launch_route_gradient_k<float>(p, vec, st);
    else if (dtype == NOMAD_BF16) launch_route_gradient_k<__bf16>(p, vec, st);
    else launch_route_gradient_k<_Float16>(p, vec, st);
    KTRY(hipGetLastError());
    return NOMAD_OK;
}

extern "C" int nomad_combine(const void* values, int32_t dtype, int64_t n_values, int64_t values_stride, int32_t d, const int32_t* slots, const float* weights,
                             int64_t n, int32_t k, void* y, int32_t device, void* stream) {
    if (!is_dtype(dtype) || n < 0 || n_values < 0 || k < 1 || d < 1 || device < 0 || (n_values > 1 && values_stride < 0)) return NOMAD_E_INVALID_ARG;
    if (n > NOMAD_MAX_ROWS / k || n_values > NOMAD_MAX_ROWS || d > NOMAD_MAX_COLUMNS) return NOMAD_E_TOO_LARGE;
    if (n == 0) return NOMAD_OK;
    if ((n_values > 0 && !values) || !slots || !y) return NOMAD_E_INVALID_ARG;
    const DeviceScope on(device);
    if (!on.ok()) return NOMAD_E_HIP;
    CombineArgs p{};
    p.values = values;
    p.values_stride = values_stride;
    p.n_values = n_values;
    p.slots = slots;
    p.weights = weights;
    p.n = n;
    p.k = k;
    p.d = d;
    p.y = y;
    const int64_t size = size_of(dtype);
    const bool vec = by(values, values_stride, size, 16) && by(y, d, size, 16);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == NOMAD_F32) launch_combine_vec<float>(p, vec, st);
    else if (dtype == NOMAD_BF16) launch_combine_vec<__bf16>(p, vec, st);
    else launch_combine_vec<_Float16>(p, vec, st);
    KTRY(hipGetLastError());
    return NOMAD_OK;
}

extern "C" int nomad_combine_gradient(const void* dy, int32_t dtype, int64_t dy_stride, const void* values, int64_t n_values, int64_t values_stride, int32_t d,
                                      const int32_t* slots, const int32_t* order, const float* weights, int64_t n, int32_t k, void* dvalues, float* dweights,
                                      int32_t device, void* stream) {
    if (!is_dtype(dtype) || n < 0 || n_values < 0 || k < 1 || d < 1 || device < 0 || dy_stride < 0 || values_stride < 0) return NOMAD_E_INVALID_ARG;
    if (n > NOMAD_MAX_ROWS / k || n_values > NOMAD_MAX_ROWS || d > NOMAD_MAX_COLUMNS) return NOMAD_E_TOO_LARGE;
    if (order && n_values != n * k) return NOMAD_E_INVALID_ARG;
    if (n == 0) return NOMAD_OK;
    if (!dy || !slots || (dweights && n_values > 0 && !values) || (!dvalues && !dweights)) return NOMAD_E_INVALID_ARG;
    const DeviceScope on(device);
    if (!on.ok()) return NOMAD_E_HIP;
    CombineArgs p{};
    p.values = values;
    p.values_stride = values_stride;
    p.n_values = n_values;
    p.slots = slots;
    p.weights = weights;
    p.n = n;
    p.k = k;
    p.d = d;
    p.dy = dy;
    p.dy_stride = dy_stride;
    p.order = order;
    p.dvalues = dvalues;
    p.dweights = dweights;
    const int64_t size = size_of(dtype);
    const bool vec = by(dy, dy_stride, size, 16) && (!dweights || by(values, values_stride, size, 16)) && (!dvalues || by(dvalues, d, size, 16)) && d % (16 / size) == 0;
    hipStream_t st = (hipStream_t)stream;
    if (dtype == NOMAD_F32) launch_combine_vec<float>(p, vec, st);
    else if (dtype == NOMAD_BF16) launch_combine_vec<__bf16>(p, vec, st);
    else launch_combine_vec<_Float16>(p, vec, st);
    KTRY(hipGetLastError());
    return NOMAD_OK;
}
#pragma GCC visibility pop
