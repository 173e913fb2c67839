// libnomad: the gradients' norm and the factor that clips a step, behind the C ABI of include/nomad.h (host side).
#include <hip/hip_runtime.h>

#include "device_scope.h"
#include "host_util.h"
#include "nomad.h"
#include "norm_kernels.h"

using namespace nomad_norm;

#pragma GCC visibility push(default)
extern "C" int64_t nomad_gradient_norm_workspace(int32_t count) { return count < 0 ? 0 : (kRuns + count) * (int64_t)sizeof(double); }

extern "C" int nomad_gradient_norm(const nomad_gradient* tensors, int32_t count, double max_norm, const float* grad_scale, float* norm, float* scale,
                                   void* workspace, int64_t workspace_bytes, int32_t device, void* stream) {
    if (count < 0 || (count > 0 && !tensors) || !(max_norm >= 0.0) || !norm || device < 0) return NOMAD_E_INVALID_ARG;
    constexpr int64_t most = (int64_t)1 << 50;
    int64_t total = 0;
    for (int32_t i = 0; i < count; ++i) {
        const nomad_gradient& t = tensors[i];
        if (t.n < 0 || (t.n > 0 && !t.g) || (t.dtype != NOMAD_F32 && t.dtype != NOMAD_BF16 && t.dtype != NOMAD_F16)) return NOMAD_E_INVALID_ARG;
        if ((uintptr_t)t.g % (t.dtype == NOMAD_F32 ? 4 : 2)) return NOMAD_E_INVALID_ARG;
        if (t.n > most || (total += t.n) > most) return NOMAD_E_TOO_LARGE;
    }
    if (!workspace || workspace_bytes < nomad_gradient_norm_workspace(count) || (uintptr_t)workspace % sizeof(double)) return NOMAD_E_INVALID_ARG;
    const DeviceScope on(device);
    if (!on.ok()) return NOMAD_E_HIP;
    hipStream_t st = (hipStream_t)stream;
    Batch b;
    b.run = std::max<int64_t>(1, (total + kRuns * kRun - 1) / (kRuns * kRun)) * kRun;
    b.part = (double*)workspace;
    b.count = 0;
    b.first[0] = 0;
    int64_t runs = 0;
    const auto flush = [&]() {
        if (b.count > 0) hipLaunchKernelGGL(k_norm_runs, dim3(b.first[b.count]), dim3(kThreads), 0, st, b);
        runs += b.first[b.count];
        b.part = (double*)workspace + runs;
        b.count = 0;
    };
    for (int32_t i = 0; i < count; ++i) {
        const nomad_gradient& t = tensors[i];
        if (t.n == 0) continue;
        if (b.count == kTensors) flush();
        b.t[b.count] = {t.g, t.n << 2 | t.dtype};
        b.first[b.count + 1] = b.first[b.count] + (uint32_t)((t.n + b.run - 1) / b.run);
        ++b.count;
    }
    flush();
    hipLaunchKernelGGL(k_norm_sum, dim3(1), dim3(kSumThreads), 0, st, (const double*)workspace, runs, grad_scale, max_norm, norm, scale);
    KTRY(hipGetLastError());
    return NOMAD_OK;
}
#pragma GCC visibility pop
