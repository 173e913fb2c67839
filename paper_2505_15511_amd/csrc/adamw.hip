// libnomad: AdamW over many tensors behind the C ABI of include/nomad.h (host side).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstddef>

#include "adamw_kernels.h"
#include "device_scope.h"
#include "host_util.h"
#include "nomad.h"

using namespace nomad_adamw;

namespace {

// launches, each with the addresses of up to kTensors tensors among its arguments
template <typename P, typename G>
void launch(const Batch& b, bool eight, bool dither, hipStream_t st) {
    const dim3 grid(b.first[b.count]), block(kThreads);
    if (eight && dither) hipLaunchKernelGGL((k_adamw<P, G, true, true>), grid, block, 0, st, b);
    else if (eight) hipLaunchKernelGGL((k_adamw<P, G, true, false>), grid, block, 0, st, b);
    else hipLaunchKernelGGL((k_adamw<P, G, false, false>), grid, block, 0, st, b);
}

int kind_of(int32_t p, int32_t g) {   // -1: no such step
    if (p == NOMAD_F32) return g == NOMAD_F32 ? 0 : g == NOMAD_BF16 ? 1 : g == NOMAD_F16 ? 2 : -1;
    if (p == NOMAD_BF16) return g == NOMAD_BF16 ? 3 : g == NOMAD_F32 ? 4 : -1;
    if (p == NOMAD_F16) return g == NOMAD_F16 ? 5 : g == NOMAD_F32 ? 6 : -1;
    return -1;
}

void launch_kind(int kind, const Batch& b, bool eight, bool dither, hipStream_t st) {
    switch (kind) {
        case 0: launch<float, float>(b, eight, dither, st); break;
        case 1: launch<float, __bf16>(b, eight, dither, st); break;
        case 2: launch<float, _Float16>(b, eight, dither, st); break;
        case 3: launch<__bf16, __bf16>(b, eight, dither, st); break;
        case 4: launch<__bf16, float>(b, eight, dither, st); break;
        case 5: launch<_Float16, _Float16>(b, eight, dither, st); break;
        default: launch<_Float16, float>(b, eight, dither, st); break;
    }
}

constexpr int64_t kMostBlocks = ((int64_t)1 << 24) - 1;     // of a launch: fewer than 2^32 lanes
constexpr int64_t kMostElements = kMostBlocks * kChunk;     // of a tensor: 3.4e10
int64_t chunks_of(int64_t n) { return (n + kChunk - 1) / kChunk; }

}  // namespace

#pragma GCC visibility push(default)
extern "C" int nomad_adamw_step(const nomad_adamw_tensor* tensors, int32_t count, const nomad_adamw_options* options) {
    constexpr size_t shorter = offsetof(nomad_adamw_options, dither);   // options without it: nearest codes
    if (!options || (options->struct_size != sizeof(nomad_adamw_options) && options->struct_size != shorter) || count < 0 || (count > 0 && !tensors)) return NOMAD_E_INVALID_ARG;
    const nomad_adamw_options& o = *options;
    const bool dither = o.struct_size != shorter && o.dither != 0;
    if ((dither && (o.dither != 1 || o.bits != 8)) || (o.bits != 8 && o.bits != 32) || o.step < 1 || o.device < 0) return NOMAD_E_INVALID_ARG;
    if (!std::isfinite(o.lr) || !std::isfinite(o.weight_decay) || !(o.eps >= 0.0) || !std::isfinite(o.eps) || !(o.beta1 >= 0.0 && o.beta1 < 1.0) ||
        !(o.beta2 >= 0.0 && o.beta2 < 1.0))
        return NOMAD_E_INVALID_ARG;
    for (int32_t i = 0; i < count; ++i) {
        const nomad_adamw_tensor& t = tensors[i];
        if (t.n < 0 || kind_of(t.p_dtype, t.g_dtype) < 0) return NOMAD_E_INVALID_ARG;
        if (t.n > kMostElements) return NOMAD_E_TOO_LARGE;
        if (t.n > 0 && (!t.p || !t.g || !t.m || !t.v || (o.bits == 8 && (!t.m_scale || !t.v_scale)))) return NOMAD_E_INVALID_ARG;
    }
    const DeviceScope on(o.device);
    if (!on.ok()) return NOMAD_E_HIP;
    hipStream_t st = (hipStream_t)o.stream;
    Batch b;
    b.s.keep = (float)(1.0 - o.lr * o.weight_decay);
    b.s.rate = (float)(o.lr / (1.0 - std::pow(o.beta1, (double)o.step)));
    b.s.b1 = (float)o.beta1;
    b.s.c1 = (float)(1.0 - o.beta1);
    b.s.b2 = (float)o.beta2;
    b.s.c2 = (float)(1.0 - o.beta2);
    b.s.root = (float)(1.0 / std::sqrt(1.0 - std::pow(o.beta2, (double)o.step)));
    b.s.eps = (float)o.eps;
    b.s.step_low = (uint32_t)o.step;
    b.s.step_high = (uint32_t)((uint64_t)o.step >> 32);
    b.s.grad_scale = o.grad_scale;
    for (int kind = 0; kind < 7; ++kind) {
        b.count = 0;
        b.first[0] = 0;
        const auto flush = [&]() {
            if (b.count > 0) launch_kind(kind, b, o.bits == 8, dither, st);
            b.count = 0;
        };
        for (int32_t i = 0; i < count; ++i) {
            const nomad_adamw_tensor& t = tensors[i];
            if (t.n == 0 || kind_of(t.p_dtype, t.g_dtype) != kind) continue;
            if (b.count == kTensors || (b.count > 0 && b.first[b.count] + chunks_of(t.n) > kMostBlocks)) flush();
            b.t[b.count] = Tensor{t.p, t.g, t.m, t.v, t.m_scale, t.v_scale, t.n};
            b.first[b.count + 1] = b.first[b.count] + (uint32_t)chunks_of(t.n);
            ++b.count;
        }
        flush();
    }
    KTRY(hipGetLastError());
    return NOMAD_OK;
}

extern "C" int nomad_adamw_state_values(const void* const* codes, const float* const* scales, float* const* out, const int64_t* n, int32_t count,
                                        int32_t second, int32_t device, void* stream) {
    if (count < 0 || (count > 0 && (!codes || !scales || !out || !n)) || (second != 0 && second != 1) || device < 0) return NOMAD_E_INVALID_ARG;
    for (int32_t i = 0; i < count; ++i) {
        if (n[i] < 0 || (n[i] > 0 && (!codes[i] || !scales[i] || !out[i]))) return NOMAD_E_INVALID_ARG;
        if (n[i] > kMostElements) return NOMAD_E_TOO_LARGE;
    }
    const DeviceScope on(device);
    if (!on.ok()) return NOMAD_E_HIP;
    hipStream_t st = (hipStream_t)stream;
    ValuesBatch b;
    b.count = 0;
    b.first[0] = 0;
    const auto flush = [&]() {
        if (b.count > 0) {
            if (second) hipLaunchKernelGGL(k_adamw_values<true>, dim3(b.first[b.count]), dim3(kThreads), 0, st, b);
            else hipLaunchKernelGGL(k_adamw_values<false>, dim3(b.first[b.count]), dim3(kThreads), 0, st, b);
        }
        b.count = 0;
    };
    for (int32_t i = 0; i < count; ++i) {
        if (n[i] == 0) continue;
        if (b.count == kTensors || (b.count > 0 && b.first[b.count] + chunks_of(n[i]) > kMostBlocks)) flush();
        b.t[b.count] = {codes[i], scales[i], out[i], n[i]};
        b.first[b.count + 1] = b.first[b.count] + (uint32_t)chunks_of(n[i]);
        ++b.count;
    }
    flush();
    KTRY(hipGetLastError());
    return NOMAD_OK;
}
#pragma GCC visibility pop
