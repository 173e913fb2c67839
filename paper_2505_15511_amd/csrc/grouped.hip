// libnomad: products over groups of rows behind the C ABI of include/nomad.h (host side).
#include <hip/hip_runtime.h>

#include <atomic>

#include "device_scope.h"
#include "grouped_launch.h"
#include "nomad.h"

using namespace nomad_grouped;

namespace {

int64_t size_of(int32_t dtype) { return dtype == NOMAD_F32 ? 4 : 2; }
bool is_dtype(int32_t dtype) { return dtype == NOMAD_F32 || dtype == NOMAD_BF16 || dtype == NOMAD_F16; }
bool by(const void* p, int64_t stride, int64_t size, int64_t bytes) { return ((uintptr_t)p | (uintptr_t)(stride * size)) % (uintptr_t)bytes == 0; }

// compute units of a device (asked for once)
int units_of(int32_t device) {
    constexpr int known = 64;
    static std::atomic<int> count[known];
    int units = device < known ? count[device].load(std::memory_order_relaxed) : 0;
    if (units > 0) return units;
    if (hipDeviceGetAttribute(&units, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess || units < 1) return 0;
    if (device < known) count[device].store(units, std::memory_order_relaxed);
    return units;
}
// What the work space of the gradients is planned for, on any device: its size must not depend on where it is asked
constexpr int kPlanUnits = 256;

}  // namespace

#pragma GCC visibility push(default)
extern "C" int nomad_grouped_product(const nomad_grouped_product_args* args) {
    if (!args || args->struct_size != sizeof(nomad_grouped_product_args)) return NOMAD_E_INVALID_ARG;
    const nomad_grouped_product_args& a = *args;
    if (!is_dtype(a.dtype) || (a.out_dtype != a.dtype && a.out_dtype != NOMAD_F32) || a.activation < NOMAD_ACT_NONE || a.activation > NOMAD_ACT_GELU) return NOMAD_E_INVALID_ARG;
    if (a.n_groups < 1 || a.rows < 0 || a.in < 1 || a.out < 1 || a.per_row < 1 || a.device < 0) return NOMAD_E_INVALID_ARG;
    if (a.slope_at && (a.bias || a.z_out)) return NOMAD_E_INVALID_ARG;
    const bool w_kc = a.w_in_stride == 1 || a.in == 1;
    if (!w_kc && a.w_out_stride != 1 && a.out != 1) return NOMAD_E_INVALID_ARG;
    if (a.x_stride < 0 || a.w_group_stride < 0 || a.w_in_stride < 0 || a.w_out_stride < 0 || a.bias_stride < 0) return NOMAD_E_INVALID_ARG;
    if (a.rows > 1 && (a.y_stride < a.out || (a.z_out && a.z_stride < a.out) || (a.slope_at && a.slope_stride < a.out))) return NOMAD_E_INVALID_ARG;
    if (a.rows > NOMAD_MAX_ROWS || a.x_rows > NOMAD_MAX_ROWS || a.n_groups > NOMAD_MAX_GROUPS || a.in > NOMAD_MAX_COLUMNS || a.out > NOMAD_MAX_COLUMNS) return NOMAD_E_TOO_LARGE;
    if (a.rows == 0) return NOMAD_OK;
    if (!a.offsets || !a.x || !a.w || !a.y || a.x_rows < 1 || (!a.order && a.x_rows < a.rows)) return NOMAD_E_INVALID_ARG;
    const DeviceScope on(a.device);
    if (!on.ok()) return NOMAD_E_HIP;
    hipStream_t st = (hipStream_t)a.stream;
    const int64_t size = size_of(a.dtype), out_size = size_of(a.out_dtype), chunk = 16 / size;
    ProductArgs p{};
    p.offsets = a.offsets;
    p.x = Source{a.x, a.x_stride, a.order, a.x_rows, a.order ? (uint32_t)a.per_row : 1u};
    p.w = a.w;
    p.w_group = a.w_group_stride;
    p.w_stride = w_kc ? a.w_out_stride : a.w_in_stride;
    p.bias = a.bias;
    p.bias_stride = a.bias_stride;
    p.slope_at = a.slope_at;
    p.slope_stride = a.slope_stride;
    p.y = a.y;
    p.y_stride = a.y_stride;
    p.z_out = a.z_out;
    p.z_stride = a.z_stride;
    p.rows = a.rows;
    p.n_groups = a.n_groups;
    p.in = a.in;
    p.out = a.out;
    p.activation = a.activation;
    // loads straight to LDS take 16 aligned bytes, and so do whole stores: rows begin and end on such a border
    const bool loads = by(a.x, a.x_stride, size, 16) && by(a.w, a.w_group_stride, size, 16) && by(a.w, p.w_stride, size, 16) && a.in % chunk == 0 && (w_kc || a.out % chunk == 0);
    const bool stores = by(a.y, a.y_stride, out_size, 16) && a.out % (16 / out_size) == 0 && (!a.z_out || (by(a.z_out, a.z_stride, size, 16) && a.out % chunk == 0));
    const int units = units_of(a.device);
    if (units < 1) return NOMAD_E_HIP;
    const bool wide = a.out_dtype != a.dtype;
    const ProductTile tile = plan_product(a.rows, a.n_groups, a.out, size == 2, w_kc, units);
    if (a.dtype == NOMAD_F32) product_f32(p, tile, wide, w_kc, loads, stores, units, st);
    else if (a.dtype == NOMAD_BF16) product_bf16(p, tile, wide, w_kc, loads, stores, units, st);
    else product_f16(p, tile, wide, w_kc, loads, stores, units, st);
    KTRY(hipGetLastError());
    return NOMAD_OK;
}

extern "C" int64_t nomad_grouped_gradient_workspace(int64_t rows, int32_t n_groups, int32_t in, int32_t out, int32_t dtype) {
    if (rows < 1 || n_groups < 1 || in < 1 || out < 1 || !is_dtype(dtype) || rows > NOMAD_MAX_ROWS || in > NOMAD_MAX_COLUMNS || out > NOMAD_MAX_COLUMNS) return 0;
    return plan_gradient(rows, n_groups, in, out, size_of(dtype) == 2, kPlanUnits).slots * ((int64_t)in + 1) * out * (int64_t)sizeof(float);
}

extern "C" int nomad_grouped_weight_gradient(const nomad_grouped_gradient_args* args) {
    if (!args || args->struct_size != sizeof(nomad_grouped_gradient_args)) return NOMAD_E_INVALID_ARG;
    const nomad_grouped_gradient_args& a = *args;
    if (!is_dtype(a.dtype) || (a.out_dtype != a.dtype && a.out_dtype != NOMAD_F32)) return NOMAD_E_INVALID_ARG;
    if (a.n_groups < 1 || a.rows < 0 || a.in < 1 || a.out < 1 || a.per_row < 1 || a.device < 0 || a.x_stride < 0 || a.dy_stride < 0) return NOMAD_E_INVALID_ARG;
    if (a.rows > NOMAD_MAX_ROWS || a.x_rows > NOMAD_MAX_ROWS || a.n_groups > NOMAD_MAX_GROUPS || a.in > NOMAD_MAX_COLUMNS || a.out > NOMAD_MAX_COLUMNS) return NOMAD_E_TOO_LARGE;
    const int64_t need = nomad_grouped_gradient_workspace(a.rows, a.n_groups, a.in, a.out, a.dtype);
    if (need > 0 && (!a.workspace || a.workspace_bytes < need || (uintptr_t)a.workspace % 16)) return NOMAD_E_INVALID_ARG;
    if (!a.offsets || !a.dw || (a.rows > 0 && (!a.x || !a.dy || a.x_rows < 1 || (!a.order && a.x_rows < a.rows)))) return NOMAD_E_INVALID_ARG;
    const DeviceScope on(a.device);
    if (!on.ok()) return NOMAD_E_HIP;
    hipStream_t st = (hipStream_t)a.stream;
    const int64_t size = size_of(a.dtype), out_size = size_of(a.out_dtype), chunk = 16 / size;
    GradientArgs p{};
    p.offsets = a.offsets;
    p.x = Source{a.x, a.x_stride, a.order, a.x_rows, a.order ? (uint32_t)a.per_row : 1u};
    p.dy = Source{a.dy, a.dy_stride, nullptr, a.rows, 1};
    p.dw = a.dw;
    p.db = a.db;
    p.rows = a.rows;
    p.n_groups = a.n_groups;
    p.in = a.in;
    p.out = a.out;
    const GradientPlan plan = plan_gradient(a.rows, a.n_groups, a.in, a.out, size == 2, kPlanUnits);
    p.part = (float*)a.workspace;
    p.most = plan.most;
    p.slot_bits = plan.slot_bits;
    p.slots = plan.slots;
    const bool loads = by(a.x, a.x_stride, size, 16) && by(a.dy, a.dy_stride, size, 16) && a.in % chunk == 0 && a.out % chunk == 0;
    const bool stores = by(a.dw, a.in, out_size, 16) && a.in % 4 == 0;   // (sums of parts are stored 16 bytes at a time too)
    const int units = units_of(a.device);
    if (units < 1) return NOMAD_E_HIP;
    const bool wide = a.out_dtype != a.dtype;
    if (a.dtype == NOMAD_F32) gradient_f32(p, plan, wide, loads, stores, units, st);
    else if (a.dtype == NOMAD_BF16) gradient_bf16(p, plan, wide, loads, stores, units, st);
    else gradient_f16(p, plan, wide, loads, stores, units, st);
    KTRY(hipGetLastError());
    return NOMAD_OK;
}
#pragma GCC visibility pop
