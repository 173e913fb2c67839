// libnomad: dense products behind the C ABI of include/nomad.h (host side).
#include <hip/hip_runtime.h>

#include <atomic>

#include "dense_launch.h"
#include "device_scope.h"
#include "nomad.h"

using namespace nomad_dense;

namespace {

int64_t size_of(int32_t dtype) { return dtype == NOMAD_F32 ? 4 : 2; }
bool is_dtype(int32_t dtype) { return dtype == NOMAD_F32 || dtype == NOMAD_BF16 || dtype == NOMAD_F16; }
bool by(const void* p, int64_t stride, int64_t size, int64_t bytes) { return ((uintptr_t)p | (uintptr_t)(stride * size)) % (uintptr_t)bytes == 0; }
int64_t round16(int64_t bytes) { return (bytes + 15) / 16 * 16; }

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
// What products are planned for, on any device: the size of their work space must not depend on where it is asked
constexpr int kPlanUnits = 256;

// Work space of a product: [parts][rows][columns] in float32 where there is more than one part
int64_t part_bytes(const Plan& plan, int64_t rows, int64_t columns) { return plan.parts > 1 ? round16(plan.parts * rows * columns * (int64_t)sizeof(float)) : 0; }
// and of whichever plan a product has: alignment and the order of W's strides, which the size does not know, have a say in it
int64_t most_bytes(int64_t rows, int64_t columns, int64_t k, bool small) {
    int64_t most = 0;
    for (int way = 0; way < 4; ++way) most = std::max(most, part_bytes(plan(rows, columns, k, small, way & 1, way & 2, kPlanUnits), rows, columns));
    return most;
}
// Where the sums go that are not finished where they are made: parts to work space, and float32 results of 16-bit operands to their place, where
// what follows is done to them
void place_sums(DenseArgs& p, Launch& l, void* work) {
    p.parts = (int32_t)l.plan.parts;
    p.length = l.plan.length;
    if (p.parts > 1) {
        p.part = (float*)work;
        p.part_stride = p.columns;
    } else if (l.wide && l.plan.tile != kFew) {
        p.part = (float*)p.f.y;
        p.part_stride = p.f.y_stride;
    }
    if (p.part) l.stores = by(p.part, p.part_stride, sizeof(float), 16) && p.columns % 4 == 0;
}

void launch(int32_t dtype, const DenseArgs& p, const Launch& l, hipStream_t st) {
    if (dtype == NOMAD_F32) dense_f32(p, l, st);
    else if (dtype == NOMAD_BF16) dense_bf16(p, l, st);
    else dense_f16(p, l, st);
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" int64_t nomad_dense_workspace(int64_t rows, int32_t in, int32_t out, int32_t dtype) {
    if (rows < 1 || in < 1 || out < 1 || !is_dtype(dtype) || rows > NOMAD_MAX_ROWS || in > NOMAD_MAX_COLUMNS || out > NOMAD_MAX_COLUMNS) return 0;
    return most_bytes(rows, out, in, size_of(dtype) == 2);
}

extern "C" int nomad_dense_product(const nomad_dense_args* args) {
    if (!args || args->struct_size != sizeof(nomad_dense_args)) return NOMAD_E_INVALID_ARG;
    const nomad_dense_args& a = *args;
    if (!is_dtype(a.dtype) || (a.out_dtype != a.dtype && a.out_dtype != NOMAD_F32) || a.activation < NOMAD_ACT_NONE || a.activation > NOMAD_ACT_GELU) return NOMAD_E_INVALID_ARG;
    if (a.rows < 0 || a.in < 1 || a.out < 1 || a.device < 0) return NOMAD_E_INVALID_ARG;
    if (a.slope_at && (a.bias || a.z_out || a.residual)) return NOMAD_E_INVALID_ARG;
    const bool w_kc = a.w_in_stride == 1 || a.in == 1;
    if (!w_kc && a.w_out_stride != 1 && a.out != 1) return NOMAD_E_INVALID_ARG;
    if (a.x_stride < 0 || a.w_in_stride < 0 || a.w_out_stride < 0 || a.residual_stride < 0) return NOMAD_E_INVALID_ARG;
    if (a.rows > 1 && (a.y_stride < a.out || (a.z_out && a.z_stride < a.out) || (a.slope_at && a.slope_stride < 0))) return NOMAD_E_INVALID_ARG;
    if (a.rows > NOMAD_MAX_ROWS || a.in > NOMAD_MAX_COLUMNS || a.out > NOMAD_MAX_COLUMNS) return NOMAD_E_TOO_LARGE;
    if (a.rows == 0) return NOMAD_OK;
    if (!a.x || !a.w || !a.y) return NOMAD_E_INVALID_ARG;
    const int64_t need = nomad_dense_workspace(a.rows, a.in, a.out, a.dtype);
    if (need > 0 && (!a.workspace || a.workspace_bytes < need || (uintptr_t)a.workspace % 16)) return NOMAD_E_INVALID_ARG;
    const DeviceScope on(a.device);
    if (!on.ok()) return NOMAD_E_HIP;
    const int units = units_of(a.device);
    if (units < 1) return NOMAD_E_HIP;
    const int64_t size = size_of(a.dtype), out_size = size_of(a.out_dtype), chunk = 16 / size;
    DenseArgs p{};
    p.a = a.w;
    p.a_stride = w_kc ? a.w_out_stride : a.w_in_stride;
    p.b = a.x;
    p.b_stride = a.x_stride;
    p.rows = a.rows;
    p.columns = a.out;
    p.k = a.in;
    p.f.bias = a.bias;
    p.f.residual = a.residual;
    p.f.residual_stride = a.residual_stride;
    p.f.slope_at = a.slope_at;
    p.f.slope_stride = a.slope_stride;
    p.f.z_out = a.z_out;
    p.f.z_stride = a.z_stride;
    p.f.y = a.y;
    p.f.y_stride = a.y_stride;
    p.f.activation = a.activation;
    p.f.factor = 1.f;
    Launch l;
    l.turn = w_kc ? kForward : kTurned;
    l.wide = a.out_dtype != a.dtype;
    // loads straight to LDS take 16 aligned bytes, and so do whole stores: rows begin and end on such a border
    l.loads = by(a.x, a.x_stride, size, 16) && by(a.w, p.a_stride, size, 16) && a.in % chunk == 0 && (w_kc || a.out % chunk == 0);
    l.stores = by(a.y, a.y_stride, out_size, 16) && a.out % chunk == 0 && (!a.z_out || by(a.z_out, a.z_stride, size, 16));
    l.plan = plan(a.rows, a.out, a.in, size == 2, w_kc, l.loads && l.stores, kPlanUnits);
    l.units = units;
    place_sums(p, l, a.workspace);
    launch(a.dtype, p, l, (hipStream_t)a.stream);
    KTRY(hipGetLastError());
    return NOMAD_OK;
}

extern "C" int64_t nomad_dense_gradient_workspace(int64_t rows, int32_t in, int32_t out, int32_t dtype, int32_t activation) {
    if (rows < 1 || in < 1 || out < 1 || !is_dtype(dtype) || rows > NOMAD_MAX_ROWS || in > NOMAD_MAX_COLUMNS || out > NOMAD_MAX_COLUMNS) return 0;
    const bool small = size_of(dtype) == 2;
    const int64_t products = std::max(most_bytes(rows, in, out, small), most_bytes(out, in, rows, small));
    if (activation == NOMAD_ACT_NONE) return products + round16(kMostParts * out * (int64_t)sizeof(float));
    return products + round16(rows * out * size_of(dtype)) + round16(plan_slope(rows, out, kPlanUnits).parts * out * (int64_t)sizeof(float));
}

extern "C" int nomad_dense_gradient(const nomad_dense_gradient_args* args) {
    if (!args || args->struct_size != sizeof(nomad_dense_gradient_args)) return NOMAD_E_INVALID_ARG;
    const nomad_dense_gradient_args& a = *args;
    if (!is_dtype(a.dtype) || (a.out_dtype != a.dtype && a.out_dtype != NOMAD_F32) || a.activation < NOMAD_ACT_NONE || a.activation > NOMAD_ACT_GELU) return NOMAD_E_INVALID_ARG;
    if (a.rows < 0 || a.in < 1 || a.out < 1 || a.device < 0 || a.dy_stride < 0 || a.x_stride < 0 || a.z_stride < 0 || a.w_in_stride < 0 || a.w_out_stride < 0) return NOMAD_E_INVALID_ARG;
    if (a.rows > NOMAD_MAX_ROWS || a.in > NOMAD_MAX_COLUMNS || a.out > NOMAD_MAX_COLUMNS) return NOMAD_E_TOO_LARGE;
    if (a.db && !a.dw) return NOMAD_E_INVALID_ARG;
    if (a.rows == 0 && !a.dw) return NOMAD_OK;   // (an empty dx is where it likes)
    if (!a.dx && !a.dw) return NOMAD_E_INVALID_ARG;
    const bool w_kc = a.w_in_stride == 1 || a.in == 1;   // (then columns of W, which dx runs along, are contiguous)
    if (a.dx && !w_kc && a.w_out_stride != 1 && a.out != 1) return NOMAD_E_INVALID_ARG;
    if (a.dx && a.rows > 1 && a.dx_stride < a.in) return NOMAD_E_INVALID_ARG;
    if (a.rows > 0 && (!a.dy || (a.dx && !a.w) || (a.dw && !a.x) || (a.activation != NOMAD_ACT_NONE && !a.z))) return NOMAD_E_INVALID_ARG;
    const int64_t need = nomad_dense_gradient_workspace(a.rows, a.in, a.out, a.dtype, a.activation);
    if (need > 0 && (!a.workspace || a.workspace_bytes < need || (uintptr_t)a.workspace % 16)) return NOMAD_E_INVALID_ARG;
    const DeviceScope on(a.device);
    if (!on.ok()) return NOMAD_E_HIP;
    const int units = units_of(a.device);
    if (units < 1) return NOMAD_E_HIP;
    hipStream_t st = (hipStream_t)a.stream;
    const int64_t size = size_of(a.dtype), out_size = size_of(a.out_dtype), chunk = 16 / size;
    const void* dz = a.dy;
    int64_t dz_stride = a.dy_stride;
    char* work = (char*)a.workspace;
    const float kept = a.dtype == NOMAD_F16 && a.rows > 0 && (a.activation == NOMAD_ACT_SILU || a.activation == NOMAD_ACT_GELU) ? 0.875f : 1.f;   // of dz (k_dense_slope)
    float* db = a.db;   // what the product of the weights' gradient is to leave; with an activation the sums are of dz before its rounding
    if (a.activation != NOMAD_ACT_NONE && a.rows > 0) {
        const SlopePlan l = plan_slope(a.rows, a.out, kPlanUnits);
        const SlopeArgs p{a.dy, a.dy_stride, a.z, a.z_stride, work, a.db ? (l.parts > 1 ? (float*)(work + round16(a.rows * a.out * size)) : a.db) : nullptr,
                          a.rows, l.length, a.out, a.activation, 0, kept};
        const bool vec = by(a.dy, a.dy_stride, size, 16) && by(a.z, a.z_stride, size, 16) && a.out % chunk == 0;
        if (a.dtype == NOMAD_F32) slope_f32(p, l.parts, vec, st);
        else if (a.dtype == NOMAD_BF16) slope_bf16(p, l.parts, vec, st);
        else slope_f16(p, l.parts, vec, st);
        if (a.db && l.parts > 1) launch_sums(p.sums, (int32_t)l.parts, a.out, a.db, st);
        dz = work;
        dz_stride = a.out;
        work += round16(a.rows * a.out * size) + round16(l.parts * a.out * (int64_t)sizeof(float));
        db = nullptr;
    }
    if (a.dx && a.rows > 0) {   // dx = dz W: rows of W turned, whichever way they lie
        DenseArgs p{};
        p.a = a.w;
        p.a_stride = w_kc ? a.w_out_stride : a.w_in_stride;
        p.b = dz;
        p.b_stride = dz_stride;
        p.rows = a.rows;
        p.columns = a.in;
        p.k = a.out;
        p.f.factor = 1.f / kept;
        p.f.y = a.dx;
        p.f.y_stride = a.dx_stride;
        Launch l;
        l.turn = w_kc ? kTurned : kForward;
        l.wide = false;
        l.loads = by(dz, dz_stride, size, 16) && by(a.w, p.a_stride, size, 16) && a.out % chunk == 0 && (!w_kc || a.in % chunk == 0);
        l.stores = by(a.dx, a.dx_stride, size, 16) && a.in % chunk == 0;
        l.plan = plan(a.rows, a.in, a.out, size == 2, false, l.loads && l.stores, kPlanUnits);
        l.units = units;
        place_sums(p, l, work);
        launch(a.dtype, p, l, st);
    }
    if (a.dw) {
        DenseArgs p{};
        p.a = a.x;
        p.a_stride = a.x_stride;
        p.b = dz;
        p.b_stride = dz_stride;
        p.rows = a.out;
        p.columns = a.in;
        p.k = a.rows;
        p.f.factor = 1.f / kept;
        p.f.y = a.dw;
        p.f.y_stride = a.in;
        Launch l;
        l.turn = kWeights;
        l.wide = a.out_dtype != a.dtype;
        l.loads = by(a.x, a.x_stride, size, 16) && by(dz, dz_stride, size, 16) && a.in % chunk == 0 && a.out % chunk == 0;
        l.stores = by(a.dw, a.in, out_size, 16) && a.in % chunk == 0;
        l.plan = plan(a.out, a.in, a.rows, size == 2, false, l.loads && l.stores, kPlanUnits);
        l.units = units;
        place_sums(p, l, work);
        p.sums = db ? (p.parts > 1 ? (float*)(work + part_bytes(l.plan, a.out, a.in)) : db) : nullptr;
        launch(a.dtype, p, l, st);
        if (db && p.parts > 1) launch_sums(p.sums, p.parts, a.out, db, st);
    }
    KTRY(hipGetLastError());
    return NOMAD_OK;
}
#pragma GCC visibility pop
