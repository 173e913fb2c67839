// libnomad: products over groups of rows behind the C ABI of include/nomad.h (host side).
#include <hip/hip_runtime.h>

#include "grouped_kernels.h"
#include "host_util.h"
#include "nomad.h"

using namespace nomad_grouped;

namespace {

int64_t size_of(int32_t dtype) { return dtype == NOMAD_F32 ? 4 : 2; }
bool is_dtype(int32_t dtype) { return dtype == NOMAD_F32 || dtype == NOMAD_BF16 || dtype == NOMAD_F16; }
bool by(const void* p, int64_t stride, int64_t size, int64_t bytes) { return ((uintptr_t)p | (uintptr_t)(stride * size)) % (uintptr_t)bytes == 0; }

template <typename T, typename O, int TA, int TB, int WA, int WB>
void launch_product(const ProductArgs& p, bool w_kc, bool async, hipStream_t st) {
    const int64_t tiles = std::min<int64_t>(p.rows, p.rows / TB + p.n_groups + 1);   // of rows: no more than one a row, one a group beyond the whole ones
    const int64_t total = tiles * ((p.out + TA - 1) / TA);
    const dim3 grid = grid_of((total + 7) / 8 * 8), block(64 * WA * WB);
    if (w_kc) {
        if (async) hipLaunchKernelGGL((k_grouped_product<T, O, TA, TB, WA, WB, true, true>), grid, block, 0, st, p);
        else hipLaunchKernelGGL((k_grouped_product<T, O, TA, TB, WA, WB, true, false>), grid, block, 0, st, p);
    } else {
        if (async) hipLaunchKernelGGL((k_grouped_product<T, O, TA, TB, WA, WB, false, true>), grid, block, 0, st, p);
        else hipLaunchKernelGGL((k_grouped_product<T, O, TA, TB, WA, WB, false, false>), grid, block, 0, st, p);
    }
}

template <typename T, typename O, int TA, int TB, int WA, int WB>
void launch_gradient(const GradientArgs& p, bool async, hipStream_t st) {
    const int64_t total = (int64_t)p.n_groups * ((p.in + TA - 1) / TA) * ((p.out + TB - 1) / TB);
    const dim3 grid = grid_of(total), block(64 * WA * WB);
    if (async) hipLaunchKernelGGL((k_grouped_gradient<T, O, TA, TB, WA, WB, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((k_grouped_gradient<T, O, TA, TB, WA, WB, false>), grid, block, 0, st, p);
}

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
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || a.device >= ndev) return NOMAD_E_HIP;
    KTRY(hipSetDevice(a.device));
    hipStream_t st = (hipStream_t)a.stream;
    const int64_t size = size_of(a.dtype), out_size = size_of(a.out_dtype), chunk = 16 / size;
    ProductArgs p{};
    p.offsets = a.offsets;
    p.x = Source{a.x, a.x_stride, a.order, a.x_rows, (uint32_t)a.per_row};
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
    p.whole_stores = by(a.y, a.y_stride, out_size, 4 * out_size) && (!a.z_out || by(a.z_out, a.z_stride, size, 4 * size)) ? 1 : 0;
    // loads straight to LDS take 16 aligned bytes: every row of either operand begins and ends on such a border
    const bool async = by(a.x, a.x_stride, size, 16) && by(a.w, a.w_group_stride, size, 16) && by(a.w, p.w_stride, size, 16) && a.in % chunk == 0 && (w_kc || a.out % chunk == 0);
    if (a.dtype == NOMAD_F32) launch_product<float, float, 128, 128, 2, 2>(p, w_kc, async, st);
    else if (a.dtype == NOMAD_BF16 && a.out_dtype == NOMAD_F32) launch_product<__bf16, float, 128, 128, 2, 2>(p, w_kc, async, st);
    else if (a.dtype == NOMAD_BF16) launch_product<__bf16, __bf16, 128, 128, 2, 2>(p, w_kc, async, st);
    else if (a.out_dtype == NOMAD_F32) launch_product<_Float16, float, 128, 128, 2, 2>(p, w_kc, async, st);
    else launch_product<_Float16, _Float16, 128, 128, 2, 2>(p, w_kc, async, st);
    KTRY(hipGetLastError());
    return NOMAD_OK;
}

extern "C" int64_t nomad_grouped_gradient_workspace(int64_t rows, int32_t n_groups, int32_t in, int32_t out, int32_t dtype) {
    (void)rows; (void)n_groups; (void)in; (void)out; (void)dtype;
    return 0;
}

extern "C" int nomad_grouped_weight_gradient(const nomad_grouped_gradient_args* args) {
    if (!args || args->struct_size != sizeof(nomad_grouped_gradient_args)) return NOMAD_E_INVALID_ARG;
    const nomad_grouped_gradient_args& a = *args;
    if (!is_dtype(a.dtype) || (a.out_dtype != a.dtype && a.out_dtype != NOMAD_F32)) return NOMAD_E_INVALID_ARG;
    if (a.n_groups < 1 || a.rows < 0 || a.in < 1 || a.out < 1 || a.per_row < 1 || a.device < 0 || a.x_stride < 0 || a.dy_stride < 0) return NOMAD_E_INVALID_ARG;
    if (a.rows > NOMAD_MAX_ROWS || a.x_rows > NOMAD_MAX_ROWS || a.n_groups > NOMAD_MAX_GROUPS || a.in > NOMAD_MAX_COLUMNS || a.out > NOMAD_MAX_COLUMNS) return NOMAD_E_TOO_LARGE;
    if (!a.offsets || !a.dw || (a.rows > 0 && (!a.x || !a.dy || a.x_rows < 1 || (!a.order && a.x_rows < a.rows)))) return NOMAD_E_INVALID_ARG;
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || a.device >= ndev) return NOMAD_E_HIP;
    KTRY(hipSetDevice(a.device));
    hipStream_t st = (hipStream_t)a.stream;
    const int64_t size = size_of(a.dtype), out_size = size_of(a.out_dtype), chunk = 16 / size;
    GradientArgs p{};
    p.offsets = a.offsets;
    p.x = Source{a.x, a.x_stride, a.order, a.x_rows, (uint32_t)a.per_row};
    p.dy = Source{a.dy, a.dy_stride, nullptr, a.rows, 1};
    p.dw = a.dw;
    p.db = a.db;
    p.rows = a.rows;
    p.n_groups = a.n_groups;
    p.in = a.in;
    p.out = a.out;
    p.whole_stores = by(a.dw, a.in, out_size, 4 * out_size) ? 1 : 0;
    const bool async = by(a.x, a.x_stride, size, 16) && by(a.dy, a.dy_stride, size, 16) && a.in % chunk == 0 && a.out % chunk == 0;
    if (a.dtype == NOMAD_F32) launch_gradient<float, float, 128, 128, 2, 2>(p, async, st);
    else if (a.dtype == NOMAD_BF16 && a.out_dtype == NOMAD_F32) launch_gradient<__bf16, float, 128, 128, 2, 2>(p, async, st);
    else if (a.dtype == NOMAD_BF16) launch_gradient<__bf16, __bf16, 128, 128, 2, 2>(p, async, st);
    else if (a.out_dtype == NOMAD_F32) launch_gradient<_Float16, float, 128, 128, 2, 2>(p, async, st);
    else launch_gradient<_Float16, _Float16, 128, 128, 2, 2>(p, async, st);
    KTRY(hipGetLastError());
    return NOMAD_OK;
}
#pragma GCC visibility pop
