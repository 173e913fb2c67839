// The norm of many tensors together (gfx950): sqrt of the sum of all squares, and the factor that clips a step.
//
// One pass over the elements in one launch for up to 192 tensors, a workgroup a run of one of them; a second kernel adds the runs up,
// in one order.  Squares and sums are float64: gradients of 1e-25 and of 1e30 count alike, and the last square of 10^9 is not lost; they go on
// under the loads.  Bound by the elements' bytes: 387 M in bfloat16 136 us a call (5.7 TB/s).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace nomad_norm {

constexpr int kTensors = 192;              // a launch: their addresses are its arguments (under 4 KB)
constexpr int kThreads = 256, kSumThreads = 1024;
constexpr int64_t kRun = 2048;             // elements of the shortest run, and what a longer one is a multiple of
constexpr int64_t kRuns = 2048;            // of all tensors together, and one a tensor more

struct Tensor {
    const void* g;
    int64_t n;                             // its type in the two lowest bits
};
struct Batch {
    Tensor t[kTensors];
    uint32_t first[kTensors + 1];          // workgroup of each tensor
    int32_t count;
    int64_t run;                           // elements a workgroup takes
    double* part;                          // a sum a workgroup
};

struct alignas(16) Chunk { uint32_t w[4]; };

__device__ __forceinline__ void add_square(double& sum, float v) {
    const double d = (double)v;
    sum = fma(d, d, sum);
}
template <typename T>
__device__ __forceinline__ void add_chunk(double (&sum)[4], const Chunk& c) {
    constexpr int n = 16 / (int)sizeof(T);
    T v[n];
    __builtin_memcpy(v, &c, 16);
#pragma unroll
    for (int i = 0; i < n; ++i) add_square(sum[i % 4], (float)v[i]);
}

template <typename T>
__device__ __forceinline__ double sum_run(const T* g, int64_t count) {
    constexpr int n = 16 / (int)sizeof(T), kAhead = 4;
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    const int tid = threadIdx.x;
    // elements before the first border of 16 bytes and behind the last one are taken one by one
    const int64_t off = (int64_t)((uintptr_t)g & 15) / (int64_t)sizeof(T), lead = off == 0 ? 0 : (n - off < count ? n - off : count);
    const int64_t chunks = (count - lead) / n, rest = lead + chunks * n;
    if (tid < lead) add_square(sum[0], (float)g[tid]);
    if (rest + tid < count) add_square(sum[1], (float)g[rest + tid]);
    const Chunk* from = (const Chunk*)(g + lead);
    int64_t c = tid;
    for (; c + (kAhead - 1) * kThreads < chunks; c += kAhead * kThreads) {
        Chunk v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) v[i] = from[c + i * kThreads];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) add_chunk<T>(sum, v[i]);
    }
    for (; c < chunks; c += kThreads) add_chunk<T>(sum, from[c]);
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// the threads' values added up, for thread 0
template <int THREADS>
__device__ __forceinline__ double sum_threads(double v) {
    __shared__ double waves[THREADS / 64];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) v += waves[w];
    return v;
}

__global__ void __launch_bounds__(kThreads) k_norm_runs(Batch b) {
    int lo = 0, hi = b.count;   // the tensor of this workgroup
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (b.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid;
    }
    const int64_t size = b.t[lo].n >> 2, begin = (int64_t)(blockIdx.x - b.first[lo]) * b.run, count = size - begin < b.run ? size - begin : b.run;
    const int type = (int)(b.t[lo].n & 3);
    double sum;
    if (type == 0) sum = sum_run((const float*)b.t[lo].g + begin, count);
    else if (type == 1) sum = sum_run((const __bf16*)b.t[lo].g + begin, count);
    else sum = sum_run((const _Float16*)b.t[lo].g + begin, count);
    sum = sum_threads<kThreads>(sum);
    if (threadIdx.x == 0) b.part[blockIdx.x] = sum;
}

// norm = |s| sqrt(sum of the runs), scale = s where that is at most `most`, otherwise s most / norm (a norm that is NaN makes it NaN,
// one that is infinite 0)
__global__ void __launch_bounds__(kSumThreads) k_norm_sum(const double* part, int64_t runs, const float* grad_scale, double most, float* norm, float* scale) {
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < runs; i += kSumThreads) sum += part[i];
    sum = sum_threads<kSumThreads>(sum);
    if (threadIdx.x != 0) return;
    const double s = grad_scale ? (double)*grad_scale : 1.0, all = fabs(s) * sqrt(sum);
    *norm = (float)all;
    if (scale) *scale = (float)(all <= most ? s : s * (most / all));
}

}  // namespace nomad_norm
