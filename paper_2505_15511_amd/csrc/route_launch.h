// What the routers' host sides share: how rows are cut into chunks, and the launches of the counting sort.
#pragma once
#include "host_util.h"
#include "nomad.h"
#include "route_kernels.h"

namespace {

inline bool is_dtype(int32_t dtype) { return dtype == NOMAD_F32 || dtype == NOMAD_BF16 || dtype == NOMAD_F16; }
inline int64_t size_of(int32_t dtype) { return dtype == NOMAD_F32 ? 4 : 2; }
inline bool by(const void* p, int64_t stride, int64_t size, int64_t bytes) { return ((uintptr_t)p | (uintptr_t)(stride * size)) % (uintptr_t)bytes == 0; }

// Rows a chunk of the counts: their scan walks the chunks of an expert, so there are about a thousand at most, and no fewer rows
// in one than keep the counts below the logits (whole calls of nomad_route on 65,536 rows of 256, 65,536 of 1,024 and 8,192 of 2,048 in float32, k = 2: 28, 75 and
// 83 us, 45, 164 and 232 with 256 rows at least)
inline int64_t chunk_rows(int64_t n) { return std::max<int64_t>(64, (n + 1023) / 1024); }
// One workgroup does it all where the logits are few (a row of 256: 4.4 us, the three kernels of the other form 12.4; 100 rows of 50: 6.4 against 40)
// (scored_launch.h has the scored router's times) and its counters and slots fit the 64 KB of LDS that a launch has without asking
inline bool is_small(int64_t n, int32_t n_experts, int32_t k) { return n * n_experts <= 32768 && n <= 1024 && n_experts + n * k <= 16384; }

// The counts of the chunks into places
inline void launch_places(const nomad_router::RouteArgs& p, hipStream_t st) {
    using namespace nomad_router;
    hipLaunchKernelGGL(k_route_scan, dim3(blocks_of(p.n_experts, kScanColumns)), dim3(kScanThreads), 0, st, p);
    // (four wavefronts' counters of 2,048 experts are 32 KB of LDS; two million slots: 28 us, 44 with one wavefront a chunk; whole calls on 65,536
    // rows of 1,024 and 2,048: 178 and 282 us, 183 and 287 with one)
    if (p.n_experts <= 2048) hipLaunchKernelGGL(k_route_place<4>, dim3((uint32_t)p.n_chunks), dim3(256), sizeof(int32_t) * 4 * (size_t)p.n_experts, st, p);
    else hipLaunchKernelGGL(k_route_place<1>, dim3((uint32_t)p.n_chunks), dim3(64), sizeof(int32_t) * (size_t)p.n_experts, st, p);
}
// What the grouping of n rows is put into
inline void fill_places(nomad_router::RouteArgs& p, int64_t n, int32_t n_experts, int32_t k, int32_t* experts, float* weights, int32_t* offsets, int32_t* order,
                        int32_t* slots, void* workspace) {
    p.n = n;
    p.n_experts = n_experts;
    p.k = k;
    p.experts = experts;
    p.weights = weights;
    p.offsets = offsets;
    p.order = order;
    p.slots = slots;
    p.chunk = (int32_t)chunk_rows(n);
    p.n_chunks = (int32_t)((n + p.chunk - 1) / p.chunk);
    p.counts = (int32_t*)workspace;
    p.totals = (int32_t*)workspace + (int64_t)p.n_chunks * n_experts;
}

}  // namespace
