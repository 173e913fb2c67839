// The router of a learned map and the weighted sum over a row's experts (gfx950).
//
// k_route_pick   the k largest of every row of logits and their weights; counts of a chunk of rows by expert
// k_route_scan   counts of all chunks -> where every chunk's slots of every expert begin, and every expert's total
// k_route_place  slots (row times k plus rank) into the order of their experts, stable
// k_route_small  all of it in one workgroup
// All are passes over the logits or over n k words: what they cost is the logits' bytes.  A million rows of 256 float32 logits, k = 2: 224 us for
// the pick (4.6 TB/s), 6 + 28 for scan and places, 187 for the gradient (5.5 TB/s written), 454 where weights are over all experts (it reads the
// row three times, from the caches after the first).  The weighted sum of 262,144 x 2 rows of 768 in bfloat16 256 us (4.7 TB/s), its gradients 416
// (4.8); of 65,536 x 2 rows of 256 in float32 38 and 85 us.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

namespace nomad_router {

constexpr int kMaxK = 8;
constexpr int kMaxExperts = 16384;
constexpr int kPickThreads = 256, kScanThreads = 1024, kScanColumns = 16;

// Workgroup number of a launch with more of them than one dimension takes (grid_of)
__device__ __forceinline__ int64_t block_number() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

template <typename T>
__device__ __forceinline__ float value_of(T v) {   // (a NaN is never chosen; both zeros are the same number)
    const float f = (float)v;
    return f == f ? f + 0.f : -INFINITY;
}

// Order of (value, lowest index first) as an integer; 0 for -inf
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index) {
    if (v == -INFINITY) return 0;
    const uint32_t u = __float_as_uint(v);
    return ((uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32) | (uint32_t)~index;
}

// The K best that a lane has seen, best first; indices come in ascending order, so the first of equals stays ahead
template <int K>
struct Best {
    float v[K];
    uint32_t e[K];
    __device__ __forceinline__ Best() {
#pragma unroll
        for (int j = 0; j < K; ++j) { v[j] = -INFINITY; e[j] = 0; }
    }
    __device__ __forceinline__ void take(float x, uint32_t index) {
        if (!(x > v[K - 1])) return;
#pragma unroll
        for (int j = K - 1; j >= 0; --j) {
            const bool before = j > 0 && x > v[j > 0 ? j - 1 : 0];
            if (before) { v[j] = v[j > 0 ? j - 1 : 0]; e[j] = e[j > 0 ? j - 1 : 0]; }
            else if (x > v[j]) { v[j] = x; e[j] = index; }
        }
    }
};

// A row of `count` elements by LANES lanes, in chunks of 16 bytes where rows are aligned to them, four on their way at once;
// visit(value, index)
template <typename T, int LANES, bool VEC, typename F>
__device__ __forceinline__ void each(const T* row, int32_t count, int sub, F visit) {
    constexpr int epc = VEC ? 16 / (int)sizeof(T) : 1;
    for (int32_t c0 = sub * epc; c0 < count; c0 += 4 * LANES * epc) {
        T part[4][epc];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int32_t c = c0 + b * LANES * epc;
            if (c >= count) continue;
            if (VEC) *(uint4*)part[b] = *(const uint4*)(row + c);
            else part[b][0] = row[c];
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int32_t c = c0 + b * LANES * epc;
            if (c >= count) continue;
#pragma unroll
            for (int i = 0; i < epc; ++i) visit(value_of(part[b][i]), (uint32_t)(c + i));
        }
    }
}

template <int LANES, typename V, typename F>
__device__ __forceinline__ V reduce(V v, F op) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) v = op(v, (V)__shfl_xor(v, d));
    return v;
}

// One row by LANES lanes: its experts and weights (every lane of the row gets them; k <= K)
template <typename T, int LANES, int K, bool VEC>
__device__ __forceinline__ void pick_row(const T* row, int32_t n_experts, int k, bool normalize, int sub, int32_t* expert, float* weight) {
    Best<K> best;
    each<T, LANES, VEC>(row, n_experts, sub, [&](float v, uint32_t e) { best.take(v, e); });
    float top = 0.f, sum = 0.f;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const uint64_t mine = key_of(best.v[0], best.e[0]);
        const uint64_t most = reduce<LANES>(mine, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
        const uint32_t hi = (uint32_t)(most >> 32);
        const float v = __uint_as_float(hi & 0x80000000u ? hi & 0x7fffffffu : ~hi);
        if (most != 0 && most == mine) {   // the lane that had it goes on to its next
#pragma unroll
            for (int i = 0; i + 1 < K; ++i) { best.v[i] = best.v[i + 1]; best.e[i] = best.e[i + 1]; }
            best.v[K - 1] = -INFINITY;
        }
        if (j == 0) top = v;
        expert[j] = most == 0 ? -1 : (int32_t)~(uint32_t)most;
        weight[j] = most == 0 ? 0.f : expf(v - top);
        if (j < k) sum += weight[j];
    }
    if (!normalize && expert[0] >= 0) {
        float part = 0.f;
        each<T, LANES, VEC>(row, n_experts, sub, [&](float v, uint32_t) { part += expf(v - top); });
        sum = reduce<LANES>(part, [](float a, float b) { return a + b; });
    }
#pragma unroll
    for (int j = 0; j < K; ++j) weight[j] = expert[j] < 0 ? 0.f : weight[j] / sum;
}

struct RouteArgs {
    const void* logits;
    int64_t n, stride;
    int32_t n_experts, k, normalize;
    int32_t chunk, n_chunks;   // rows a chunk of the counts
    int32_t* experts;
    float* weights;
    int32_t* offsets;
    int32_t* order;
    int32_t* slots;
    int32_t* counts;           // [n_chunks, n_experts]
    int32_t* totals;           // [n_experts]
};

template <typename T, int LANES, int K, bool VEC>
__global__ void __launch_bounds__(kPickThreads) k_route_pick(RouteArgs p) {
    extern __shared__ int32_t tally[];
    const int tid = threadIdx.x, sub = tid % LANES;
    for (int32_t e = tid; e < p.n_experts; e += kPickThreads) tally[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * p.chunk, stop = first + p.chunk < p.n ? first + p.chunk : p.n;
    for (int64_t i = first + tid / LANES; i < stop; i += kPickThreads / LANES) {
        int32_t expert[K];
        float weight[K];
        pick_row<T, LANES, K, VEC>((const T*)p.logits + i * p.stride, p.n_experts, p.k, p.normalize, sub, expert, weight);
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (j < p.k && sub == j % LANES) {
                p.experts[i * p.k + j] = expert[j];
                p.weights[i * p.k + j] = weight[j];
                if (expert[j] >= 0) atomicAdd(&tally[expert[j]], 1);
            }
    }
    __syncthreads();
    for (int32_t e = tid; e < p.n_experts; e += kPickThreads) p.counts[(int64_t)blockIdx.x * p.n_experts + e] = tally[e];
}

// 16 experts a workgroup, the chunks cut into 64 runs
static __global__ void __launch_bounds__(kScanThreads) k_route_scan(RouteArgs p) {
    __shared__ int32_t part[kScanThreads / kScanColumns][kScanColumns];
    constexpr int runs = kScanThreads / kScanColumns;
    const int col = threadIdx.x % kScanColumns, run = threadIdx.x / kScanColumns;
    const int32_t e = blockIdx.x * kScanColumns + col, length = (p.n_chunks + runs - 1) / runs;
    const int32_t from = run * length, to = from + length < p.n_chunks ? from + length : p.n_chunks;
    int32_t sum = 0;
    if (e < p.n_experts)
#pragma unroll 8
        for (int32_t c = from; c < to; ++c) sum += p.counts[(int64_t)c * p.n_experts + e];
    part[run][col] = sum;
    __syncthreads();
    if (e >= p.n_experts) return;
    int32_t before = 0;
    for (int r = 0; r < run; ++r) before += part[r][col];
    for (int32_t c = from; c < to; c += 8) {
        int32_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < to ? p.counts[(int64_t)(c + j) * p.n_experts + e] : 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < to) {
                p.counts[(int64_t)(c + j) * p.n_experts + e] = before;
                before += v[j];
            }
    }
    if (run == runs - 1) p.totals[e] = before;
}

// The number of lower lanes with the same expert, and whether this is the last lane with it
__device__ __forceinline__ int rank_among(int32_t expert, bool there, int bits, int lane, bool& last) {
    uint64_t same = __ballot(there);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((expert >> b) & 1);
        same &= (expert >> b) & 1 ? set : ~set;
    }
    last = (same >> lane) == 1;
    return __popcll(same & ((1ull << lane) - 1));
}

__device__ __forceinline__ int32_t lanes_inclusive(int32_t v, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// slots first .. stop into their experts' places; next[e]: the first free place of expert e (one wavefront); experts[s]: of slot s
__device__ __forceinline__ void place_slots(const RouteArgs& p, const int32_t* experts, int64_t first, int64_t stop, int32_t* next, int lane) {
    const int bits = 32 - __clz(p.n_experts);
    int32_t ahead = first + lane < stop ? experts[first + lane] : -1;
    for (int64_t s0 = first; s0 < stop; s0 += 64) {
        const int64_t s = s0 + lane;
        const int32_t expert = ahead;
        ahead = s + 64 < stop ? experts[s + 64] : -1;
        const bool there = expert >= 0;
        bool last;
        const int rank = rank_among(there ? expert : 0, there, bits, lane, last);
        const int32_t base = there ? next[expert] : 0;
        __builtin_amdgcn_wave_barrier();
        if (there && last) next[expert] = base + rank + 1;
        __builtin_amdgcn_wave_barrier();
        if (there) p.order[base + rank] = (int32_t)s;
        if (s < stop) p.slots[s] = there ? base + rank : -1;
    }
}

// WAVES wavefronts a chunk, each a run of its slots: they count theirs first, so that each knows where its own begin
template <int WAVES>
__global__ void __launch_bounds__(64 * WAVES) k_route_place(RouteArgs p) {
    extern __shared__ int32_t next[];   // [WAVES][n_experts]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t all = p.n * p.k, chunk_first = (int64_t)blockIdx.x * p.chunk * p.k;
    const int64_t chunk_stop = chunk_first + (int64_t)p.chunk * p.k < all ? chunk_first + (int64_t)p.chunk * p.k : all;
    const int64_t length = (((chunk_stop - chunk_first) + WAVES - 1) / WAVES + 63) / 64 * 64;
    const int64_t first = chunk_first + wave * length < chunk_stop ? chunk_first + wave * length : chunk_stop;
    const int64_t stop = first + length < chunk_stop ? first + length : chunk_stop;
    if (WAVES > 1) {
        for (int32_t e = threadIdx.x; e < WAVES * p.n_experts; e += 64 * WAVES) next[e] = 0;
        __syncthreads();
#pragma unroll 4
        for (int64_t s = first + lane; s < stop; s += 64) {
            const int32_t expert = p.experts[s];
            if (expert >= 0) atomicAdd(&next[wave * p.n_experts + expert], 1);
        }
        __syncthreads();
    }
    // every wavefront adds the totals up by itself, 64 experts at a time, and the first one turns counts into places
    int32_t before = 0;
    for (int32_t e0 = 0; e0 < p.n_experts; e0 += 64) {
        const int32_t e = e0 + lane, total = e < p.n_experts ? p.totals[e] : 0;
        const int32_t upto = before + lanes_inclusive(total, lane);
        if (e < p.n_experts && wave == 0) {
            int32_t place = upto - total + p.counts[(int64_t)blockIdx.x * p.n_experts + e];
            if (WAVES == 1) next[e] = place;
            else
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const int32_t mine = next[w * p.n_experts + e];
                    next[w * p.n_experts + e] = place;
                    place += mine;
                }
            if (blockIdx.x == 0) p.offsets[e] = upto - total;
        }
        before = __shfl(upto, 63);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) p.offsets[p.n_experts] = before;
    for (int64_t s = first + lane; s < stop; s += 64)
        if (s >= before) p.order[s] = -1;   // places that no slot takes
    __syncthreads();
    place_slots(p, p.experts, first, stop, next + wave * p.n_experts, lane);
}

constexpr int kSmallThreads = 1024;
// The end of a call that one workgroup does: counts of the experts in `next` to places and offsets, by its first wavefront
__device__ __forceinline__ void place_few(const RouteArgs& p, int32_t* next, const int32_t* slots, int tid) {
    if (tid >= 64) return;
    const int lane = tid;
    int32_t before = 0;
    for (int32_t e0 = 0; e0 < p.n_experts; e0 += 64) {
        const int32_t e = e0 + lane, total = e < p.n_experts ? next[e] : 0;
        const int32_t upto = before + lanes_inclusive(total, lane);
        if (e < p.n_experts) { next[e] = upto - total; p.offsets[e] = upto - total; }
        before = __shfl(upto, 63);
    }
    if (lane == 0) p.offsets[p.n_experts] = before;
    for (int64_t s = before + lane; s < p.n * p.k; s += 64) p.order[s] = -1;
    __builtin_amdgcn_wave_barrier();
    place_slots(p, slots, 0, p.n * p.k, next, lane);
}

template <typename T, int LANES, int K, bool VEC>
__global__ void __launch_bounds__(kSmallThreads) k_route_small(RouteArgs p) {
    extern __shared__ int32_t next[];   // [n_experts], behind it the experts of the slots [n k]
    int32_t* slots = next + p.n_experts;
    const int tid = threadIdx.x, sub = tid % LANES;
    for (int32_t e = tid; e < p.n_experts; e += kSmallThreads) next[e] = 0;
    __syncthreads();
    for (int64_t i = tid / LANES; i < p.n; i += kSmallThreads / LANES) {
        int32_t expert[K];
        float weight[K];
        pick_row<T, LANES, K, VEC>((const T*)p.logits + i * p.stride, p.n_experts, p.k, p.normalize, sub, expert, weight);
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (j < p.k && sub == j % LANES) {
                p.experts[i * p.k + j] = expert[j];
                p.weights[i * p.k + j] = weight[j];
                slots[i * p.k + j] = expert[j];
                if (expert[j] >= 0) atomicAdd(&next[expert[j]], 1);
            }
    }
    __syncthreads();
    place_few(p, next, slots, tid);
}

struct RouteGradientArgs {
    const void* logits;
    int64_t n, stride;
    int32_t n_experts, k, normalize;
    const int32_t* experts;
    const float* weights;
    const float* dweights;
    void* dlogits;             // [n, n_experts]
};

// 16 bytes, or one element, past the caches: a later kernel reads them (a million rows of 256: 273 -> 226 us)
template <typename T, bool VEC>
__device__ __forceinline__ void store_chunk(T* to, const T* part) {
    typedef uint32_t Word __attribute__((ext_vector_type(4)));
    if (VEC) __builtin_nontemporal_store(*(const Word*)part, (Word*)to);
    else *to = part[0];
}

// dl_e = w_e (dw_e - sum w dw) on the chosen, and -p_e sum w dw on the others where the weights are those of all experts
template <typename T, int LANES, int K, bool VEC>
__global__ void __launch_bounds__(256) k_route_gradient(RouteGradientArgs p) {
    const int sub = threadIdx.x % LANES;
    const int64_t i = block_number() * (256 / LANES) + threadIdx.x / LANES;
    if (i >= p.n) return;   // (whole rows leave; the others' lanes stay together)
    constexpr int epc = VEC ? 16 / (int)sizeof(T) : 1;
    int32_t expert[K];
    float weight[K], given[K], inner = 0.f;
#pragma unroll
    for (int j = 0; j < K; ++j) {   // (all loads at once, no branches: their way is what a row takes)
        const int64_t at = i * p.k + (j < p.k ? j : 0);
        expert[j] = p.experts[at];
        weight[j] = p.weights[at];
        given[j] = p.dweights[at];
    }
#pragma unroll
    for (int j = 0; j < K; ++j) {
        if (j >= p.k) expert[j] = -1;
        weight[j] = expert[j] < 0 ? 0.f : weight[j];
        given[j] = expert[j] < 0 ? 0.f : given[j];
        inner += weight[j] * given[j];
    }
    T* out = (T*)p.dlogits + i * p.n_experts;
    if (p.normalize || expert[0] < 0) {
#pragma unroll
        for (int j = 0; j < K; ++j) given[j] = weight[j] * (given[j] - inner);
        for (int32_t c = sub * epc; c < p.n_experts; c += LANES * epc) {
            T part[epc];
#pragma unroll
            for (int t = 0; t < epc; ++t) {
                float v = 0.f;
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (expert[j] == c + t) v = given[j];
                part[t] = (T)v;
            }
            store_chunk<T, VEC>(out + c, part);
        }
        return;
    }
    const T* row = (const T*)p.logits + i * p.stride;
    float top = -INFINITY, sum = 0.f;
    each<T, LANES, VEC>(row, p.n_experts, sub, [&](float v, uint32_t) { top = fmaxf(top, v); });
    top = reduce<LANES>(top, [](float a, float b) { return fmaxf(a, b); });
    each<T, LANES, VEC>(row, p.n_experts, sub, [&](float v, uint32_t) { sum += expf(v - top); });
    sum = reduce<LANES>(sum, [](float a, float b) { return a + b; });
    for (int32_t c = sub * epc; c < p.n_experts; c += LANES * epc) {
        T in[epc], part[epc];
        if (VEC) *(uint4*)in = *(const uint4*)(row + c);
        else in[0] = row[c];
#pragma unroll
        for (int t = 0; t < epc; ++t) {
            float v = -inner;
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (expert[j] == c + t) v += given[j];
            part[t] = (T)(expf(value_of(in[t]) - top) / sum * v);
        }
        store_chunk<T, VEC>(out + c, part);
    }
}

// ---- the weighted sum over a row's slots

struct CombineArgs {
    const void* values;        // [n_values, d]
    int64_t values_stride, n_values;
    const int32_t* slots;      // [n, k]
    const float* weights;      // [n, k] or NULL: ones
    int64_t n;
    int32_t k, d;
    void* y;                   // [n, d]
    // gradient
    const void* dy;
    int64_t dy_stride;
    const int32_t* order;      // [n k] or NULL
    void* dvalues;             // [n_values, d]
    float* dweights;           // [n, k]
};

template <typename T, int LANES, int VEC>
__global__ void __launch_bounds__(256) k_combine(CombineArgs p) {
    const int sub = threadIdx.x % LANES;
    const int64_t i = block_number() * (256 / LANES) + threadIdx.x / LANES;
    if (i >= p.n) return;
    for (int32_t c = sub * VEC; c < p.d; c += LANES * VEC) {
        float sum[VEC];
#pragma unroll
        for (int t = 0; t < VEC; ++t) sum[t] = 0.f;
#pragma unroll 2
        for (int j = 0; j < p.k; ++j) {
            const int32_t slot = p.slots[i * p.k + j];
            if (slot < 0 || slot >= p.n_values) continue;
            const float w = p.weights ? p.weights[i * p.k + j] : 1.f;
            struct alignas(VEC * sizeof(T)) Part { T v[VEC]; };
            const Part part = *(const Part*)((const T*)p.values + slot * p.values_stride + c);
#pragma unroll
            for (int t = 0; t < VEC; ++t) sum[t] += w * (float)part.v[t];
        }
        struct alignas(VEC * sizeof(T)) Part { T v[VEC]; } out;
#pragma unroll
        for (int t = 0; t < VEC; ++t) out.v[t] = (T)sum[t];
        *(Part*)((T*)p.y + i * p.d + c) = out;
    }
}

// dv_slot = w dy_i, dw = dy_i . v_slot; the places i k .. i k + k - 1 that no slot takes get zeros
template <typename T, int LANES, int VEC>
__global__ void __launch_bounds__(256) k_combine_gradient(CombineArgs p) {
    const int sub = threadIdx.x % LANES;
    const int64_t i = block_number() * (256 / LANES) + threadIdx.x / LANES;
    if (i >= p.n) return;
    struct alignas(VEC * sizeof(T)) Part { T v[VEC]; };
    const T* dy = (const T*)p.dy + i * p.dy_stride;
    for (int j = 0; j < p.k; ++j) {
        const int32_t slot = p.slots[i * p.k + j];
        const bool there = slot >= 0 && slot < p.n_values;
        const float w = p.weights ? p.weights[i * p.k + j] : 1.f;
        float dot = 0.f;
        if (there)
            for (int32_t c = sub * VEC; c < p.d; c += LANES * VEC) {
                const Part g = *(const Part*)(dy + c);
                if (p.dvalues) {
                    Part out;
#pragma unroll
                    for (int t = 0; t < VEC; ++t) out.v[t] = (T)(w * (float)g.v[t]);
                    *(Part*)((T*)p.dvalues + (int64_t)slot * p.d + c) = out;
                }
                if (p.dweights) {
                    const Part v = *(const Part*)((const T*)p.values + slot * p.values_stride + c);
#pragma unroll
                    for (int t = 0; t < VEC; ++t) dot += (float)g.v[t] * (float)v.v[t];
                }
            }
        if (p.dweights) {
            dot = reduce<LANES>(dot, [](float a, float b) { return a + b; });
            if (sub == 0) p.dweights[i * p.k + j] = dot;
        }
        const int64_t place = i * p.k + j;
        if (p.dvalues && p.order && place < p.n_values && p.order[place] < 0)
            for (int32_t c = sub * VEC; c < p.d; c += LANES * VEC) *(Part*)((T*)p.dvalues + place * p.d + c) = Part{};
    }
}

}  // namespace nomad_router
