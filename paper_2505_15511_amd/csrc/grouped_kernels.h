// Matrix products over groups of rows for gfx950: every group has its own weights and any number of rows.
//
//   product           y_p = act(x_row(p) W_e^T + b_e)        for o_e <= p < o_{e+1}
//   weight gradient   dW_e = sum_p dy_p^T x_row(p),  db_e = sum_p dy_p
//
// Both are tiles of C[b][a] = sum_k A[a][k] B[b][k] with a running along the result's contiguous columns: a lane of a 16x16
// matrix instruction ends up with four neighbouring values of a, one 8- or 16-byte store.  Product: a = columns of W's rows,
// b = rows p, k = columns of x.  Weight gradient: a = columns of x, b = columns of dy, k = rows p of the group.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace nomad_grouped {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

enum Activation { kNone = 0, kRelu = 1, kSilu = 2, kGelu = 3 };

// Workgroup number of a launch with more of them than one dimension takes (grid_of)
__device__ __forceinline__ int64_t block_number() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// ---- element types: 16 bytes are one fragment of a matrix step (two or four instructions' worth for float32)

template <typename T> struct Elem;
template <> struct Elem<__bf16> {
    static __device__ __forceinline__ f32x4 mma(uint4 a, uint4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint4 ones() { return make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u); }
};
template <> struct Elem<_Float16> {
    static __device__ __forceinline__ f32x4 mma(uint4 a, uint4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint4 ones() { return make_uint4(0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u); }
};
// float32: four steps of four k each; lane group g holds k = 4 g + t of step t in both operands, so the order of k differs from
// the columns' but is the same on either side
template <> struct Elem<float> {
    static __device__ __forceinline__ f32x4 mma(uint4 a, uint4 b, f32x4 c) {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int t = 0; t < 4; ++t) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[t], y[t], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ uint4 ones() { return make_uint4(0x3f800000u, 0x3f800000u, 0x3f800000u, 0x3f800000u); }
};

template <typename T>
__device__ __forceinline__ float to_f32(T v) { return (float)v; }

__device__ __forceinline__ float activate(float z, int act) {
    if (act == kRelu) return z < 0.f ? 0.f : z;                       // (a NaN stays one)
    if (act == kSilu) return z / (1.f + __expf(-z));
    if (act == kGelu) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    return z;
}
__device__ __forceinline__ float activation_slope(float z, int act) {
    if (act == kRelu) return z > 0.f ? 1.f : (z != z ? z : 0.f);
    if (act == kSilu) {
        const float s = 1.f / (1.f + __expf(-z));
        return s + z * s * (1.f - s);
    }
    if (act == kGelu) return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * 0.39894228040143268f * __expf(-0.5f * z * z);
    return 1.f;
}

// ---- the groups' work items

// Items of a launch: group e has ceil(its rows / step) of them (at least `least`), and one group behind the last stands for the
// rows that belong to no group.  Every wavefront finds the item of its workgroup by itself, 64 groups at a time.
struct Item {
    int64_t begin, end;   // rows of the group
    int32_t group;        // n_groups: rows of no group
    int32_t index;        // of this item among the group's
    int32_t first;        // items before this group's
    int32_t total;        // items of all groups
};

__device__ __forceinline__ int64_t group_end(const int32_t* offsets, int32_t e, int32_t n_groups, int64_t rows) {   // (whatever the offsets hold, rows stay in range)
    if (e > n_groups) return rows;
    const int64_t o = offsets[e];
    return o < 0 ? 0 : o > rows ? rows : o;
}

__device__ __forceinline__ int32_t wave_inclusive(int32_t v, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

__device__ __forceinline__ int32_t group_items(int64_t begin, int64_t end, int32_t step, int32_t least, bool tail) {
    const int64_t count = end > begin ? end - begin : 0;
    const int32_t items = (int32_t)((count + step - 1) / step);
    return tail ? items : items < least ? least : items;
}

// Item number `at` of the list (total alone, and group -1, where at is beyond it)
__device__ __forceinline__ int32_t count_items(const int32_t* offsets, int32_t n_groups, int64_t rows, int32_t step, int32_t least, bool tail, int lane) {
    const int32_t groups = n_groups + (tail ? 1 : 0);
    int32_t total = 0;
    for (int32_t g0 = 0; g0 < groups; g0 += 64) {
        const int32_t e = g0 + lane;
        int32_t items = 0;
        if (e < groups) items = group_items(group_end(offsets, e, n_groups, rows), group_end(offsets, e + 1, n_groups, rows), step, least, e == n_groups);
        total += __shfl(wave_inclusive(items, lane), 63);
    }
    return total;
}
__device__ __forceinline__ Item find_item(const int32_t* offsets, int32_t n_groups, int64_t rows, int32_t step, int32_t least, bool tail, int32_t at, int lane) {
    const int32_t groups = n_groups + (tail ? 1 : 0);
    Item it;
    it.group = -1;
    int32_t before = 0;
    for (int32_t g0 = 0; g0 < groups; g0 += 64) {
        const int32_t e = g0 + lane;
        int64_t begin = 0, end = 0;
        int32_t items = 0;
        if (e < groups) {
            begin = group_end(offsets, e, n_groups, rows);
            end = group_end(offsets, e + 1, n_groups, rows);
            items = group_items(begin, end, step, least, e == n_groups);
        }
        const int32_t upto = before + wave_inclusive(items, lane);
        const uint64_t mask = __ballot(upto > at);
        if (mask) {
            const int who = __builtin_ctzll(mask);
            it.group = g0 + who;
            it.begin = __shfl(begin, who);
            it.end = __shfl(end, who);
            if (it.end < it.begin) it.end = it.begin;
            it.first = __shfl(upto - items, who);
            it.index = at - it.first;
            break;
        }
        before = __shfl(upto, 63);
    }
    return it;
}

// ---- operands: a tile of TILE rows and 128 bytes of k, in LDS, from global memory

__device__ const uint4 kZeros[1] = {{0, 0, 0, 0}};   // what a lane reads whose chunk lies outside (it is written to LDS by the load itself)

constexpr int kStepBytes = 128;   // of k a stage holds
constexpr int kTileChunks = kStepBytes / 16;

// LDS holds 16-byte chunks.  KC (k is contiguous in memory): rows of 8 chunks, chunk c of row r at place c ^ ((r >> 1) & 7).
// Otherwise (the tile's own index is contiguous): k rows of TILE elements; a matrix fragment takes 16 elements of several k rows at
// once, 32 bytes (64 for float32) each, so those units are spread by k.
template <typename T, int TILE, bool KC>
__device__ __forceinline__ int chunk_twist(int row) {
    if (KC) return (row >> 1) & 7;
    constexpr int units = TILE * (int)sizeof(T) / (sizeof(T) == 4 ? 64 : 32);   // of a k row
    constexpr int mask = units >= 8 ? 7 : units - 1;
    if (sizeof(T) == 4) return ((row >> 2) & mask) << 2;
    return (((row & 3) | ((row >> 1) & 4)) & mask) << 1;
}

// Where a tile comes from: rows of `length` elements; row r of the source is base + r * stride, or, gathered,
// base + (order[r] / per_row) * stride, and zeros where that is no row.
struct Source {
    const void* base;
    int64_t stride;        // elements
    const int32_t* order;  // NULL: rows as they are
    int64_t rows;          // of the source, where gathered
    uint32_t per_row;
    __device__ __forceinline__ int64_t row_of(int64_t p) const {
        if (!order) return p;
        const int32_t slot = order[p];
        if (slot < 0) return -1;
        const int64_t r = per_row == 1 ? (uint32_t)slot : (uint32_t)slot / per_row;
        return r < rows ? r : -1;
    }
};

// TILE rows (KC) or columns (not KC) by one stage of k, for NT threads.  ASYNC: loads go to LDS directly, whole 16-byte chunks;
// otherwise through registers, element by element where a chunk is cut off.
template <typename T, int TILE, bool KC, bool ASYNC, int NT>
struct Operand {
    static constexpr int kEpc = 16 / (int)sizeof(T);             // elements a chunk
    static constexpr int kBk = kStepBytes / (int)sizeof(T);      // k of a stage
    static constexpr int kCpr = KC ? kTileChunks : TILE / kEpc;  // chunks a row of LDS
    static constexpr int kChunks = TILE * kTileChunks;           // of a stage
    static constexpr int kPer = (kChunks + NT - 1) / NT;         // a thread
    static constexpr bool kWhole = kChunks % NT == 0;
    const T* row[KC ? kPer : 1];   // KC: the thread's rows (NULL: none)
    Source src;
    int64_t first;                 // not KC: the source row of k = 0
    int32_t across;                // not KC: columns before the tile
    int32_t limit;                 // k there are (KC: of every row)
    int32_t width;                 // not KC: columns there are, from the tile's first
    uint4 held[ASYNC ? 1 : kPer];

    __device__ __forceinline__ static bool has(int it, int tid) { return kWhole || it * NT + tid < kChunks; }

    // KC: rows first_row .. of the source, `count` of them; k < k_limit
    __device__ __forceinline__ void open_rows(const Source& s, int64_t first_row, int64_t count, int32_t k_limit, int tid) {
        src = s;
        limit = k_limit;
#pragma unroll
        for (int it = 0; it < kPer; ++it) {
            const int r = (it * NT + tid) / kCpr;
            row[KC ? it : 0] = nullptr;
            if (has(it, tid) && r < count) {
                const int64_t at = s.row_of(first_row + r);
                if (at >= 0) row[KC ? it : 0] = (const T*)s.base + at * s.stride;
            }
        }
    }
    // not KC: columns from `column` on (`columns` in all), k = source rows first_k ..
    __device__ __forceinline__ void open_columns(const Source& s, int64_t first_k, int32_t k_limit, int32_t column, int32_t columns) {
        src = s;
        first = first_k;
        limit = k_limit;
        across = column;
        width = columns - column;
    }
    __device__ __forceinline__ void chunk(int it, int tid, int32_t k0, const T*& from, int& elements) const {
        const int l = it * NT + tid, r = l / kCpr, c = (l % kCpr) ^ chunk_twist<T, TILE, KC>(r);
        if (KC) {
            const int32_t k = k0 + c * kEpc;
            from = row[KC ? it : 0] + k;
            elements = row[KC ? it : 0] ? limit - k : 0;
        } else {
            const int32_t k = k0 + r;
            const int64_t at = k < limit ? src.row_of(first + k) : -1;
            from = (const T*)src.base + at * src.stride + across + c * kEpc;
            elements = at >= 0 ? width - c * kEpc : 0;
        }
    }
    // asks for the stage that begins at k0
    __device__ __forceinline__ void ask(uint4* lds, int32_t k0, int tid) {
#pragma unroll
        for (int it = 0; it < kPer; ++it) {
            if (!has(it, tid)) continue;   // (kChunks is a multiple of 64: whole wavefronts)
            const T* from;
            int elements;
            chunk(it, tid, k0, from, elements);
            if (ASYNC) {
                const void* p = elements > 0 ? (const void*)from : (const void*)kZeros;
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)p,
                                                 (__attribute__((address_space(3))) uint32_t*)(lds + it * NT + (tid & ~63)), 16, 0, 0);
            } else {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (elements >= kEpc) {
                    __builtin_memcpy(&v, from, 16);   // (aligned as an element is)
                } else if (elements > 0) {
                    T part[kEpc] = {};
#pragma unroll
                    for (int i = 0; i < kEpc; ++i)
                        if (i < elements) part[i] = from[i];
                    __builtin_memcpy(&v, part, 16);
                }
                held[ASYNC ? 0 : it] = v;
            }
        }
    }
    // puts down what was asked for, where the loads did not
    __device__ __forceinline__ void put(uint4* lds, int tid) const {
        if (ASYNC) return;
#pragma unroll
        for (int it = 0; it < kPer; ++it)
            if (has(it, tid)) lds[it * NT + tid] = held[ASYNC ? 0 : it];
    }
    // fragment of the 16 rows (columns) from `at` on, matrix step s of the stage's two
    static __device__ __forceinline__ uint4 fragment(const uint4* lds, int at, int s, int lane) {
        const int g = lane >> 4, i = lane & 15;
        if (KC) {
            const int r = at + i;
            return lds[r * kTileChunks + ((s * 4 + g) ^ chunk_twist<T, TILE, KC>(r))];
        }
        if (sizeof(T) == 4) {
            uint4 v;
            uint32_t* out = (uint32_t*)&v;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int k = s * 16 + 4 * g + t, e = at + i;
                out[t] = ((const uint32_t*)lds)[(k * kCpr + ((e >> 2) ^ chunk_twist<T, TILE, KC>(k))) * 4 + (e & 3)];
            }
            return v;
        }
        // four k rows of 16 elements, turned on the way: lane i of the group gets element i of the four rows
        union { i16x4 half[2]; uint4 whole; } v;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = s * 32 + 8 * g + 4 * h + (i >> 2), e = at + 4 * (i & 3);
            const int c = (e >> 3) ^ chunk_twist<T, TILE, KC>(k);
            v.half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)((const char*)(lds + k * kCpr + c) + (e & 4) * 2));
        }
        return v.whole;
    }
};

// ---- a tile of the result

template <typename T, int TA, int TB, int WA, int WB, bool A_KC, bool B_KC, bool ASYNC>
struct Tile {
    static constexpr int kNt = 64 * WA * WB;
    static constexpr int kFa = TA / WA / 16, kFb = TB / WB / 16;
    static constexpr int kBk = kStepBytes / (int)sizeof(T);
    typedef Operand<T, TA, A_KC, ASYNC, kNt> A;
    typedef Operand<T, TB, B_KC, ASYNC, kNt> B;
    f32x4 acc[kFa][kFb];

    // acc = sum over k < limit; with SUMS also the sums of B alone over k
    template <bool SUMS>
    __device__ __forceinline__ void run(A& a, B& b, uint4* a0, uint4* b0, uint4* a1, uint4* b1, int32_t limit, f32x4* sums, int tid) {
        const int lane = tid & 63, wave = tid >> 6, wa = (wave % WA) * (TA / WA), wb = (wave / WA) * (TB / WB);
#pragma unroll
        for (int x = 0; x < kFa; ++x)
#pragma unroll
            for (int y = 0; y < kFb; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
        const auto step = [&](const uint4* la, const uint4* lb) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                uint4 fa[kFa], fb[kFb];
#pragma unroll
                for (int x = 0; x < kFa; ++x) fa[x] = A::fragment(la, wa + 16 * x, s, lane);
#pragma unroll
                for (int y = 0; y < kFb; ++y) fb[y] = B::fragment(lb, wb + 16 * y, s, lane);
#pragma unroll
                for (int x = 0; x < kFa; ++x)
#pragma unroll
                    for (int y = 0; y < kFb; ++y) acc[x][y] = Elem<T>::mma(fa[x], fb[y], acc[x][y]);
                if (SUMS)
#pragma unroll
                    for (int y = 0; y < kFb; ++y) sums[y] = Elem<T>::mma(Elem<T>::ones(), fb[y], sums[y]);
            }
        };
        // every wavefront's loads have landed, then all have arrived (a barrier alone does not wait for loads to LDS)
        const auto meet = [&]() {
            if (ASYNC) __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
            __syncthreads();
        };
        if (limit <= 0) return;
        a.ask(a0, 0, tid);
        b.ask(b0, 0, tid);
        a.put(a0, tid);
        b.put(b0, tid);
        meet();
        // two stages a round, so that each has its own half of LDS by name: loads into one go on under the products of the other
        for (int32_t k = 0;;) {
            if (k + kBk < limit) { a.ask(a1, k + kBk, tid); b.ask(b1, k + kBk, tid); }
            step(a0, b0);
            if ((k += kBk) >= limit) break;
            a.put(a1, tid);
            b.put(b1, tid);
            meet();
            if (k + kBk < limit) { a.ask(a0, k + kBk, tid); b.ask(b0, k + kBk, tid); }
            step(a1, b1);
            if ((k += kBk) >= limit) break;
            a.put(a0, tid);
            b.put(b0, tid);
            meet();
        }
    }
};

struct ProductArgs {
    const int32_t* offsets;
    Source x;
    const void* w;
    int64_t w_group, w_stride;   // elements between groups, between rows of the contiguous direction
    const void* bias;
    int64_t bias_stride;
    const void* slope_at;        // z of the activation whose slope multiplies the result; NULL: activation itself
    int64_t slope_stride;
    void* y;
    int64_t y_stride;
    void* z_out;
    int64_t z_stride;
    int64_t rows;
    int32_t n_groups, in, out, activation;
    int32_t whole_stores;        // y, z_out and slope_at take four columns at a time
};

template <typename O>
__device__ __forceinline__ void store4(O* to, const float* v, int n, bool whole) {
    if (whole) {
        O part[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) part[i] = (O)v[i];
        struct alignas(4 * sizeof(O)) Four { O v[4]; };
        *(Four*)to = *(Four*)part;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) to[i] = (O)v[i];
    }
}

// y = act(x W^T + b), or (x W^T) act'(z).  One workgroup a tile of TB rows and TA columns; consecutive workgroups of an XCD take
// the column tiles of one row tile after the other, so that x is read from memory once and a group's weights stay in its L2.
template <typename T, typename O, int TA, int TB, int WA, int WB, bool W_KC, bool ASYNC>
__global__ void __launch_bounds__(64 * WA * WB) k_grouped_product(ProductArgs p) {
    typedef Tile<T, TA, TB, WA, WB, W_KC, true, ASYNC> Work;
    __shared__ uint4 a0[TA * kTileChunks], a1[TA * kTileChunks], b0[TB * kTileChunks], b1[TB * kTileChunks];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t across = (p.out + TA - 1) / TA;
    const int64_t total = (int64_t)count_items(p.offsets, p.n_groups, p.rows, TB, 0, true, lane) * across;
    const int64_t block = block_number();
    const int64_t per = (total + 7) / 8, turn = block >> 3;
    const int64_t at = (block & 7) * per + turn;
    if (turn >= per || at >= total) return;
    const Item it = find_item(p.offsets, p.n_groups, p.rows, TB, 0, true, (int32_t)(at / across), lane);
    const int32_t a_first = (int32_t)(at % across) * TA;
    const int64_t b_first = it.begin + (int64_t)it.index * TB;
    const int32_t count = (int32_t)(it.end - b_first < TB ? it.end - b_first : TB);
    Work work;
    f32x4 none[1];
    if (it.group < p.n_groups) {
        typename Work::A a;
        typename Work::B b;
        const Source w{(const T*)p.w + (int64_t)it.group * p.w_group, p.w_stride, nullptr, 0, 1};
        if (W_KC) a.open_rows(w, a_first, p.out - a_first, p.in, tid);
        else a.open_columns(w, 0, p.in, a_first, p.out);
        b.open_rows(p.x, b_first, count, p.in, tid);
        work.template run<false>(a, b, a0, b0, a1, b1, p.in, none, tid);
    } else {
#pragma unroll
        for (int x = 0; x < Work::kFa; ++x)
#pragma unroll
            for (int y = 0; y < Work::kFb; ++y) work.acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const bool inside = it.group < p.n_groups;
    const int wa = (wave % WA) * (TA / WA), wb = (wave / WA) * (TB / WB), g = lane >> 4, i = lane & 15;
#pragma unroll
    for (int x = 0; x < Work::kFa; ++x) {
        const int32_t col = a_first + wa + 16 * x + 4 * g;
        const int n = p.out - col;
        if (n <= 0) continue;
        const bool whole = p.whole_stores && n >= 4;
        float bias[4] = {0.f, 0.f, 0.f, 0.f};
        if (p.bias && inside) {
            const T* from = (const T*)p.bias + (int64_t)it.group * p.bias_stride + col;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < n) bias[j] = (float)from[j];
        }
#pragma unroll
        for (int y = 0; y < Work::kFb; ++y) {
            const int r = wb + 16 * y + i;
            if (r >= count) continue;
            const int64_t row = b_first + r;
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = work.acc[x][y][j] + bias[j];
            if (inside && p.slope_at) {
                const T* z = (const T*)p.slope_at + row * p.slope_stride + col;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < n) v[j] *= activation_slope((float)z[j], p.activation);
            } else if (inside) {
                if (p.z_out) store4((T*)p.z_out + row * p.z_stride + col, v, n, whole);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = activate(v[j], p.activation);
            } else if (p.z_out) {
                store4((T*)p.z_out + row * p.z_stride + col, v, n, whole);
            }
            store4((O*)p.y + row * p.y_stride + col, v, n, whole);
        }
    }
}

struct GradientArgs {
    const int32_t* offsets;
    Source x, dy;            // x: [.., in], gathered; dy: [rows, out]
    void* dw;                // [n_groups, out, in]
    float* db;               // NULL or [n_groups, out]
    int64_t rows;
    int32_t n_groups, in, out;
    int32_t whole_stores;
};

// dW = sum over the group's rows of dy^T x: one workgroup a tile of TA columns of x and TB of dy.
template <typename T, typename O, int TA, int TB, int WA, int WB, bool ASYNC>
__global__ void __launch_bounds__(64 * WA * WB) k_grouped_gradient(GradientArgs p) {
    typedef Tile<T, TA, TB, WA, WB, false, false, ASYNC> Work;
    __shared__ uint4 a0[TA * kTileChunks], a1[TA * kTileChunks], b0[TB * kTileChunks], b1[TB * kTileChunks];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t across = (p.in + TA - 1) / TA, down = (p.out + TB - 1) / TB;
    const int64_t block = block_number(), tiles = (int64_t)across * down;
    if (block >= p.n_groups * tiles) return;
    const int64_t tile = block % tiles;
    const int32_t group = (int32_t)(block / tiles);
    const int64_t begin = group_end(p.offsets, group, p.n_groups, p.rows), stop = group_end(p.offsets, group + 1, p.n_groups, p.rows);
    const int32_t count = stop > begin ? (int32_t)(stop - begin) : 0;
    const int32_t a_first = (int32_t)(tile % across) * TA, b_first = (int32_t)(tile / across) * TB;
    Work work;
    typename Work::A a;
    typename Work::B b;
    a.open_columns(p.x, begin, count, a_first, p.in);
    b.open_columns(p.dy, begin, count, b_first, p.out);
    f32x4 sums[Work::kFb];
#pragma unroll
    for (int y = 0; y < Work::kFb; ++y) sums[y] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bool bias = p.db && a_first == 0;
    if (bias) work.template run<true>(a, b, a0, b0, a1, b1, count, sums, tid);
    else work.template run<false>(a, b, a0, b0, a1, b1, count, sums, tid);
    const int wa = (wave % WA) * (TA / WA), wb = (wave / WA) * (TB / WB), g = lane >> 4, i = lane & 15;
#pragma unroll
    for (int y = 0; y < Work::kFb; ++y) {
        const int32_t r = b_first + wb + 16 * y + i;
        if (r >= p.out) continue;
        if (bias && wave % WA == 0 && g == 0) p.db[(int64_t)group * p.out + r] = sums[y][0];
#pragma unroll
        for (int x = 0; x < Work::kFa; ++x) {
            const int32_t col = a_first + wa + 16 * x + 4 * g;
            const int n = p.in - col;
            if (n <= 0) continue;
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = work.acc[x][y][j];
            store4((O*)p.dw + ((int64_t)group * p.out + r) * p.in + col, v, n, p.whole_stores && n >= 4);
        }
    }
}

}  // namespace nomad_grouped
