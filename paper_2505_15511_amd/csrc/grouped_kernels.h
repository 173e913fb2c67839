// Matrix products over groups of rows for gfx950: every group has its own weights and any number of rows.
//
//   product           y_p = act(x_row(p) W_e^T + b_e)        for o_e <= p < o_{e+1}
//   weight gradient   dW_e = sum_p dy_p^T x_row(p),  db_e = sum_p dy_p
//
// Both are tiles of C[b][a] = sum_k A[a][k] B[b][k] with a running along the result's contiguous columns.  Product: a = columns
// of W's rows, b = rows p, k = columns of x.  Weight gradient: a = columns of x, b = columns of dy, k = rows p of the group.
//
// A wavefront's share of a tile is made of 16x16 matrix instructions.  Which columns the 16 rows r of an instruction stand for is free: in
// sets of Q instructions, row r of the set's instruction x is column 4 Q (r / 4) + 4 x + r % 4, so that a lane, which holds four
// rows r of every instruction, ends up with 4 Q neighbouring columns of one row of the result.  Q makes that 16 bytes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace nomad_grouped {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

enum Activation { kNone = 0, kRelu = 1, kSilu = 2, kGelu = 3 };

// Workgroup number of a launch with more of them than one dimension takes (grid_of)
__device__ __forceinline__ int64_t block_number() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// ---- element types: 16 bytes are one fragment of a matrix step (one instruction, four for float32)

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

template <int V> struct Constant { static constexpr int value = V; };

// FULL: for results in float32, good to a few units of their last place wherever z lies; the others to 2^-16 of themselves, of which a rounding to
// 16 bits shows nothing.
//
// e^x for x in [-104, 88], the nearer end beyond it (and for a NaN): the hardware's power of two is good to a unit, but its argument x log2(e)
// loses x 2^-24 to rounding, which FULL puts back
template <bool FULL>
__device__ __forceinline__ float exponential(float x) {
    if (!FULL) return __expf(x);
    x = __builtin_amdgcn_fmed3f(x, -104.f, 88.f);
    const float power = x * 1.44269504f, rest = fmaf(x, 1.92596303e-8f, fmaf(x, 1.44269504f, -power)), e = __builtin_amdgcn_exp2f(power);
    return fmaf(e, rest * 0.69314718f, e);
}
template <bool FULL>
__device__ __forceinline__ float bell(float z) {   // e^(-z^2 / 2)
    const float square = z * z, e = exponential<FULL>(-0.5f * square);
    return FULL ? fmaf(e, -0.5f * fmaf(z, z, -square), e) : e;   // (with what the square's rounding lost)
}
template <bool FULL>   // (the hardware's reciprocal: one unit in the last place)
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + exponential<FULL>(-z)); }

// 1 + erf(z / sqrt 2) = erfc(-z / sqrt 2), which below zero is small and keeps its digits this way: erfc(x) = e^(-x^2) t P(t) for x > 0 with
// t = 1 / (1 + 0.4 x), where e^(x^2) erfc(x) / t is smooth from 1 (t = 1) to 0.4 / sqrt(pi) (t -> 0); P fitted to it by least squares of the relative
// error with weights that level its peaks: 1.3e-7 (eighth degree), 4.8e-6 (sixth).  `e`: bell(z)
template <bool FULL>
__device__ __forceinline__ float one_plus_erf(float z, float e) {
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.4f * 0.70710678118654752f, 1.f));
    float tail;
    if (FULL) {
        tail = fmaf(0.050258245f, t, -0.18288736f);
        tail = fmaf(tail, t, 0.16906485f);
        tail = fmaf(tail, t, -0.0055921078f);
        tail = fmaf(tail, t, 0.14142513f);
        tail = fmaf(tail, t, 0.16854335f);
        tail = fmaf(tail, t, 0.20784256f);
        tail = fmaf(tail, t, 0.22566961f);
        tail = fmaf(tail, t, 0.22567587f);
    } else {
        tail = fmaf(-0.095308885f, t, 0.18682611f);
        tail = fmaf(tail, t, 0.068062447f);
        tail = fmaf(tail, t, 0.18213749f);
        tail = fmaf(tail, t, 0.20694368f);
        tail = fmaf(tail, t, 0.22565743f);
        tail = fmaf(tail, t, 0.22567692f);
    }
    tail = tail * t * e;
    return z < 0.f ? tail : 2.f - tail;
}

template <int ACT, bool FULL>
__device__ __forceinline__ float activate(float z) {
    if (ACT == kRelu) return z < 0.f ? 0.f : z;                       // (a NaN stays one)
    if (ACT == kSilu) return z * sigmoid<FULL>(z);
    if (ACT == kGelu) return 0.5f * z * one_plus_erf<FULL>(z, bell<FULL>(z));
    return z;
}
template <int ACT, bool FULL, bool TAIL = FULL>   // TAIL: the longer fit of erfc
__device__ __forceinline__ float activation_slope(float z) {
    if (ACT == kRelu) return z > 0.f ? 1.f : (z != z ? z : 0.f);
    if (ACT == kSilu) {
        const float s = sigmoid<FULL>(z);
        return s + z * s * (1.f - s);
    }
    if (ACT == kGelu) {
        const float e = bell<FULL>(z);
        return 0.5f * one_plus_erf<TAIL>(z, e) + z * 0.39894228040143268f * e;
    }
    return 1.f;
}

// ---- the groups' work items

// Items of a product: group e has ceil(its rows / step) of them, and one group behind the last stands for the rows that belong to
// no group.  Every wavefront finds the item of its workgroup by itself, 64 groups at a time.
struct Item {
    int64_t begin, end;   // rows of the group
    int32_t group;        // n_groups: rows of no group
    int32_t first;        // items before this group's
    int32_t items;        // the group has
};

__device__ __forceinline__ int64_t group_end(const int32_t* offsets, int32_t e, int32_t n_groups, int64_t rows) {   // (whatever the offsets hold, rows stay in range)
    if (e > n_groups) return rows;
    const int64_t o = offsets[e];
    return o < 0 ? 0 : o > rows ? rows : o;
}

// a lane's value for all, in scalar registers (__shfl leaves one in every lane)
__device__ __forceinline__ int32_t of_lane(int32_t v, int who) { return __builtin_amdgcn_readlane(v, who); }
__device__ __forceinline__ int64_t of_lane(int64_t v, int who) {
    return (int64_t)((uint64_t)(uint32_t)of_lane((int32_t)(v >> 32), who) << 32 | (uint32_t)of_lane((int32_t)v, who));
}

__device__ __forceinline__ int32_t wave_inclusive(int32_t v, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

__device__ __forceinline__ int32_t items_of(int64_t begin, int64_t end, int32_t step) { return end > begin ? (int32_t)((end - begin + step - 1) / step) : 0; }

__device__ __forceinline__ int32_t count_items(const int32_t* offsets, int32_t n_groups, int64_t rows, int32_t step, int lane) {
    int32_t mine = 0;
#pragma unroll 4
    for (int32_t e = lane; e <= n_groups; e += 64) mine += items_of(group_end(offsets, e, n_groups, rows), group_end(offsets, e + 1, n_groups, rows), step);
    return of_lane(wave_inclusive(mine, lane), 63);
}
// Item number `at` of the list (group -1 where it is beyond it).  `it`: an item found before, no later than this one, or one with
// group 0 and first 0: the search goes on from its group.
__device__ __forceinline__ void find_item(Item& it, const int32_t* offsets, int32_t n_groups, int64_t rows, int32_t step, int32_t at, int lane) {
    int32_t before = it.first;
    for (int32_t g0 = it.group; g0 <= n_groups; g0 += 64) {
        const int32_t e = g0 + lane;
        int64_t begin = 0, end = 0;
        int32_t items = 0;
        if (e <= n_groups) {
            begin = group_end(offsets, e, n_groups, rows);
            end = group_end(offsets, e + 1, n_groups, rows);
            items = items_of(begin, end, step);
        }
        const int32_t upto = before + wave_inclusive(items, lane);
        const uint64_t mask = __ballot(upto > at);
        if (mask) {
            const int who = __builtin_ctzll(mask);
            it.group = g0 + who;
            it.begin = of_lane(begin, who);
            it.end = of_lane(end, who);
            it.first = of_lane(upto - items, who);
            it.items = of_lane(items, who);
            return;
        }
        before = of_lane(upto, 63);
    }
    it.group = -1;
}

// ---- operands: a tile of TILE rows and 128 bytes of k, in LDS, from global memory

__device__ const uint4 kZeros[1] = {{0, 0, 0, 0}};   // what a lane reads whose chunk lies outside (it is written to LDS by the load itself)

constexpr int kStepBytes = 128;   // of k a stage holds
constexpr int kTileChunks = kStepBytes / 16;

// LDS holds 16-byte chunks.  KC (k is contiguous in memory): rows of 8 chunks.  Otherwise (the tile's own index is contiguous): k rows
// of TILE elements.  Chunk c of row r stands at place c ^ twist(r), so that the lanes that read together meet different banks
// (measured: no conflicts).  Q as above for the operand a; the other one's fragments are 16 neighbours, Q = 1.
constexpr int log2_of(int v) { return v <= 1 ? 0 : 1 + log2_of(v / 2); }

template <typename T, int TILE, bool KC, int Q>
__device__ __forceinline__ int chunk_twist(int row) {
    // lanes read one chunk each of 16 rows: neighbours, or fours of neighbours 4 Q apart
    if (KC) return ((row >> 1) & 1) | ((row >> log2_of(4 * Q)) & 3) << 1;
    // lanes read pieces of the same columns in several k rows: rows k .. k + 3 together (16 bits, turned on the way), or the k
    // of the four lane groups (32 bits).  Bits of the row go to bits of the chunk that the columns leave alone.
    constexpr int chunks = TILE * (int)sizeof(T) / 16, lq = log2_of(Q);
    int t;
    if (sizeof(T) == 4) t = ((row >> 2) & 3) << (lq == 0 ? 2 : 3);                  // 16 neighbours: chunks 0..3; Q = 2: 0, 2, 4, 6
    else if (Q == 1) t = (row & 3) << 1 | ((row >> 3) & 1) << 3;                    // 16 neighbours: chunks 0 and 1
    else t = (row & 3) << 2;                                                        // Q = 2: chunks 0..3
    return t & (chunks - 1);
}

// Where a tile comes from: rows of `length` elements; row r of the source is base + r * stride, or, gathered,
// base + (order[r] / per_row) * stride, and zeros where that is no row.
struct Source {
    const void* base;
    int64_t stride;        // elements
    const int32_t* order;  // NULL: rows as they are
    int64_t rows;          // of the source, where gathered
    uint32_t per_row;
    __device__ __forceinline__ int64_t row_at(int32_t slot) const {   // of an entry of the order; -1: none
        if (slot < 0) return -1;
        const int64_t r = per_row == 1 ? (uint32_t)slot : (uint32_t)slot / per_row;
        return r < rows ? r : -1;
    }
    __device__ __forceinline__ int64_t row_of(int64_t p) const { return order ? row_at(order[p]) : p; }
};

// TILE rows (KC) or columns (not KC) by one stage of k, for NT threads.  PICKED: source rows anywhere (KC: a pointer each; otherwise
// the numbers of 64 rows at a time in a register of the wavefront, the next 64 on their way).  ASYNC: loads go to LDS directly, whole
// 16-byte chunks; otherwise through registers, wherever rows begin and end.
template <typename T, int TILE, bool KC, bool PICKED, int Q, bool ASYNC, int NT>
struct Operand {
    static constexpr int kEpc = 16 / (int)sizeof(T);             // elements a chunk
    static constexpr int kBk = kStepBytes / (int)sizeof(T);      // k of a stage
    static constexpr int kCpr = KC ? kTileChunks : TILE / kEpc;  // chunks a row of LDS
    static constexpr int kChunks = TILE * kTileChunks;           // of a stage
    static constexpr int kPer = (kChunks + NT - 1) / NT;         // a thread
    static constexpr bool kWhole = kChunks % NT == 0;
    const T* row[KC && PICKED ? kPer : 1];   // KC: the thread's rows (picked: NULL where there is none)
    int32_t rows;                  // KC, not picked: rows there are from the thread's first on
    Source src;
    int64_t first;                 // not KC: the place of k = 0
    int32_t across;                // not KC: columns before the tile
    int32_t now, next;             // not KC, picked: source rows of 64 places (-1: none), entries of the order of the 64 behind them
    int32_t limit;                 // k there are (KC: of every row)
    int32_t width;                 // not KC: columns there are, from the tile's first
    uint4 held[ASYNC ? 1 : kPer];

    __device__ __forceinline__ static bool has(int it, int tid) { return kWhole || it * NT + tid < kChunks; }

    // KC: rows first_row .. of the source, `count` of them; k < k_limit
    __device__ __forceinline__ void open_rows(const Source& s, int64_t first_row, int64_t count, int32_t k_limit, int tid) {
        src = s;
        limit = k_limit;
        if (!PICKED) {
            const int r = tid / kCpr;
            row[0] = (const T*)s.base + (first_row + r) * s.stride;
            rows = (int32_t)(count < TILE ? count : TILE) - r;
            return;
        }
#pragma unroll
        for (int it = 0; it < kPer; ++it) {
            const int r = (it * NT + tid) / kCpr;
            row[PICKED ? it : 0] = nullptr;
            if (has(it, tid) && r < count) {
                const int64_t at = s.row_of(first_row + r);
                if (at >= 0) row[PICKED ? it : 0] = (const T*)s.base + at * s.stride;
            }
        }
    }
    // not KC: columns from `column` on (`columns` in all), k = source rows (places of the order) first_k ..
    __device__ __forceinline__ void open_columns(const Source& s, int64_t first_k, int32_t k_limit, int32_t column, int32_t columns, int tid) {
        src = s;
        first = first_k;
        limit = k_limit;
        across = column;
        width = columns - column;
        if (PICKED) next = entry(tid & 63);
        else row[0] = (const T*)s.base + (first_k + tid / kCpr) * s.stride + column;
    }
    __device__ __forceinline__ int32_t entry(int32_t k) const { return k >= limit ? -1 : src.order ? src.order[first + k] : (int32_t)(first + k); }
    __device__ __forceinline__ void chunk(int it, int tid, int32_t k0, const T*& from, int& elements) const {
        const int l = it * NT + tid, r = l / kCpr, c = (l % kCpr) ^ chunk_twist<T, TILE, KC, Q>(r);
        if (KC) {
            const int32_t k = k0 + c * kEpc;
            constexpr int apart = NT / kCpr;   // rows between the thread's chunks
            from = PICKED ? row[PICKED ? it : 0] + k : row[0] + (int64_t)(it * apart) * src.stride + k;
            elements = (PICKED ? row[PICKED ? it : 0] != nullptr : it * apart < rows) ? limit - k : 0;
        } else {
            const int32_t k = k0 + r;
            int64_t at = 0;
            if (PICKED) {
                at = __shfl(now, k & 63);
                from = (const T*)src.base + at * src.stride + across + c * kEpc;
            } else {
                constexpr int apart = NT / kCpr;
                from = row[0] + (int64_t)(k0 + it * apart) * src.stride + c * kEpc;
            }
            elements = k < limit && at >= 0 ? width - c * kEpc : 0;
        }
    }
    // asks for the stage that begins at k0 (stages in their order)
    __device__ __forceinline__ void ask(uint4* lds, int32_t k0, int tid) {
        if (!KC && PICKED && (k0 & 63) == 0) {
            now = (int32_t)src.row_at(next);
            next = entry(k0 + 64 + (tid & 63));
        }
        if (!ASYNC && !KC && shorter()) {
#pragma unroll
            for (int it = 0; it < kPer; ++it) {
                const T* from;
                int elements;
                chunk(it, tid, k0, from, elements);
                held[ASYNC ? 0 : it] = has(it, tid) ? one_by_one(from, elements) : make_uint4(0, 0, 0, 0);
            }
            return;
        }
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
                if (!KC) {
                    if (elements > 0) __builtin_memcpy(&v, from - (elements < kEpc ? kEpc - elements : 0), 16);   // (aligned as an element is)
                } else if (elements >= kEpc) {
                    __builtin_memcpy(&v, from, 16);
                } else if (elements > 0) {
                    v = one_by_one(from, elements);
                }
                held[ASYNC ? 0 : it] = v;
            }
        }
    }
    static __device__ __forceinline__ uint4 one_by_one(const T* from, int elements) {   // (fewer than a chunk)
        T part[kEpc] = {};
#pragma unroll
        for (int i = 0; i < kEpc - 1; ++i)
            if (i < elements) part[i] = from[i];
        uint4 v;
        __builtin_memcpy(&v, part, 16);
        return v;
    }
    __device__ __forceinline__ bool shorter() const { return across + width < kEpc; }   // not KC: whole rows, than a chunk
    // Puts down what was asked for, where the loads did not.  A chunk that is cut off: where k is contiguous that is in the last stage
    // alone, and its elements were loaded one by one; columns are cut off in every row of k, and what is left of a chunk was loaded as the
    // last 16 bytes of its row and moves to its beginning here (200,006 rows of float32, weights' gradient of 129 x 50: 102 us, 133 with
    // elements one by one; products of 64 -> 129 the other way round: 80 us, 89 moved).
    __device__ __forceinline__ void put(uint4* lds, int tid) {
        if (ASYNC) return;
        if (!KC && width < TILE && !shorter()) {
#pragma unroll
            for (int it = 0; it < kPer; ++it) {
                const int l = it * NT + tid, r = l / kCpr, c = (l % kCpr) ^ chunk_twist<T, TILE, KC, Q>(r);
                const int over = (c + 1) * kEpc - width, bytes = (over > 0 && over < kEpc ? over : 0) * (int)sizeof(T);
                uint4& v = held[ASYNC ? 0 : it];
                if (bytes & 8) v = make_uint4(v.z, v.w, 0, 0);
                if (bytes & 4) v = make_uint4(v.y, v.z, v.w, 0);
                if (sizeof(T) == 2 && bytes & 2) v = make_uint4(v.x >> 16 | v.y << 16, v.y >> 16 | v.z << 16, v.z >> 16 | v.w << 16, v.w >> 16);
            }
        }
#pragma unroll
        for (int it = 0; it < kPer; ++it)
            if (has(it, tid)) lds[it * NT + tid] = held[ASYNC ? 0 : it];
    }
    // fragment number x of the rows (columns) from `at` on, matrix step s of the stage's two
    static __device__ __forceinline__ uint4 fragment(const uint4* lds, int at, int x, int s, int lane) {
        const int g = lane >> 4, i = lane & 15;
        const int set = at + 16 * Q * (x / Q) + 4 * (x % Q), four = set + 4 * Q * (i >> 2);   // the first of lane i's four neighbours
        if (KC) {
            const int r = four + (i & 3);
            return lds[r * kTileChunks + ((s * 4 + g) ^ chunk_twist<T, TILE, KC, Q>(r))];
        }
        if (sizeof(T) == 4) {
            uint4 v;
            uint32_t* out = (uint32_t*)&v;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int k = s * 16 + 4 * g + t;
                out[t] = ((const uint32_t*)lds)[(k * kCpr + ((four >> 2) ^ chunk_twist<T, TILE, KC, Q>(k))) * 4 + (i & 3)];
            }
            return v;
        }
        // a lane group asks for 16 elements of four k rows, four a lane; they come turned: lane i has element i of the four rows
        const int part = set + 4 * Q * (i & 3);
        union { i16x4 half[2]; uint4 whole; } v;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = s * 32 + 8 * g + 4 * h + (i >> 2);
            const int c = (part >> 3) ^ chunk_twist<T, TILE, KC, Q>(k);
            v.half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)((const char*)(lds + k * kCpr + c) + (part & 4) * 2));
        }
        return v.whole;
    }
};

// ---- a tile of the result

template <typename T, typename O, int TA, int TB, int WA, int WB, bool A_KC, bool A_PICKED, bool B_KC, bool B_PICKED, bool ASYNC>
struct Tile {
    static constexpr int kNt = 64 * WA * WB;
    static constexpr int kFa = TA / WA / 16, kFb = TB / WB / 16;
    static constexpr int kQ = sizeof(O) == 2 && kFa % 2 == 0 ? 2 : 1, kN = 4 * kQ, kSets = kFa / kQ;   // columns a lane holds side by side, and how often
    static constexpr int kBk = kStepBytes / (int)sizeof(T);
    typedef Operand<T, TA, A_KC, A_PICKED, kQ, ASYNC, kNt> A;
    typedef Operand<T, TB, B_KC, B_PICKED, 1, ASYNC, kNt> B;
    f32x4 acc[kFa][kFb];

    static __device__ __forceinline__ int column(int set, int tid) { return ((tid >> 6) % WA) * (TA / WA) + 16 * kQ * set + kN * ((tid & 63) >> 4); }   // of the tile: the lane's first
    static __device__ __forceinline__ int row(int y, int tid) { return ((tid >> 6) / WA) * (TB / WB) + 16 * y + (tid & 15); }
    __device__ __forceinline__ auto& at(int set, int y, int j) { return ((float*)&acc[set * kQ + j / 4][y])[j % 4]; }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int x = 0; x < kFa; ++x)
#pragma unroll
            for (int y = 0; y < kFb; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // 16 rows of the widest result a wavefront, in the stages that the next tile's first loads do not use
    static constexpr int kPatch = 16 * 16 * kFa * 4, kInA = TA * kStepBytes / kPatch;
    static_assert(kInA + TB * kStepBytes / kPatch >= WA * WB, "every wavefront has a patch");
    static __device__ __forceinline__ char* patch(uint4* a1, uint4* b1, int tid) {
        const int wave = tid >> 6;
        return wave < kInA ? (char*)a1 + wave * kPatch : (char*)b1 + (wave - kInA) * kPatch;
    }
    // every wavefront's loads have landed, then all have arrived (a barrier alone does not wait for loads to LDS)
    static __device__ __forceinline__ void meet() {
        if (ASYNC) __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
        __syncthreads();
    }
    // acc += sum over k < limit, the first stage having been asked for.  Behind it all four stages are free.  SUMS: also the
    // sums of B alone over k; the wavefronts side by side along a share their columns, kSums fragments each.
    static constexpr int kSums = kFb < WA ? 1 : kFb / WA;
    static __device__ __forceinline__ bool sums_of(int y, int tid) { return y / kSums == (tid >> 6) % WA; }
    template <bool SUMS>
    __device__ __forceinline__ void run(A& a, B& b, uint4* a0, uint4* b0, uint4* a1, uint4* b1, int32_t limit, f32x4* sums, int tid) {
        const int lane = tid & 63, wave = tid >> 6, wa = (wave % WA) * (TA / WA), wb = (wave / WA) * (TB / WB);
        const int ws = wb + (wave % WA * kSums < kFb ? wave % WA * kSums * 16 : 0);   // (read once more: choosing among the fragments at hand would be a branch)
        const auto step = [&](const uint4* la, const uint4* lb) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                uint4 fa[kFa], fb[kFb];
#pragma unroll
                for (int x = 0; x < kFa; ++x) fa[x] = A::fragment(la, wa, x, s, lane);
#pragma unroll
                for (int y = 0; y < kFb; ++y) fb[y] = B::fragment(lb, wb, y, s, lane);
#pragma unroll
                for (int y = 0; y < kFb; ++y)
#pragma unroll
                    for (int x = 0; x < kFa; ++x) acc[x][y] = Elem<T>::mma(fa[x], fb[y], acc[x][y]);
                if (SUMS)
#pragma unroll
                    for (int q = 0; q < kSums; ++q) sums[q] = Elem<T>::mma(Elem<T>::ones(), B::fragment(lb, ws, q, s, lane), sums[q]);
            }
            if constexpr (!A_KC && B_KC && sizeof(T) == 2 && kFb > 1) {
                // the order of the stage's instructions: what the first products need, then reads between products, two of B's fragments
                // ahead (left to itself the compiler reads all of a step, waits for it, and multiplies: LDS and matrix cores take turns)
                constexpr int ra = kFa * (A_KC ? 1 : 2), rb = (B_KC ? 1 : 2), reads = 2 * (ra + kFb * rb), ahead = ra + 2 * rb, slots = kFb > 1 ? 2 * kFb - 2 : 1;
                __builtin_amdgcn_sched_group_barrier(0x100, ahead, 0);
#pragma unroll
                for (int i = 0; i < 2 * kFb; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, kFa, 0);
                    if (i < slots) __builtin_amdgcn_sched_group_barrier(0x100, (reads - ahead + slots - 1) / slots, 0);
                }
            }
        };
        if (limit <= 0) return;
        a.put(a0, tid);
        b.put(b0, tid);
        meet();
        // two stages a round, so that each has its own half of LDS by name: loads into one go on under the products of the other
        for (int32_t k = 0; k < limit; k += 2 * kBk) {
            const bool second = k + kBk < limit, third = k + 2 * kBk < limit;
            if (second) { a.ask(a1, k + kBk, tid); b.ask(b1, k + kBk, tid); }
            step(a0, b0);
            if (second) { a.put(a1, tid); b.put(b1, tid); }
            meet();
            if (third) { a.ask(a0, k + 2 * kBk, tid); b.ask(b0, k + 2 * kBk, tid); }
            if (second) step(a1, b1);
            if (third) { a.put(a0, tid); b.put(b0, tid); }
            meet();
        }
    }
};

// The items of a launch in eight runs, one an XCD (consecutive workgroups go to the eight XCDs in turn), whose workgroups take a run's
// items in turn: what an XCD works on at one time are neighbours, which share operands in its L2.
struct Deal { int64_t at, stop, step; };
__device__ __forceinline__ Deal my_items(int64_t total) {
    const int64_t blocks = (int64_t)gridDim.x * gridDim.y, b = block_number();
    if (blocks % 8) return Deal{b, total, blocks};
    const int64_t xcd = b & 7, from = total * xcd / 8, to = total * (xcd + 1) / 8;
    return Deal{from + (b >> 3), to, blocks >> 3};
}

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
};

// A wavefront's 16 rows of finished values to memory in whole rows: a matrix instruction leaves 16 consecutive lanes with 16
// rows, and stores go out 16 lanes at a time, so rows pass through LDS first and leave 128 bytes and more side by side (pieces of 16 bytes
// straight from the registers were written to memory 1.4 times, and a large product took 15 % longer).  They pass the caches by:
// a later kernel reads them.
template <typename W, typename X>
struct Rows16 {
    static constexpr int kCols = 16 * W::kFa, kChunks = kCols * (int)sizeof(X) / 16, kMask = (kChunks < 8 ? kChunks : 8) - 1;
    static __device__ __forceinline__ void put(char* patch, int set, const float* v, int lane) {   // the lane's piece of its row
        constexpr int n = W::kN * (int)sizeof(X) > 16 ? 16 / (int)sizeof(X) : W::kN;   // values at a time: 16 bytes or a part of them
        const int row = lane & 15;
#pragma unroll
        for (int j = 0; j < W::kN; j += n) {
            X part[n];
#pragma unroll
            for (int i = 0; i < n; ++i) part[i] = (X)v[j + i];
            const int byte = (16 * W::kQ * set + W::kN * (lane >> 4) + j) * (int)sizeof(X);
            __builtin_memcpy(__builtin_assume_aligned(patch + row * kCols * (int)sizeof(X) + (((byte >> 4) ^ (row & kMask)) << 4) + (byte & 15), sizeof(part)), part, sizeof(part));
        }
    }
    // rows 0 .. count - 1 of the 16, columns below `columns` from `to` on, 16 bytes at a time; not whole: wherever rows begin, and one by
    // one behind the last 16
    template <bool WHOLE>
    static __device__ __forceinline__ void send(const char* patch, X* to, int64_t stride, int count, int columns, int lane) {
        if (!WHOLE) {
            constexpr int n = 16 / (int)sizeof(X);
#pragma unroll
            for (int t = 0; t < 16 * kChunks; t += 64) {
                const int at = t + lane, row = at / kChunks, chunk = at % kChunks, left = columns - chunk * n;
                if ((16 * kChunks >= 64 || at < 16 * kChunks) && row < count && left > 0) {
                    X part[n];
                    __builtin_memcpy(part, __builtin_assume_aligned(patch + (row * kChunks + (chunk ^ (row & kMask))) * 16, 16), 16);
                    X* at_row = to + row * stride + chunk * n;
                    if (left >= n) __builtin_memcpy(at_row, part, 16);   // (aligned as an element is)
                    else
#pragma unroll
                        for (int j = 0; j < n - 1; ++j)
                            if (j < left) at_row[j] = part[j];
                }
            }
            return;
        }
        typedef uint32_t Word __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int t = 0; t < 16 * kChunks; t += 64) {
            const int at = t + lane, row = at / kChunks, chunk = at % kChunks;
            if ((16 * kChunks >= 64 || at < 16 * kChunks) && row < count && chunk * (16 / (int)sizeof(X)) < columns) {
                const Word w = *(const Word*)(patch + (row * kChunks + (chunk ^ (row & kMask))) * 16);
                __builtin_nontemporal_store(w, (Word*)(to + row * stride + chunk * (16 / (int)sizeof(X))));
            }
        }
    }
};

// y = act(x W^T + b), or (x W^T) act'(z).  Workgroups stay and take tiles in turn, the column tiles of a row tile next to each
// other: x comes from memory once, a group's weights stay in the XCD's L2.  The next tile's first stage is asked for before the results
// of this one are finished and stored.
//
// What bounds it: the matrix cores, and what does not go on under them, a tile's activation and stores.  524,288 rows of 768 -> 2,048 in
// bfloat16, gathered, with bias and SiLU: 2.0 ms, 830 TFLOP/s (a plain library product of that size 1.57 ms); without the SiLU 1.88;
// 48 rows through 64 experts of that size 30 us, 6.7 TB/s of weights.
// LOADS, STORES: rows are made of whole aligned 16-byte chunks where they are read (straight to LDS), where they are written; otherwise
// through registers, and wherever rows begin and end: 200,006 rows of 50 -> 129 in float32 113 us, of 52 -> 132 81.
template <typename T, typename O, int TA, int TB, int WA, int WB, bool W_KC, bool LOADS, bool STORES>
__global__ void __launch_bounds__(64 * WA * WB, 2) k_grouped_product(ProductArgs p) {
    typedef Tile<T, O, TA, TB, WA, WB, W_KC, false, true, true, LOADS> Work;
    constexpr int N = Work::kN;
    __shared__ uint4 a0[TA * kTileChunks], a1[TA * kTileChunks], b0[TB * kTileChunks], b1[TB * kTileChunks];
    const int lane = threadIdx.x & 63, tid = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * 64 + lane;   // (the wavefront's number in a scalar register)
    const int32_t across = (p.out + TA - 1) / TA;
    Deal deal = my_items((int64_t)count_items(p.offsets, p.n_groups, p.rows, TB, lane) * across);
    Work work;
    typename Work::A a;
    typename Work::B b;
    Item it{0, 0, 0, 0, 0};
    // what is in the works: a tile whose first stage has been asked for
    int32_t row_tile = -1, group = 0, column = 0, count = 0;
    int64_t first = 0;
    for (bool have = false;; have = true) {
        if (have) {
            // the sums begin with the bias
            float start[Work::kSets][N] = {};
            if (p.bias && group < p.n_groups) {
                const T* from = (const T*)p.bias + (int64_t)group * p.bias_stride + column;
#pragma unroll
                for (int set = 0; set < Work::kSets; ++set) {
                    const int32_t col = Work::column(set, tid), n = p.out - column - col;
                    T some[N] = {};
                    if (n >= N) __builtin_memcpy(some, from + col, sizeof(some));   // (aligned as an element is)
                    else if (n > 0)
                        for (int j = 0; j < N; ++j)
                            if (j < n) some[j] = from[col + j];
#pragma unroll
                    for (int j = 0; j < N; ++j) start[set][j] = (float)some[j];
                }
            }
#pragma unroll
            for (int set = 0; set < Work::kSets; ++set)
#pragma unroll
                for (int j = 0; j < N; ++j)
#pragma unroll
                    for (int y = 0; y < Work::kFb; ++y) work.at(set, y, j) = start[set][j];
            work.template run<false>(a, b, a0, b0, a1, b1, group < p.n_groups ? p.in : 0, nullptr, tid);
        }
        const int32_t done_group = group, done_column = column, done_count = count;
        const int64_t done_first = first;
        const bool more = deal.at < deal.stop;
        if (more) {
            const int32_t tile = (int32_t)(deal.at / across);
            column = (int32_t)(deal.at - (int64_t)tile * across) * TA;
            if (tile != row_tile) {
                row_tile = tile;
                if (tile >= it.first + it.items) find_item(it, p.offsets, p.n_groups, p.rows, TB, tile, lane);
                group = it.group;
                first = it.begin + (int64_t)(tile - it.first) * TB;
                count = (int32_t)(it.end - first < TB ? it.end - first : TB);
                b.open_rows(p.x, first, count, p.in, tid);
            }
            if (group < p.n_groups) {
                const Source w{(const T*)p.w + (int64_t)group * p.w_group, p.w_stride, nullptr, 0, 1};
                if (W_KC) a.open_rows(w, column, p.out - column, p.in, tid);
                else a.open_columns(w, 0, p.in, column, p.out, tid);
                a.ask(a0, 0, tid);
                b.ask(b0, 0, tid);
            }
            deal.at += deal.step;
        }
        if (have) {
            const bool inside = done_group < p.n_groups;
            char* patch = Work::patch(a1, b1, tid);
            const auto finish = [&](auto act, auto slope) {
                constexpr int ACT = decltype(act)::value, SLOPE = decltype(slope)::value;
                const int32_t wave_column = done_column + Work::column(0, tid & ~63);
#pragma unroll
                for (int y = 0; y < Work::kFb; ++y) {
                    const int r0 = Work::row(y, tid & ~63), r = Work::row(y, tid);
                    if (r0 >= done_count) continue;
                    float v[Work::kSets][N];
#pragma unroll
                    for (int set = 0; set < Work::kSets; ++set) {
                        const int32_t col = done_column + Work::column(set, tid);
                        const int n = r < done_count ? p.out - col : 0;
#pragma unroll
                        for (int j = 0; j < N; ++j) v[set][j] = work.at(set, y, j);
                        if (SLOPE) {
                            const T* from = (const T*)p.slope_at + (done_first + r) * p.slope_stride + col;
                            T z[N];
                            if (STORES && n > 0) __builtin_memcpy(z, from, sizeof(z));   // (aligned as an element is)
                            else
#pragma unroll
                                for (int j = 0; j < N; ++j) z[j] = j < n ? from[j] : (T)0.f;
#pragma unroll
                            for (int j = 0; j < N; ++j) v[set][j] *= activation_slope<ACT, sizeof(O) == 4>((float)z[j]);
                        } else if (p.z_out) {
                            Rows16<Work, T>::put(patch, set, v[set], lane);
                        }
                    }
                    if (!SLOPE && p.z_out)
                        Rows16<Work, T>::template send<STORES>(patch, (T*)p.z_out + (done_first + r0) * p.z_stride + wave_column, p.z_stride, done_count - r0, p.out - wave_column, lane);
#pragma unroll
                    for (int set = 0; set < Work::kSets; ++set) {
                        if (!SLOPE && inside)
#pragma unroll
                            for (int j = 0; j < N; ++j) v[set][j] = activate<ACT, sizeof(O) == 4>(v[set][j]);
                        Rows16<Work, O>::put(patch, set, v[set], lane);
                    }
                    Rows16<Work, O>::template send<STORES>(patch, (O*)p.y + (done_first + r0) * p.y_stride + wave_column, p.y_stride, done_count - r0, p.out - wave_column, lane);
                }
            };
            const int act = inside ? p.activation : (int)kNone;   // (one copy of the code for each, outside the loops over rows)
            if (p.slope_at && act == kRelu) finish(Constant<kRelu>{}, Constant<1>{});
            else if (p.slope_at && act == kSilu) finish(Constant<kSilu>{}, Constant<1>{});
            else if (p.slope_at && act == kGelu) finish(Constant<kGelu>{}, Constant<1>{});
            else if (act == kRelu) finish(Constant<kRelu>{}, Constant<0>{});
            else if (act == kSilu) finish(Constant<kSilu>{}, Constant<0>{});
            else if (act == kGelu) finish(Constant<kGelu>{}, Constant<0>{});
            else finish(Constant<kNone>{}, Constant<0>{});
        }
        if (!more) break;
    }
}

// The same for few rows, where the groups' weights are read once and there are too few tiles for all compute units: a workgroup takes 16
// rows and 16 columns, its wavefronts share k, two steps (128 bytes of every row) at a time, straight from memory to
// registers, and add up in LDS.  Latency is all it costs: one row of bfloat16 through two experts of 768 x 2,048 takes 5.6 us (6.3 MB of
// weights, 1.2 us at the rate of a large copy), 15.4 in tiles of 128.
constexpr int kFewWaves = 8;
template <typename T, typename O>
__global__ void __launch_bounds__(64 * kFewWaves) k_grouped_few(ProductArgs p) {
    constexpr int epc = 16 / (int)sizeof(T), step = 4 * epc;   // k a step: a chunk for every lane group
    constexpr bool full = sizeof(O) == 4;
    __shared__ f32x4 part[kFewWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), g = lane >> 4, i = lane & 15;
    const int32_t across = (p.out + 15) / 16;
    const int64_t block = block_number();
    const int32_t tile = (int32_t)(block / across), column = (int32_t)(block - (int64_t)tile * across) * 16;
    Item it{0, 0, 0, 0, 0};
    find_item(it, p.offsets, p.n_groups, p.rows, 16, tile, lane);
    if (it.group < 0) return;
    const int64_t first = it.begin + (int64_t)(tile - it.first) * 16;
    const int32_t count = (int32_t)(it.end - first < 16 ? it.end - first : 16);
    const bool inside = it.group < p.n_groups;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (inside) {
        const int64_t at = i < count ? p.x.row_of(first + i) : -1;
        const T* x = at >= 0 ? (const T*)p.x.base + at * p.x.stride : nullptr;
        const T* w = column + i < p.out ? (const T*)p.w + (int64_t)it.group * p.w_group + (int64_t)(column + i) * p.w_stride : nullptr;
        const auto chunk = [&](const T* row, int32_t k) {
            uint4 v = make_uint4(0, 0, 0, 0);
            const int n = row ? p.in - k : 0;
            if (n >= epc) {
                __builtin_memcpy(&v, row + k, 16);   // (aligned as an element is)
            } else if (n > 0) {
                T some[epc] = {};
#pragma unroll
                for (int j = 0; j < epc; ++j)
                    if (j < n) some[j] = row[k + j];
                __builtin_memcpy(&v, some, 16);
            }
            return v;
        };
        for (int32_t k0 = wave * 2 * step; k0 < p.in; k0 += kFewWaves * 2 * step * 2) {   // four steps on their way at once
            uint4 a[4], b[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int32_t k = k0 + (s & 1) * step + (s >> 1) * kFewWaves * 2 * step + g * epc;
                a[s] = chunk(w, k);
                b[s] = chunk(x, k);
            }
#pragma unroll
            for (int s = 0; s < 4; ++s) acc = Elem<T>::mma(a[s], b[s], acc);
        }
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave > 0 || i >= count) return;
#pragma unroll
    for (int j = 1; j < kFewWaves; ++j) acc += part[j][lane];
    const int64_t row = first + i;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int32_t col = column + 4 * g + j;
        if (col >= p.out) break;
        float v = acc[j];
        if (inside && p.slope_at) {
            const float z = (float)((const T*)p.slope_at)[row * p.slope_stride + col];
            v *= p.activation == kRelu ? activation_slope<kRelu, full>(z) : p.activation == kSilu ? activation_slope<kSilu, full>(z) : p.activation == kGelu ? activation_slope<kGelu, full>(z) : 1.f;
        } else {
            if (inside && p.bias) v += (float)((const T*)p.bias)[(int64_t)it.group * p.bias_stride + col];
            if (p.z_out) ((T*)p.z_out)[row * p.z_stride + col] = (T)v;
            if (inside) v = p.activation == kRelu ? activate<kRelu, full>(v) : p.activation == kSilu ? activate<kSilu, full>(v) : p.activation == kGelu ? activate<kGelu, full>(v) : v;
        }
        ((O*)p.y)[row * p.y_stride + col] = (O)v;
    }
}

struct GradientArgs {
    const int32_t* offsets;
    Source x, dy;            // x: [.., in], gathered; dy: [rows, out]
    void* dw;                // [n_groups, out, in]
    float* db;               // NULL or [n_groups, out]
    float* part;             // [slots][out, in] sums of parts of long groups, behind them [slots][out] of db
    int64_t slots;
    int64_t rows;
    int32_t n_groups, in, out;
    int32_t most;            // rows a part has at most
    int32_t slot_bits;
};

// A group of more than `most` rows is taken in parts of equal length (at least most / 2 rows), so that no workgroup has much more to do than the
// others; their sums meet in k_grouped_parts, always in the same order.
__device__ __forceinline__ int32_t parts_of(int32_t count, int32_t most) { return count <= most ? 1 : (int32_t)(((uint32_t)count + (uint32_t)most - 1) / (uint32_t)most); }
__device__ __forceinline__ int64_t part_begin(int64_t begin, int32_t count, int32_t part, int32_t parts) {
    const uint32_t each = (uint32_t)count / (uint32_t)parts, left = (uint32_t)count - each * (uint32_t)parts;
    return begin + (int64_t)part * each + ((uint32_t)part < left ? (uint32_t)part : left);
}
// Parts of long groups begin at least most / 2 rows apart, and 2^slot_bits is no more: the place for their sums
__device__ __forceinline__ int64_t slot_of(int64_t part_begin, int32_t slot_bits) { return part_begin >> slot_bits; }

struct Unit {
    int64_t begin;
    int32_t group, count, parts;
    int32_t length, from, before;   // where the search for the next one begins: class of lengths, group, parts before it
};
// Parts in the order in which they are taken: long ones first (four classes by length), so that what is left at the end is short.
__device__ __forceinline__ int32_t length_class(int32_t parts, int32_t count, int32_t most) {   // (a part of a long group has more than half of `most` rows)
    return parts > 1 || count > most / 2 ? 0 : count > most / 4 ? 1 : count > most / 8 ? 2 : 3;
}
__device__ __forceinline__ int32_t rows_of_group(const GradientArgs& p, int32_t e, int64_t& begin) {
    begin = group_end(p.offsets, e, p.n_groups, p.rows);
    const int64_t rows = group_end(p.offsets, e + 1, p.n_groups, p.rows) - begin;
    return rows < 0 ? 0 : (int32_t)rows;
}
__device__ __forceinline__ int32_t count_units(const GradientArgs& p, int lane) {
    int32_t mine = 0;
#pragma unroll 4
    for (int32_t e = lane; e < p.n_groups; e += 64) {
        int64_t begin;
        mine += parts_of(rows_of_group(p, e, begin), p.most);
    }
    return of_lane(wave_inclusive(mine, lane), 63);
}
// Part number `at` of that order, which there is, and which is no earlier than the one in `u`
__device__ __forceinline__ void find_unit(const GradientArgs& p, Unit& u, int32_t at, int lane) {
    int32_t before = u.before, g0 = u.from;
    for (int32_t length = u.length; length < 4; ++length, g0 = 0)
        for (; g0 < p.n_groups; g0 += 64) {
            const int32_t e = g0 + lane;
            int64_t begin = 0;
            int32_t count = 0, parts = 0, mine = 0;
            if (e < p.n_groups) {
                count = rows_of_group(p, e, begin);
                parts = parts_of(count, p.most);
                if (length_class(parts, count, p.most) == length) mine = parts;
            }
            const int32_t upto = before + wave_inclusive(mine, lane);
            const uint64_t mask = __ballot(upto > at);
            if (mask) {
                const int who = __builtin_ctzll(mask);
                const int64_t b = of_lane(begin, who);
                const int32_t c = of_lane(count, who);
                u.parts = of_lane(parts, who);
                const int32_t part = at - of_lane(upto - mine, who);
                u.group = g0 + who;
                u.begin = part_begin(b, c, part, u.parts);
                u.count = (int32_t)(part_begin(b, c, part + 1, u.parts) - u.begin);
                u.length = length;
                u.from = g0;
                u.before = before;
                return;
            }
            before = of_lane(upto, 63);
        }
}

// dW = sum over the group's rows of dy^T x: tiles of TA columns of x and TB of dy.  The tiles of a part go to one XCD, side by side: they read
// the same rows.  Workgroups stay and take every so many-th tile of their XCD, in turn from either end, as the parts get shorter.
// Both operands are turned on their way out of LDS.  524,288 rows, 2,048 x 768 in bfloat16: 2.0 ms, 810 TFLOP/s; 200,006 rows in 256 groups,
// 512 x 768: 0.31 ms, where rows and results alone are 0.15 at the rate of a large copy.
template <typename T, typename O, int TA, int TB, int WA, int WB, bool LOADS, bool STORES>
__global__ void __launch_bounds__(64 * WA * WB, 2) k_grouped_gradient(GradientArgs p) {
    typedef Tile<T, O, TA, TB, WA, WB, false, true, false, false, LOADS> Work;
    constexpr int N = Work::kN;
    __shared__ uint4 a0[TA * kTileChunks], a1[TA * kTileChunks], b0[TB * kTileChunks], b1[TB * kTileChunks];
    const int lane = threadIdx.x & 63, tid = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * 64 + lane;   // (the wavefront's number in a scalar register)
    const int32_t across = (p.in + TA - 1) / TA, tiles = across * ((p.out + TB - 1) / TB);
    const int32_t units = count_units(p, lane);
    const int32_t xcds = gridDim.x % 8 == 0 ? 8 : 1, xcd = (int32_t)blockIdx.x % xcds, local = (int32_t)blockIdx.x / xcds, locals = (int32_t)gridDim.x / xcds;
    Work work;
    typename Work::A a;
    typename Work::B b;
    Unit unit{0, -1, 0, 0, 0, 0, 0};
    int32_t unit_at = -1, a_first = 0, b_first = 0;
    int32_t turn = 0;
    for (bool have = false;; have = true) {
        f32x4 sums[Work::kSums];
        const bool bias = have && p.db && a_first == 0;
        if (have) {
            work.clear();
#pragma unroll
            for (int y = 0; y < Work::kSums; ++y) sums[y] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (bias) work.template run<true>(a, b, a0, b0, a1, b1, unit.count, sums, tid);
            else work.template run<false>(a, b, a0, b0, a1, b1, unit.count, sums, tid);
        }
        const Unit done = unit;
        const int32_t done_a = a_first, done_b = b_first;
        // the next tile: number t of this XCD's
        const int64_t t = (int64_t)turn * locals + (turn & 1 ? locals - 1 - local : local), band = t / tiles;
        const int64_t next = band * xcds + (band & 1 ? xcds - 1 - xcd : xcd);
        ++turn;
        const bool more = next < units;
        if (more) {
            const int32_t tile = (int32_t)(t - band * tiles);
            if (next != unit_at) find_unit(p, unit, (int32_t)next, lane);
            unit_at = (int32_t)next;
            a_first = tile % across * TA;
            b_first = tile / across * TB;
            a.open_columns(p.x, unit.begin, unit.count, a_first, p.in, tid);
            b.open_columns(p.dy, unit.begin, unit.count, b_first, p.out, tid);
            if (unit.count > 0) {
                a.ask(a0, 0, tid);
                b.ask(b0, 0, tid);
            }
        }
        if (have) {
            const int64_t slot = slot_of(done.begin, p.slot_bits);
            if (bias && lane < 16) {
                float* to = done.parts == 1 ? p.db + (int64_t)done.group * p.out : p.part + p.slots * p.out * p.in + slot * p.out;
#pragma unroll
                for (int y = 0; y < Work::kFb; ++y) {
                    const int32_t r = done_b + Work::row(y, tid);
                    if (Work::sums_of(y, tid) && r < p.out) to[r] = sums[y % Work::kSums][0];
                }
            }
            char* patch = Work::patch(a1, b1, tid);
            const int32_t wave_column = done_a + Work::column(0, tid & ~63);
            const auto out = [&](auto* to) {
                typedef typename std::remove_pointer<decltype(to)>::type X;
#pragma unroll
                for (int y = 0; y < Work::kFb; ++y) {
                    const int32_t r0 = done_b + Work::row(y, tid & ~63);
                    if (r0 >= p.out) continue;
#pragma unroll
                    for (int set = 0; set < Work::kSets; ++set) {
                        float v[N];
#pragma unroll
                        for (int j = 0; j < N; ++j) v[j] = work.at(set, y, j);
                        Rows16<Work, X>::put(patch, set, v, lane);
                    }
                    Rows16<Work, X>::template send<STORES>(patch, to + (int64_t)r0 * p.in + wave_column, p.in, p.out - r0, p.in - wave_column, lane);
                }
            };
            if (done.parts == 1) out((O*)p.dw + (int64_t)done.group * p.out * p.in);
            else out(p.part + slot * p.out * p.in);
        }
        if (!more) break;
    }
}

// The sums of the parts of long groups, in the order of the parts, sixteen loads on their way at once: a workgroup takes 256 PER elements
// of one group
template <typename O, int PER>
__global__ void __launch_bounds__(256) k_grouped_parts(GradientArgs p) {
    const int64_t size = (int64_t)p.out * p.in, pieces = (size + 256 * PER - 1) / (256 * PER), block = block_number();
    const int64_t number = block / pieces, piece = block - number * pieces;
    const int lane = threadIdx.x & 63;
    // long group `number`
    int32_t group = -1, before = 0, count = 0;
    int64_t begin = 0;
    for (int32_t g0 = 0; g0 < p.n_groups; g0 += 64) {
        const int32_t e = g0 + lane;
        int64_t rows = 0;
        if (e < p.n_groups) {
            begin = group_end(p.offsets, e, p.n_groups, p.rows);
            rows = group_end(p.offsets, e + 1, p.n_groups, p.rows) - begin;
        }
        const uint64_t mask = __ballot(rows > p.most);
        const int found = __popcll(mask);
        if (number < before + found) {
            uint64_t left = mask;
            for (int64_t j = before; j < number; ++j) left &= left - 1;
            const int who = __builtin_ctzll(left);
            group = g0 + who;
            begin = of_lane(begin, who);
            count = of_lane((int32_t)rows, who);
            break;
        }
        before += found;
    }
    if (group < 0) return;
    const int32_t parts = parts_of(count, p.most);
    // sums over the parts of the elements i, i + 256, ... of an array of `apart` a slot
    const auto add = [&](const float* from, int64_t apart, int64_t i, float (&sum)[PER]) {
        constexpr int batch = 16 / PER;
#pragma unroll
        for (int q = 0; q < PER; ++q) sum[q] = 0.f;
        for (int32_t j0 = 0; j0 < parts; j0 += batch) {
            float v[batch][PER];
#pragma unroll
            for (int j = 0; j < batch; ++j) {
                const float* slot = from + slot_of(part_begin(begin, count, j0 + j < parts ? j0 + j : 0, parts), p.slot_bits) * apart;
#pragma unroll
                for (int q = 0; q < PER; ++q) v[j][q] = j0 + j < parts && i + q * 256 < apart ? slot[i + q * 256] : 0.f;
            }
#pragma unroll
            for (int j = 0; j < batch; ++j)
#pragma unroll
                for (int q = 0; q < PER; ++q) sum[q] += v[j][q];
        }
    };
    float sum[PER];
    if (p.db && piece == 0)
        for (int64_t r = threadIdx.x; r < p.out; r += 256 * PER) {
            add(p.part + p.slots * size, p.out, r, sum);
#pragma unroll
            for (int q = 0; q < PER; ++q)
                if (r + q * 256 < p.out) p.db[(int64_t)group * p.out + r + q * 256] = sum[q];
        }
    const int64_t i = piece * (256 * PER) + threadIdx.x;
    add(p.part, size, i, sum);
#pragma unroll
    for (int q = 0; q < PER; ++q)
        if (i + q * 256 < size) ((O*)p.dw)[(int64_t)group * size + i + q * 256] = (O)sum[q];
}

}  // namespace nomad_grouped
