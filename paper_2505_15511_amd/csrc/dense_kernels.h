// Dense matrix products for gfx950, with what follows them in the same pass.
//
//   forward            y = act(x W^T + b) + r
//   rows' gradient     dx = dz W (times the slope of the activation before)
//   weights' gradient  dW = dz^T x,  db = sum of dz
//
// All are tiles of C[b][a] = sum_k A[a][k] B[b][k] as in grouped_kernels.h, of which operands, tiles and their ways through LDS are taken.
// A sum over k may be cut into parts, for products with few tiles: their float32 sums go to work space and meet in k_dense_parts, always
// in the same order.
//
// What bounds them: the matrix cores, and of a large product what stands beside them: a tile's activation, residual and stores, since a unit
// holds one workgroup of 256 x 256 and all units finish a tile at about the same time.  65,536 rows of 4,096 -> 4,096 in bfloat16: 1.87 ms by
// themselves (1,175 TFLOP/s; a plain library product 1.44), 1.97 with bias and GELU, 2.1 with a residual too; dx 1.81, dW 1.78 ms (library 1.65 and
// 1.82).  Taken back: a wavefront a SIMD with a quarter of a tile and its next operands read ahead (256 sums and 128 operands a lane did not fit
// the registers), the residual read in the order of the stores, its lines into L2 under the products (both slower).
#pragma once
#include "grouped_kernels.h"

namespace nomad_dense {

using namespace nomad_grouped;

struct Finish {                  // what follows the sum
    const void* bias;            // NULL: none
    const void* residual;        // NULL: none
    int64_t residual_stride;
    const void* slope_at;        // z of the activation whose slope multiplies the result; NULL: activation itself
    int64_t slope_stride;
    void* z_out;
    int64_t z_stride;
    void* y;
    int64_t y_stride;
    int32_t activation;
    float factor;                // of the sum, without a bias (1: what an operand was kept smaller by)
};
struct DenseArgs {
    const void* a;               // A_KC: rows a, k contiguous; otherwise rows k, a contiguous
    int64_t a_stride;
    const void* b;
    int64_t b_stride;
    int64_t rows;                // of C
    int32_t columns;
    int64_t k, length;           // of the sum, of a part of it
    int32_t parts;
    float* part;                 // NULL: finish here; otherwise [parts][rows][columns] sums, rows part_stride apart
    int64_t part_stride;
    float* sums;                 // NULL, or [parts][rows] sums of B over k
    Finish f;
};

// The residual's sum is rounded by itself, never as one with a product that an activation ends in: results do not depend on the way a tile is finished
__device__ __forceinline__ float plus(float v, float residual) {
#pragma clang fp contract(off)
    return v + residual;
}

// Tiles in the order in which they are taken: runs of eight rows of them, down each column of a run first, so that neighbours in
// time share both operands
__device__ __forceinline__ void tile_at(int64_t at, int64_t down, int64_t across, int64_t& row, int32_t& column) {
    constexpr int64_t run = 8;
    const int64_t first = at / (run * across) * run, here = down - first < run ? down - first : run, in = at - first * across;
    row = first + in % here;
    column = (int32_t)(in / here);
}

template <typename T, int TA, int TB, int WA, int WB, bool A_KC, bool B_KC, bool LOADS, bool STORES>
__global__ void __launch_bounds__(64 * WA * WB, 2) k_dense(DenseArgs p) {
    typedef Tile<T, T, TA, TB, WA, WB, A_KC, false, B_KC, false, LOADS> Work;
    constexpr int N = Work::kN;
    constexpr bool SUMS = !A_KC && !B_KC, FULL = sizeof(T) == 4;
    __shared__ uint4 a0[TA * kTileChunks], a1[TA * kTileChunks], b0[TB * kTileChunks], b1[TB * kTileChunks];
    const int lane = threadIdx.x & 63, tid = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * 64 + lane;   // (the wavefront's number in a scalar register)
    const int64_t across = (p.columns + TA - 1) / TA, down = (p.rows + TB - 1) / TB, tiles = across * down;
    Deal deal = my_items(tiles * p.parts);
    Work work;
    typename Work::A a;
    typename Work::B b;
    int64_t first = 0;
    int32_t column = 0, part = 0, count = 0, limit = 0;
    for (bool have = false;; have = true) {
        f32x4 sums[Work::kSums];
        const bool summed = SUMS && have && p.sums && column == 0;
        if (have) {
            if (p.f.bias && !p.part) {   // the sums begin with the bias
                const T* from = (const T*)p.f.bias + column;
#pragma unroll
                for (int set = 0; set < Work::kSets; ++set) {
                    const int32_t col = Work::column(set, tid), n = p.columns - column - col;
                    T some[N] = {};
                    if (n >= N) __builtin_memcpy(some, from + col, sizeof(some));   // (aligned as an element is)
                    else if (n > 0)
                        for (int j = 0; j < N; ++j)
                            if (j < n) some[j] = from[col + j];
#pragma unroll
                    for (int j = 0; j < N; ++j)
#pragma unroll
                        for (int y = 0; y < Work::kFb; ++y) work.at(set, y, j) = (float)some[j];
                }
            } else {
                work.clear();
            }
            if (SUMS) {
#pragma unroll
                for (int y = 0; y < Work::kSums; ++y) sums[y] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            if (summed) work.template run<SUMS>(a, b, a0, b0, a1, b1, limit, sums, tid);
            else work.template run<false>(a, b, a0, b0, a1, b1, limit, nullptr, tid);
        }
        const int32_t done_column = column, done_count = count, done_part = part;
        const int64_t done_first = first;
        const bool more = deal.at < deal.stop;
        if (more) {
            part = (int32_t)(deal.at / tiles);
            int64_t row;
            tile_at(deal.at - part * tiles, down, across, row, column);
            first = row * TB;
            column *= TA;
            count = (int32_t)(p.rows - first < TB ? p.rows - first : TB);
            const int64_t k0 = part * p.length;
            limit = (int32_t)(p.k - k0 < p.length ? p.k - k0 : p.length);
            const Source sa{(const T*)p.a + (A_KC ? k0 : 0), p.a_stride, nullptr, 0, 1}, sb{(const T*)p.b + (B_KC ? k0 : 0), p.b_stride, nullptr, 0, 1};
            if (A_KC) a.open_rows(sa, column, p.columns - column, limit, tid);
            else a.open_columns(sa, k0, limit, column, p.columns, tid);
            if (B_KC) b.open_rows(sb, first, count, limit, tid);
            else b.open_columns(sb, k0, limit, (int32_t)first, (int32_t)p.rows, tid);
            if (limit > 0) {
                a.ask(a0, 0, tid);
                b.ask(b0, 0, tid);
            }
            deal.at += deal.step;
        }
        if (have) {
            if (SUMS && summed && lane < 16)
#pragma unroll
                for (int y = 0; y < Work::kFb; ++y) {
                    const int r = Work::row(y, tid);
                    if (Work::sums_of(y, tid) && r < done_count) p.sums[(int64_t)done_part * p.rows + done_first + r] = sums[y % Work::kSums][0];
                }
            char* patch = Work::patch(a1, b1, tid);
            const int32_t wave_column = done_column + Work::column(0, tid & ~63);
            if (p.part) {
                float* to = p.part + ((int64_t)done_part * p.rows + done_first) * p.part_stride + wave_column;
#pragma unroll
                for (int y = 0; y < Work::kFb; ++y) {
                    const int r0 = Work::row(y, tid & ~63);
                    if (r0 >= done_count) continue;
#pragma unroll
                    for (int set = 0; set < Work::kSets; ++set) {
                        float v[N];
#pragma unroll
                        for (int j = 0; j < N; ++j) v[j] = work.at(set, y, j);
                        Rows16<Work, float>::put(patch, set, v, lane);
                    }
                    Rows16<Work, float>::template send<STORES>(patch, to + (int64_t)r0 * p.part_stride, p.part_stride, done_count - r0, p.columns - wave_column, lane);
                }
            } else {
                const auto finish = [&](auto act, auto slope) {
                    constexpr int ACT = decltype(act)::value, SLOPE = decltype(slope)::value;
                    const auto piece = [&](const void* base, int64_t stride, int r, int32_t col, int n, float (&v)[N]) {   // the lane's columns of a row
                        const T* from = (const T*)base + (done_first + r) * stride + col;
                        T some[N];
                        if (STORES && n > 0) __builtin_memcpy(some, from, sizeof(some));   // (aligned as an element is)
                        else
#pragma unroll
                            for (int j = 0; j < N; ++j) some[j] = j < n ? from[j] : (T)0.f;
#pragma unroll
                        for (int j = 0; j < N; ++j) v[j] = (float)some[j];
                    };
#pragma unroll
                    for (int y = 0; y < Work::kFb; ++y) {
                        const int r0 = Work::row(y, tid & ~63), r = Work::row(y, tid);
                        if (r0 >= done_count) continue;
                        float v[Work::kSets][N];
#pragma unroll
                        for (int set = 0; set < Work::kSets; ++set) {
                            const int32_t col = done_column + Work::column(set, tid);
                            const int n = r < done_count ? p.columns - col : 0;
#pragma unroll
                            for (int j = 0; j < N; ++j) v[set][j] = work.at(set, y, j);
                            if (ACT == kNone && !SLOPE)
#pragma unroll
                                for (int j = 0; j < N; ++j) v[set][j] *= p.f.factor;
                            if (SLOPE) {
                                float z[N];
                                piece(p.f.slope_at, p.f.slope_stride, r, col, n, z);
#pragma unroll
                                for (int j = 0; j < N; ++j) v[set][j] *= activation_slope<ACT, FULL>(z[j]);
                            } else if (p.f.z_out) {
                                Rows16<Work, T>::put(patch, set, v[set], lane);
                            }
                        }
                        if (!SLOPE && p.f.z_out)
                            Rows16<Work, T>::template send<STORES>(patch, (T*)p.f.z_out + (done_first + r0) * p.f.z_stride + wave_column, p.f.z_stride, done_count - r0,
                                                                   p.columns - wave_column, lane);
#pragma unroll
                        for (int set = 0; set < Work::kSets; ++set) {
                            if (!SLOPE)
#pragma unroll
                                for (int j = 0; j < N; ++j) v[set][j] = activate<ACT, FULL>(v[set][j]);
                            if (p.f.residual) {
                                const int32_t col = done_column + Work::column(set, tid);
                                float more_v[N];
                                piece(p.f.residual, p.f.residual_stride, r, col, r < done_count ? p.columns - col : 0, more_v);
#pragma unroll
                                for (int j = 0; j < N; ++j) v[set][j] = plus(v[set][j], more_v[j]);
                            }
                            Rows16<Work, T>::put(patch, set, v[set], lane);
                        }
                        Rows16<Work, T>::template send<STORES>(patch, (T*)p.f.y + (done_first + r0) * p.f.y_stride + wave_column, p.f.y_stride, done_count - r0,
                                                               p.columns - wave_column, lane);
                    }
                };
                // A whole tile with a residual, without z_out: no branches, so that the compiler knows how many loads and stores are on their way, and waits for a piece of
                // the residual without waiting for the stores behind it (memory operations come back in order). Two rows of pieces are asked for ahead:
                // 65,536 rows of 768 -> 2,048 in bfloat16 with GELU and a residual 325 us, 359 with one, 328 with three, 364 in the general form.
                const auto finish_whole = [&](auto act) {
                    constexpr int ACT = decltype(act)::value, ahead = 2;
                    struct alignas(sizeof(T)) Piece { T v[N]; } held[ahead][Work::kSets];
                    const T* residual = (const T*)p.f.residual + (done_first + Work::row(0, tid)) * p.f.residual_stride + done_column + Work::column(0, tid);
                    const auto ask = [&](int y) {
#pragma unroll
                        for (int set = 0; set < Work::kSets; ++set) held[y % ahead][set] = *(const Piece*)(residual + 16 * y * p.f.residual_stride + 16 * Work::kQ * set);
                    };
                    T* to = (T*)p.f.y + (done_first + Work::row(0, tid & ~63)) * p.f.y_stride + wave_column;
#pragma unroll
                    for (int y = 0; y < ahead && y < Work::kFb; ++y) ask(y);
#pragma unroll
                    for (int y = 0; y < Work::kFb; ++y) {
#pragma unroll
                        for (int set = 0; set < Work::kSets; ++set) {
                            float v[N];
#pragma unroll
                            for (int j = 0; j < N; ++j) v[j] = plus(activate<ACT, FULL>(work.at(set, y, j)), (float)held[y % ahead][set].v[j]);
                            Rows16<Work, T>::put(patch, set, v, lane);
                        }
                        if (y + ahead < Work::kFb) ask(y + ahead);
                        typedef uint32_t Word __attribute__((ext_vector_type(4)));
                        typedef Rows16<Work, T> Rows;
#pragma unroll
                        for (int t = 0; t < 16 * Rows::kChunks; t += 64) {
                            const int at = t + lane, row = at / Rows::kChunks, chunk = at % Rows::kChunks;
                            const Word w = *(const Word*)(patch + (row * Rows::kChunks + (chunk ^ (row & Rows::kMask))) * 16);
                            __builtin_nontemporal_store(w, (Word*)(to + (16 * y + row) * p.f.y_stride + chunk * (16 / (int)sizeof(T))));
                        }
                    }
                };
                const int act = p.f.activation;   // (one copy of the code for each, outside the loops over rows)
                if constexpr (LOADS && STORES && A_KC && TA >= 128) {
                    if (p.f.residual && !p.f.z_out && done_count == TB && done_column + TA <= p.columns) {
                        if (act == kRelu) finish_whole(Constant<kRelu>{});
                        else if (act == kSilu) finish_whole(Constant<kSilu>{});
                        else if (act == kGelu) finish_whole(Constant<kGelu>{});
                        else finish_whole(Constant<kNone>{});
                        if (!more) break;
                        continue;
                    }
                }
                if (p.f.slope_at && act == kRelu) finish(Constant<kRelu>{}, Constant<1>{});
                else if (p.f.slope_at && act == kSilu) finish(Constant<kSilu>{}, Constant<1>{});
                else if (p.f.slope_at && act == kGelu) finish(Constant<kGelu>{}, Constant<1>{});
                else if (act == kRelu) finish(Constant<kRelu>{}, Constant<0>{});
                else if (act == kSilu) finish(Constant<kSilu>{}, Constant<0>{});
                else if (act == kGelu) finish(Constant<kGelu>{}, Constant<0>{});
                else finish(Constant<kNone>{}, Constant<0>{});
            }
        }
        if (!more) break;
    }
}

template <bool FULL>
__device__ __forceinline__ float activate_by(int activation, float z) {
    return activation == kRelu ? activate<kRelu, FULL>(z) : activation == kSilu ? activate<kSilu, FULL>(z) : activation == kGelu ? activate<kGelu, FULL>(z) : z;
}
template <bool FULL>
__device__ __forceinline__ float slope_by(int activation, float z) {
    return activation == kRelu ? activation_slope<kRelu, FULL>(z) : activation == kSilu ? activation_slope<kSilu, FULL>(z) : activation == kGelu ? activation_slope<kGelu, FULL>(z) : 1.f;
}
// one result from its sum (with the bias where there is one)
template <typename T, typename O>
__device__ __forceinline__ void finish_one(const Finish& f, int64_t row, int32_t col, float v) {
    constexpr bool full = sizeof(O) == 4;
    v *= f.factor;
    if (f.slope_at) v *= slope_by<full>(f.activation, (float)((const T*)f.slope_at)[row * f.slope_stride + col]);
    else {
        if (f.z_out) ((T*)f.z_out)[row * f.z_stride + col] = (T)v;
        v = activate_by<full>(f.activation, v);
    }
    if (f.residual) v = plus(v, (float)((const T*)f.residual)[row * f.residual_stride + col]);
    ((O*)f.y)[row * f.y_stride + col] = (O)v;
}

// Up to 64 rows, k contiguous on either side: the weights are read once and there are too few tiles for all compute units. A workgroup takes
// 16 columns and all rows (ROWS sixteens of them), its wavefronts share k, straight from memory to registers, and add up in LDS.  24 rows of
// 8,192 -> 4,096 in float16: 24.4 us, 67 MB of weights at 2.7 TB/s; rows of x come from L2, twice the weights' bytes.
template <typename T, typename O, int ROWS>
__global__ void __launch_bounds__(64 * kFewWaves) k_dense_few(DenseArgs p) {
    constexpr int epc = 16 / (int)sizeof(T), step = 4 * epc;   // k a step: a chunk for every lane group
    constexpr int kAhead = ROWS > 2 ? 2 : 4;                   // steps on their way at once, neighbours in twos
    __shared__ f32x4 held[kFewWaves][ROWS][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), g = lane >> 4, i = lane & 15;
    const int32_t across = (p.columns + 15) / 16, part = (int32_t)(blockIdx.x / (uint32_t)across), column = (int32_t)(blockIdx.x - (uint32_t)(part * across)) * 16;
    const int64_t k0 = part * p.length, stop = p.k - k0 < p.length ? p.k : k0 + p.length;
    f32x4 acc[ROWS];
#pragma unroll
    for (int y = 0; y < ROWS; ++y) acc[y] = f32x4{0.f, 0.f, 0.f, 0.f};
    const T* w = column + i < p.columns ? (const T*)p.a + (int64_t)(column + i) * p.a_stride : nullptr;
    const T* x[ROWS];
#pragma unroll
    for (int y = 0; y < ROWS; ++y) x[y] = 16 * y + i < p.rows ? (const T*)p.b + (16 * y + i) * p.b_stride : nullptr;
    const auto chunk = [&](const T* row, int64_t k) {
        uint4 v = make_uint4(0, 0, 0, 0);
        const int64_t n = row ? stop - k : 0;
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
    for (int64_t k = k0 + wave * 2 * step; k < stop; k += kFewWaves * kAhead * step) {
        uint4 a[kAhead], b[kAhead][ROWS];
#pragma unroll
        for (int s = 0; s < kAhead; ++s) {
            const int64_t at = k + (s & 1) * step + (s >> 1) * kFewWaves * 2 * step + g * epc;
            a[s] = chunk(w, at);
#pragma unroll
            for (int y = 0; y < ROWS; ++y) b[s][y] = chunk(x[y], at);
        }
#pragma unroll
        for (int s = 0; s < kAhead; ++s)
#pragma unroll
            for (int y = 0; y < ROWS; ++y) acc[y] = Elem<T>::mma(a[s], b[s][y], acc[y]);
    }
#pragma unroll
    for (int y = 0; y < ROWS; ++y) held[wave][y][lane] = acc[y];
    __syncthreads();
    if (wave >= ROWS) return;   // a wavefront for every sixteen rows
    f32x4 sum = held[0][wave][lane];
#pragma unroll
    for (int j = 1; j < kFewWaves; ++j) sum += held[j][wave][lane];
    const int64_t row = 16 * wave + i;
    if (row >= p.rows) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int32_t col = column + 4 * g + j;
        if (col >= p.columns) break;
        if (p.part) p.part[((int64_t)part * p.rows + row) * p.part_stride + col] = sum[j];
        else finish_one<T, O>(p.f, row, col, sum[j] + (p.f.bias ? (float)((const T*)p.f.bias)[col] : 0.f));
    }
}

// The sums of the parts, in their order, and what follows them: VEC neighbouring columns of a row a lane
template <typename T, typename O, int VEC>
__global__ void __launch_bounds__(256) k_dense_parts(DenseArgs p) {
    const int64_t pieces = (p.columns + VEC - 1) / VEC, at = block_number() * 256 + threadIdx.x;
    if (at >= p.rows * pieces) return;
    const int64_t row = at / pieces;
    const int32_t col = (int32_t)(at - row * pieces) * VEC;
    const int64_t apart = p.rows * p.part_stride, from = row * p.part_stride + col;
    struct alignas(4 * VEC) Part { float v[VEC]; };
    float sum[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum[j] = p.f.bias ? (float)((const T*)p.f.bias)[col + j] : 0.f;
    constexpr int ahead = 8;
    for (int32_t s0 = 0; s0 < p.parts; s0 += ahead) {
        Part v[ahead];
#pragma unroll
        for (int s = 0; s < ahead; ++s)
            if (s0 + s < p.parts) v[s] = *(const Part*)(p.part + (s0 + s) * apart + from);
#pragma unroll
        for (int s = 0; s < ahead; ++s)
            if (s0 + s < p.parts)
#pragma unroll
                for (int j = 0; j < VEC; ++j) sum[j] += v[s].v[j];
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) finish_one<T, O>(p.f, row, col + j, sum[j]);
}

// Sums of columns: those of the parts added up, sixteen runs of parts side by side
constexpr int kSumColumns = 16;
static __global__ void __launch_bounds__(256) k_dense_sums(const float* part, int32_t parts, int64_t columns, float* to) {
    constexpr int runs = 256 / kSumColumns;
    __shared__ float held[runs][kSumColumns];
    const int col = threadIdx.x % kSumColumns, run = threadIdx.x / kSumColumns;
    const int64_t i = (int64_t)blockIdx.x * kSumColumns + col;
    const int32_t each = (parts + runs - 1) / runs, from = run * each, to_part = from + each < parts ? from + each : parts;
    float sum = 0.f;
    if (i < columns)
#pragma unroll 8
        for (int32_t s = from; s < to_part; ++s) sum += part[s * columns + i];
    held[run][col] = sum;
    __syncthreads();
    if (run > 0 || i >= columns) return;
    sum = 0.f;
#pragma unroll
    for (int r = 0; r < runs; ++r) sum += held[r][col];
    to[i] = sum;
}

// dz = dy act'(z), kept in the operands' type, as the products multiply it, and the sums of dz before it is rounded (of the rounded ones a float32 db
// would be good to 16 bits' rounding only). Slopes of SiLU and GELU go up to 1.13: in float16 7/8 of dz is kept, which no finite dy takes beyond 65,504, and the products'
// sums are multiplied by 8/7 (bfloat16 and float32 end where float32 does). db is float32 and has slopes to match: the longer fit of erfc (db of 65,536 rows
// with GELU good to 2.6e-7, 1.5e-6 with the one for 16-bit results; a call 2 % longer).  A workgroup takes 256 pieces of VEC columns: `wide` side by side, the others in the rows below, and goes
// down a run of rows.  Bound by its bytes: 65,536 x 2,048 in bfloat16 150 us (5.4 TB/s).
struct SlopeArgs {
    const void* dy;
    int64_t dy_stride;
    const void* z;
    int64_t z_stride;
    void* dz;
    float* sums;               // [parts][columns], or NULL
    int64_t rows, length;      // rows of a part
    int32_t columns, activation, wide;
    float factor;              // of dz as it is kept
};
template <typename T, int VEC>
__global__ void __launch_bounds__(256) k_dense_slope(SlopeArgs p) {
    __shared__ float held[256 * VEC];
    const int tid = threadIdx.x, across = tid % p.wide, down = tid / p.wide, step = 256 / p.wide;
    const int32_t strips = (p.columns + p.wide * VEC - 1) / (p.wide * VEC), strip = (int32_t)(blockIdx.x % (uint32_t)strips);
    const int64_t part = blockIdx.x / (uint32_t)strips, first = part * p.length, stop = first + p.length < p.rows ? first + p.length : p.rows;
    const int32_t col = (strip * p.wide + across) * VEC;
    struct alignas(sizeof(T) * VEC) Part { T v[VEC]; };
    float sum[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum[j] = 0.f;
    if (col < p.columns) {
        const auto rows = [&](auto act) {
            constexpr int ACT = decltype(act)::value;
#pragma unroll 4
            for (int64_t row = first + down; row < stop; row += step) {
                const Part g = *(const Part*)((const T*)p.dy + row * p.dy_stride + col), x = *(const Part*)((const T*)p.z + row * p.z_stride + col);
                Part out;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float v = (float)g.v[j] * activation_slope<ACT, sizeof(T) == 4, true>((float)x.v[j]);
                    sum[j] += v;
                    out.v[j] = (T)(p.factor * v);
                }
                *(Part*)((T*)p.dz + row * p.columns + col) = out;
            }
        };
        if (p.activation == kRelu) rows(Constant<kRelu>{});
        else if (p.activation == kSilu) rows(Constant<kSilu>{});
        else rows(Constant<kGelu>{});
    }
    if (!p.sums) return;
#pragma unroll
    for (int j = 0; j < VEC; ++j) held[j * 256 + tid] = sum[j];
    __syncthreads();
    if (down > 0 || col >= p.columns) return;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        float all = 0.f;
        for (int r = 0; r < step; ++r) all += held[j * 256 + r * p.wide + across];
        p.sums[part * p.columns + col + j] = all;
    }
}

}  // namespace nomad_dense
