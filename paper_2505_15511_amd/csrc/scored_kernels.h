// Routing by scores (gfx950): sigmoid or softmax scores, a bias that has a say in the choice but not in the weights, groups of experts of
// which a row uses a few, weights renormalised and scaled.
//
//   s_e = 1 / (1 + e^-l_e) or e^l_e / sum e^l,   c_e = s_e + b_e,   G groups of neighbours, scored by their one or two largest c
//   the k largest c in the best groups;   w_j = scale s_j [/ sum over the chosen]
//
// What is chosen is what 64 bits say.  A row's c are found in 32 bits first, whose error has a bound (Trust); where two c (or two groups'
// scores) that a choice lies between are nearer than that, and do not come of the same logit and bias, the row is done again in
// 64 bits.  Without a bias experts are compared by their logits, which are exact.
//
// k_scored_quick     rows of up to 256 experts: read once, held by sixteen lanes
// k_scored_rest      the rows that it leaves to 64 bits
// k_scored_pick      rows of more experts, or of more than 16 groups: read several times, from the caches after the first
// k_scored_small     all of it in one workgroup
// k_scored_gradient_rows, k_scored_gradient   the logits' gradient, made in LDS; of a softmax over all experts, and of rows of more than 512
//
// Bound by arithmetic and bytes alike: 500,000 rows of 256 in float32, sigmoid and bias, k = 2: 142 us (3.6 TB/s; exponentials and reciprocals, at a
// quarter of the other instructions' rate, are a third of it); 300,000 rows in bfloat16, k = 8 of 4 groups out of 8, 147 us; the gradients 112 (4.7 TB/s written) and 47.
// Rows for 64 bits cost a wavefront's way each: with a bias of zero and sigmoids that are all but 1 every row is one, and 500,000 of 256 take 1,050 us a call (170 with a bias of
// 0.02 deviations), 300,000 with k = 8 of groups 1,200 (176); where all logits are the same 1,070 and 1,210.  Over 256 experts, 8,192 rows of 4,096 in float32,
// k = 2, take 344 us a call by their logits and 515 with a bias, 26 us of bytes.
#pragma once
#include "route_kernels.h"
#include "scored_keys.h"

namespace nomad_router {

constexpr int kMaxRouteGroups = 64;

struct ScoredArgs {
    RouteArgs r;               // (normalize among them)
    const float* bias;         // NULL: none
    float scale;
    int32_t sigmoid;           // 0: softmax
    int32_t groups, top_groups, best;
    int32_t size;              // experts a group
    int32_t team;              // lanes that share a group while groups are scored, a power of two
    int32_t open_team;         // the same while experts of open groups are compared
};

// ---- among the LANES neighbours that share a row

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
template <int CTRL, typename V>
__device__ __forceinline__ V moved(V v) {
    if constexpr (sizeof(V) == 4) {
        return __builtin_bit_cast(V, dpp<CTRL>(__builtin_bit_cast(uint32_t, v)));
    } else {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        return __builtin_bit_cast(V, (uint64_t)dpp<CTRL>((uint32_t)(u >> 32)) << 32 | dpp<CTRL>((uint32_t)u));
    }
}
// op over all LANES values, for each of them: neighbours, pairs, mirrored halves and mirrored rows of 16 without a way through LDS
template <int LANES, typename V, typename F>
__device__ __forceinline__ V fold(V v, F op) {
    v = op(v, moved<0xb1>(v));     // lane ^ 1
    v = op(v, moved<0x4e>(v));     // lane ^ 2
    v = op(v, moved<0x141>(v));    // 7 - lane: the other four
    v = op(v, moved<0x140>(v));    // 15 - lane: the other eight
    if (LANES == 64) {
        v = op(v, (V)__shfl_xor(v, 16));
        v = op(v, (V)__shfl_xor(v, 32));
    }
    return v;
}
template <int LANES, typename V>
__device__ __forceinline__ V most_of(V v) { return fold<LANES>(v, [](V a, V b) { return a > b ? a : b; }); }
template <int LANES, typename V>
__device__ __forceinline__ V least_of(V v) { return fold<LANES>(v, [](V a, V b) { return a < b ? a : b; }); }
template <int LANES>
__device__ __forceinline__ bool any_of(bool v, int lane) {   // of the row's lanes
    const uint64_t all = __ballot(v);
    return LANES == 64 ? all != 0 : (all >> (lane & ~(LANES - 1)) & ((1ull << (LANES & 63)) - 1)) != 0;
}

// ---- scores

__device__ __forceinline__ float score_sigmoid(float v, float) { return __builtin_amdgcn_rcpf(1.f + __expf(-v)); }
__device__ __forceinline__ double score_sigmoid(float v, double) { return 1.0 / (1.0 + exp(-(double)v)); }
__device__ __forceinline__ float exponent(float x) { return expf(x); }
__device__ __forceinline__ double exponent(double x) { return exp(x); }

template <typename R>
struct Scores {
    const float* bias;
    bool sigmoid, by_logit;    // by_logit: c is the logit
    R top, inv;                // softmax: the largest logit, one over the sum
    __device__ __forceinline__ R score(float v) const {
        if (sigmoid) return score_sigmoid(v, (R)0);
        return exponent((R)v - top) * inv;
    }
    // -inf: not to be chosen
    __device__ __forceinline__ R of(float v, uint32_t e) const {
        if (by_logit) return (R)v;
        if (v == -INFINITY) return (R)-INFINITY;
        R c = score(v);
        if (bias) c += (R)bias[e];
        return c == c ? c : (R)-INFINITY;
    }
};

// The K largest c that a lane has seen, first ones first among equals, and the largest that it has let go
template <int K, typename R>
struct Largest {
    R c[K];
    uint32_t e[K];
    R gone;
    __device__ __forceinline__ Largest() {
#pragma unroll
        for (int j = 0; j < K; ++j) { c[j] = (R)-INFINITY; e[j] = 0; }
        gone = (R)-INFINITY;
    }
    __device__ __forceinline__ void take(R x, uint32_t index) {
        if (!(x > c[K - 1])) {
            gone = x > gone ? x : gone;
            return;
        }
        gone = c[K - 1] > gone ? c[K - 1] : gone;
#pragma unroll
        for (int j = K - 1; j >= 0; --j) {
            const bool before = j > 0 && x > c[j > 0 ? j - 1 : 0];
            if (before) { c[j] = c[j > 0 ? j - 1 : 0]; e[j] = e[j > 0 ? j - 1 : 0]; }
            else if (x > c[j]) { c[j] = x; e[j] = index; }
        }
    }
    __device__ __forceinline__ void drop_first() {
#pragma unroll
        for (int i = 0; i + 1 < K; ++i) { c[i] = c[i + 1]; e[i] = e[i + 1]; }
        c[K - 1] = (R)-INFINITY;
    }
};

// elements begin .. end - 1 of a row by `lanes` lanes, four loads on their way at once; VEC: 16 bytes a load, begin and end on their borders
template <typename T, bool VEC, typename F>
__device__ __forceinline__ void each_of(const T* row, int32_t begin, int32_t end, int lane, int lanes, F visit) {
    constexpr int epc = VEC ? 16 / (int)sizeof(T) : 1;
    for (int32_t c0 = begin + lane * epc; c0 < end; c0 += 4 * lanes * epc) {
        T part[4][epc];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int32_t c = c0 + b * lanes * epc;
            if (c >= end) continue;
            if (VEC) *(uint4*)part[b] = *(const uint4*)(row + c);
            else part[b][0] = row[c];
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int32_t c = c0 + b * lanes * epc;
            if (c >= end) continue;
#pragma unroll
            for (int i = 0; i < epc; ++i) visit(value_of(part[b][i]), (uint32_t)(c + i));
        }
    }
}

// What 32 bits can be wrong by: a sigmoid by 2^-23 (a slope of 1/4 on an argument good to 2^-24 of itself, a power of two and a
// reciprocal good to a unit), a softmax by a unit for every term of its sum that a lane adds up and a few more, relative to the largest
// score; then the sum with the bias.  Two c that are this far apart are in the right order.
struct Trust {
    float near;
    __device__ __forceinline__ float at(float c) const { return near + 0x1p-21f * fabsf(c); }
};

// One row by LANES lanes: its experts, best first (every lane of the row gets them; k <= K); false: 32 bits cannot tell
template <typename R, typename T, int LANES, int K, bool VEC>
__device__ __forceinline__ bool choose(const T* row, const ScoredArgs& p, int sub, int32_t (&expert)[K]) {
    constexpr bool FIRST = sizeof(R) == 4;
    const int lane = (int)(threadIdx.x & 63), base = lane - sub;
    const int32_t n_experts = p.r.n_experts;
    const R none = (R)-INFINITY;
    Scores<R> s;
    s.bias = p.bias;
    s.sigmoid = p.sigmoid != 0;
    s.by_logit = p.bias == nullptr;
    s.top = s.inv = (R)0;
    float near = 0x1p-21f;
    if (!s.sigmoid && (p.bias || (p.groups > 1 && p.best == 2))) {
        float top = -INFINITY;
        each_of<T, VEC>(row, 0, n_experts, sub, LANES, [&](float v, uint32_t) { top = fmaxf(top, v); });
        top = most_of<LANES>(top);
        s.top = (R)top;
        R sum = (R)0;
        each_of<T, VEC>(row, 0, n_experts, sub, LANES, [&](float v, uint32_t) { sum += exponent((R)v - s.top); });
        sum = fold<LANES>(sum, [](R a, R b) { return a + b; });
        s.inv = (R)1 / sum;
        if (!(top < INFINITY)) s.by_logit = true;   // a logit of +inf (or a row without any): the row has no scores
        near = (float)s.inv * ((float)(n_experts / LANES) + 32.f) * 0x1p-23f;
    }
    const Trust trust{near};
    bool sure = true;
    uint64_t open = 1;
    if (p.groups > 1) {
        // c of groups: by teams of lanes, a few groups one after the other
        Scores<R> in_group = s;
        const bool as_logits = s.by_logit && (p.best == 1 || !(s.sigmoid || s.top < (R)INFINITY));
        if (s.by_logit && !as_logits) in_group.by_logit = false;   // (two scores are added: logits do not do)
        const int teams = LANES / p.team, mine = sub / p.team, at = sub % p.team;
        R score[kMaxRouteGroups / 16];
        float large = 0.f;   // the largest magnitude in a sum
#pragma unroll
        for (int t = 0; t < kMaxRouteGroups / 16; ++t) {
            score[t] = none;
            const int g = t * teams + mine;
            if (t * teams < p.groups) {
                R first = none, second = none;
                if (g < p.groups)
                    each_of<T, VEC>(row, g * p.size, (g + 1) * p.size, at, p.team, [&](float v, uint32_t e) {
                        const R c = in_group.of(v, e);
                        second = c > first ? first : c > second ? c : second;
                        first = c > first ? c : first;
                    });
                for (int d = 1; d < p.team; d <<= 1) {
                    const R other = __shfl_xor(first, d), behind = __shfl_xor(second, d), low = first < other ? first : other;
                    second = second > behind ? second : behind;
                    second = low > second ? low : second;
                    first = first > other ? first : other;
                }
                const bool both = p.best == 2 && second > none;
                score[t] = both ? first + second : first;
                if (FIRST && first > none) large = fmaxf(large, fmaxf(fabsf((float)first), both ? fabsf((float)second) : 0.f));
            }
        }
        // a group is open if fewer than top_groups are ahead of it
        int ahead[kMaxRouteGroups / 16] = {};
        for (int h = 0; h < p.groups; ++h) {
            const int from = base + (h % teams) * p.team, round = h / teams;
            R other = score[0];
#pragma unroll
            for (int t = 1; t < kMaxRouteGroups / 16; ++t) other = round == t ? score[t] : other;
            other = __shfl(other, from);
#pragma unroll
            for (int t = 0; t < kMaxRouteGroups / 16; ++t) {
                const int g = t * teams + mine;
                ahead[t] += other > score[t] || (other == score[t] && h < g) ? 1 : 0;
            }
        }
        open = 0;
        R lowest = (R)INFINITY, highest = none;   // of the open groups, of the others
#pragma unroll
        for (int t = 0; t < kMaxRouteGroups / 16; ++t) {
            const int g = t * teams + mine;
            if (g >= p.groups || !(score[t] > none)) continue;
            if (ahead[t] < p.top_groups) {
                open |= 1ull << g;
                lowest = score[t] < lowest ? score[t] : lowest;
            } else {
                highest = score[t] > highest ? score[t] : highest;
            }
        }
        open = fold<LANES>(open, [](uint64_t a, uint64_t b) { return a | b; });
        if (FIRST && !as_logits) {
            lowest = least_of<LANES>(lowest);
            highest = most_of<LANES>(highest);
            if (highest > none && !(lowest - highest > 2.f * trust.at(most_of<LANES>(large)))) sure = false;
        }
    }
    Largest<K, R> best;
    const int open_teams = LANES / p.open_team, in_team = sub % p.open_team;
    uint64_t left = open;
    for (int skip = sub / p.open_team; skip > 0; --skip) left &= left - 1;
    while (left) {
        const int g = __builtin_ctzll(left);
        each_of<T, VEC>(row, g * p.size, (g + 1) * p.size, in_team, p.open_team, [&](float v, uint32_t e) { best.take(s.of(v, e), e); });
        for (int skip = open_teams; skip > 0; --skip) left &= left - 1;
    }
    R last = none;          // the k-th c
    R before = none;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        expert[j] = -1;
        if (j >= p.r.k) continue;
        const R c = most_of<LANES>(best.c[0]);
        const uint32_t e = least_of<LANES>(best.c[0] == c ? best.e[0] : 0xffffffffu);
        if (!(c > none)) { last = none; continue; }
        if (best.c[0] == c && best.e[0] == e) best.drop_first();
        expert[j] = (int32_t)e;
        if (FIRST && !s.by_logit && j > 0 && !(before - c > trust.at((float)before))) {
            const int32_t other = expert[j > 0 ? j - 1 : 0];
            if (!(before == c && value_of(row[other]) == value_of(row[e]) && (!s.bias || s.bias[other] == s.bias[e]))) sure = false;
        }
        before = last = c;
    }
    if (FIRST && !s.by_logit && last > none) {
        // whatever was not chosen is further below the last one than 32 bits are wrong, or its equal
        const R border = last - (R)trust.at((float)last);
        if (!(best.gone < border) && best.gone > none) sure = false;
        uint32_t at = 0;
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (j == p.r.k - 1) at = (uint32_t)expert[j];
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (best.c[j] > none && !(best.c[j] < border) &&
                !(best.c[j] == last && value_of(row[at]) == value_of(row[best.e[j]]) && (!s.bias || s.bias[at] == s.bias[best.e[j]])))
                sure = false;
    }
    return !FIRST || !any_of<LANES>(!sure, lane);
}

// ---- rows of up to 16 CAP experts, whose logits 16 lanes hold in registers, CAP each, and read once
//
// A lane's experts are of one group.  A sum c becomes a key of 32 bits: a whole number of steps above the smallest bias, below it the expert's
// number, lower ones larger, so that comparing, sorting and taking the best are one instruction each.  (A step is 2^-24 or 2^-25 of the sums'
// range.)  Without a bias the step is what is left of a logit's own order, all of it for logits of 16 bits.

__device__ __forceinline__ float power_of_e(float x) {   // for x <= 0, to a unit or two: what rounding x log2(e) loses is put back
    const float power = x * 1.44269504f, rest = fmaf(x, 1.92596303e-8f, fmaf(x, 1.44269504f, -power)), e = __builtin_amdgcn_exp2f(power);
    return x < -150.f ? 0.f : fmaf(e, rest * 0.69314718f, e);
}

template <typename T, int CAP, int K, bool VEC, bool GROUPED>
struct Quick {
    static constexpr int kLanes = 16, kEpc = VEC ? 16 / (int)sizeof(T) : 1, kChunks = CAP / kEpc;
    static constexpr int kBits = CAP == 8 ? 7 : 8;                            // of an expert's number
    static constexpr float kSteps = (float)((1ull << (32 - kBits)) - 64);     // (rounding takes a key a few steps further)
    struct alignas(VEC ? 16 : sizeof(T)) Chunk { T v[kEpc]; };
    const ScoredArgs& p;
    int sub, lane, group, from;            // from: of the group, the lane's first expert
    int32_t first;                         // expert
    bool hopeless;
    float low;                             // the smallest bias
    float steps;                           // of the keys: a unit's
    float start[CAP];                      // steps of the bias above the smallest one
    float slack;                           // of a sum, beside its score's

    __device__ __forceinline__ Quick(const ScoredArgs& args, int tid) : p(args) {
        sub = tid % kLanes;
        lane = tid & 63;
        group = sub / p.team;
        from = sub % p.team * kEpc;
        first = group * p.size + from;
        hopeless = false;
        low = 0.f;
        float high = 0.f;
#pragma unroll
        for (int i = 0; i < CAP; ++i) start[i] = 0.f;
        if (p.bias) {
            low = INFINITY;
            high = -INFINITY;
            float wrong = 0.f;
#pragma unroll
            for (int i = 0; i < CAP; ++i) start[i] = p.bias[there(i) ? number(i) : 0];   // (all on their way at once)
#pragma unroll
            for (int i = 0; i < CAP; ++i) {
                low = fminf(low, start[i]);
                high = fmaxf(high, start[i]);
                wrong += start[i] * 0.f;               // NaN where it is not a number
            }
            low = least_of<kLanes>(low);
            high = most_of<kLanes>(high);
            hopeless = fold<kLanes>(wrong, [](float a, float b) { return a + b; }) != 0.f || !(high - low < 1e30f);
        }
        steps = kSteps / (1.f + (high - low));
#pragma unroll
        for (int i = 0; i < CAP; ++i) start[i] = (start[i] - low) * steps + 1.f;
        slack = 0x1p-21f * (fmaxf(fabsf(low), fabsf(high)) + 1.f);
    }
    __device__ __forceinline__ int32_t offset(int i) const { return (i / kEpc) * (p.team * kEpc) + i % kEpc; }
    __device__ __forceinline__ int32_t number(int i) const { return first + offset(i); }
    __device__ __forceinline__ bool there(int i) const { return group < p.groups && from + offset(i) < p.size; }

    // what a lane's places hold that no expert has
    __device__ __forceinline__ static void clear(Chunk (&raw)[kChunks]) {
#pragma unroll
        for (int j = 0; j < kChunks; ++j)
#pragma unroll
            for (int i = 0; i < kEpc; ++i) raw[j].v[i] = (T)-INFINITY;
    }
    __device__ __forceinline__ void load(const T* row, Chunk (&raw)[kChunks]) const {
#pragma unroll
        for (int j = 0; j < kChunks; ++j)
            if (there(j * kEpc)) raw[j] = *(const Chunk*)(row + number(j * kEpc));
    }

    // The row's experts, best first, for every lane of the row; false: not to be told by 32 bits.  top, sum: of a softmax
    __device__ __forceinline__ bool choose_quick(const T* row, const Chunk (&raw)[kChunks], int32_t (&expert)[K], float& top, float& sum) const {
        const float none = -INFINITY;
        float v[CAP];
#pragma unroll
        for (int i = 0; i < CAP; ++i) v[i] = fmaxf((float)raw[i / kEpc].v[i % kEpc], none);   // (a NaN is -inf)
        bool sure = !hopeless;
        top = none;
        sum = 1.f;
        float near = 0x1p-21f;
        const bool by_logit = p.bias == nullptr, two = GROUPED && p.best == 2, scored = !by_logit || two;
        float c[CAP];
        if (!p.sigmoid && (scored || !p.r.normalize)) {
#pragma unroll
            for (int i = 0; i < CAP; ++i) top = fmaxf(top, v[i]);
            top = most_of<kLanes>(top);
            if (scored && !(top < INFINITY)) sure = false;
            const float base = top > none ? top : 0.f;
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < CAP; ++i) {
                c[i] = power_of_e(v[i] - base);
                sum += c[i];
            }
            sum = fold<kLanes>(sum, [](float a, float b) { return a + b; });
            const float inv = 1.f / sum;
            near = inv * ((float)CAP + 32.f) * 0x1p-23f;
#pragma unroll
            for (int i = 0; i < CAP; ++i) c[i] *= inv;
        } else if (scored) {
#pragma unroll
            for (int i = 0; i < CAP; ++i) c[i] = score_sigmoid(v[i], 0.f);
        }
        if (!by_logit)
#pragma unroll
            for (int i = 0; i < CAP; ++i) c[i] = fmaf(c[i], steps, start[i]);   // (the sum, in steps)
        bool open = true;
        if (GROUPED) {
            const bool as_logits = by_logit && !two;
            float one = none, second = none, score;
#pragma unroll
            for (int i = 0; i < CAP; ++i) {
                const float x = v[i] == none ? none : as_logits ? v[i] : c[i];
                second = fmaxf(second, fminf(one, x));
                one = fmaxf(one, x);
            }
            const auto join = [&](float other, float behind) {
                second = fmaxf(fmaxf(second, behind), fminf(one, other));
                one = fmaxf(one, other);
            };
            if (p.team > 1) join(moved<0xb1>(one), moved<0xb1>(second));
            if (p.team > 2) join(moved<0x4e>(one), moved<0x4e>(second));
            if (p.team > 4) join(moved<0x141>(one), moved<0x141>(second));
            const bool both = p.best == 2 && second > none;
            score = both ? one + second : one;
            if (!by_logit) score = both ? fmaf(score - 2.f, 1.f / steps, 2.f * low) : fmaf(score - 1.f, 1.f / steps, low);
            int ahead = 0;
            const int base = lane - sub;
            for (int g = 0; g < p.groups; ++g) {
                const float other = __shfl(score, base + g * p.team);
                ahead += other > score || (other == score && g < group) ? 1 : 0;
            }
            open = group < p.groups && score > none && ahead < p.top_groups;
            if (!as_logits) {
                const float lowest = least_of<kLanes>(open ? score : INFINITY), highest = most_of<kLanes>(open || group >= p.groups ? none : score);
                if (highest > none && !(lowest - highest > 2.f * (near + slack * 2.f))) sure = false;
            }
        }
        constexpr uint32_t mask = (1u << kBits) - 1u;
        uint32_t key[CAP];
        if (by_logit) {
#pragma unroll
            for (int i = 0; i < CAP; ++i) {
                const uint32_t u = __float_as_uint(v[i] + 0.f);   // (both zeros are the same number)
                key[i] = u & 0x80000000u ? ~u : u | 0x80000000u;
            }
#pragma unroll
            for (int i = 0; i < CAP; ++i) key[i] = (key[i] & ~mask) | (mask - (uint32_t)number(i));
        } else {
#pragma unroll
            for (int i = 0; i < CAP; ++i) key[i] = (uint32_t)c[i] << kBits | (mask - (uint32_t)number(i));
        }
#pragma unroll
        for (int i = 0; i < CAP; ++i) key[i] = v[i] > none ? key[i] : 0u;
        Kept<CAP, K> kept;
        kept.keep(key, !GROUPED || open);
        // steps within which keys may be in the wrong order
        const uint32_t apart = by_logit ? 0u : (uint32_t)fminf((near + slack) * steps, 1e9f) + 2u;
        const auto same = [&](uint32_t a, uint32_t b) {   // (a key's expert and another's: equal in every bit of logit and bias)
            const int32_t ea = (int32_t)(mask - (a & mask)), eb = (int32_t)(mask - (b & mask));
            return value_of(row[ea]) == value_of(row[eb]) && (by_logit || p.bias[ea] == p.bias[eb]);
        };
        const bool exact = by_logit && sizeof(T) == 2;    // equal steps are equal logits
        uint32_t last = 0, before = 0;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            expert[j] = -1;
            if (j >= p.r.k) continue;
            const uint32_t best = most_of<kLanes>(kept.list[0]);
            kept.give(best);
            if (best) expert[j] = (int32_t)(mask - (best & mask));
            if (!exact && best && before && (before >> kBits) - (best >> kBits) <= apart && !same(before, best)) sure = false;
            before = best;
            last = j == p.r.k - 1 ? best : last;
        }
        if (!exact && kept.unsure(last, apart, kBits, same)) sure = false;
        return !any_of<kLanes>(!sure, lane);
    }
};

// log s up to what the chosen have in common, as a factor: s_j / s_m, for any logits
__device__ __forceinline__ float sigmoid_ratio(float v, float m) {
    return power_of_e(fminf(v, 0.f) - fminf(m, 0.f)) * ((1.f + power_of_e(-fabsf(m))) * __builtin_amdgcn_rcpf(1.f + power_of_e(-fabsf(v))));
}

// A row's weights from its experts: lane j of the row gets the j-th (top, sum: of a softmax over all)
template <typename T, int LANES, int K>
__device__ __forceinline__ float weigh(const T* row, const ScoredArgs& p, int sub, const int32_t (&expert)[K], float top, float sum) {
    int32_t mine = -1;
#pragma unroll
    for (int j = 0; j < K; ++j)
        if (j == sub && j < p.r.k) mine = expert[j];
    const float v = mine >= 0 ? value_of(row[mine]) : -INFINITY;
    float share = 0.f;
    if (p.r.normalize) {
        const float most = most_of<LANES>(v);
        if (mine >= 0) share = p.sigmoid ? sigmoid_ratio(v, most) : power_of_e(v - most);
        const float chosen = fold<LANES>(share, [](float a, float b) { return a + b; });
        if (mine >= 0) share /= chosen;   // (of one alone exactly 1)
    } else if (p.sigmoid) {
        if (mine >= 0) share = power_of_e(fminf(v, 0.f)) * __builtin_amdgcn_rcpf(1.f + power_of_e(-fabsf(v)));
    } else if (mine >= 0) {
        share = expf(v - top) / sum;
    }
    return p.scale * share;
}

// One row: experts and, in lane j of the row for its j-th expert, the weight.  R = double: 32 bits have been tried
template <typename R, typename T, int LANES, int K, bool VEC>
__device__ __forceinline__ float score_row(const T* row, const ScoredArgs& p, int sub, int32_t (&expert)[K]) {
    if (sizeof(R) == 8 || !choose<float, T, LANES, K, VEC>(row, p, sub, expert)) (void)choose<double, T, LANES, K, false>(row, p, sub, expert);
    float top = -INFINITY, sum = 0.f;
    if (!p.sigmoid && !p.r.normalize) {
        each_of<T, VEC>(row, 0, p.r.n_experts, sub, LANES, [&](float x, uint32_t) { top = fmaxf(top, x); });
        top = most_of<LANES>(top);
        each_of<T, VEC>(row, 0, p.r.n_experts, sub, LANES, [&](float x, uint32_t) { sum += expf(x - top); });
        sum = fold<LANES>(sum, [](float a, float b) { return a + b; });
    }
    return weigh<T, LANES, K>(row, p, sub, expert, top, sum);
}

// Chunks of rows as in k_route_pick, sixteen lanes a row; a lane asks for its next row before it looks at this one.  Rows that 32 bits do not tell
// apart are marked and left to k_scored_rest: 64 bits in here took the registers of every row (500,000 rows of 256 in float32: 217 us).
constexpr int kQuickThreads = 512;
constexpr int32_t kLeft = -2;
template <typename T, int CAP, int K, bool VEC, bool GROUPED>
__global__ void __launch_bounds__(kQuickThreads) k_scored_quick(ScoredArgs p) {
    typedef Quick<T, CAP, K, VEC, GROUPED> Row;
    __shared__ int32_t tally[16 * CAP];
    const int tid = threadIdx.x, sub = tid % 16;
    if (tid < p.r.n_experts) tally[tid] = 0;
    __syncthreads();
    const Row q(p, tid);
    const int64_t first = (int64_t)blockIdx.x * p.r.chunk, stop = first + p.r.chunk < p.r.n ? first + p.r.chunk : p.r.n;
    int64_t i = first + tid / 16;
    typename Row::Chunk raw[Row::kChunks], ahead[Row::kChunks];
    Row::clear(raw);
    Row::clear(ahead);
    if (i < stop) q.load((const T*)p.r.logits + i * p.r.stride, raw);
    for (; i < stop; i += kQuickThreads / 16) {
        const T* row = (const T*)p.r.logits + i * p.r.stride;
        const int64_t next = i + kQuickThreads / 16;
        if (next < stop) q.load((const T*)p.r.logits + next * p.r.stride, ahead);
        int32_t expert[K];
        float top, sum;
        const bool sure = q.choose_quick(row, raw, expert, top, sum);
        const float weight = weigh<T, 16, K>(row, p, sub, expert, top, sum);
        int32_t mine = kLeft;
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (sure && sub == j) mine = expert[j];
        if (sub < p.r.k) {
            p.r.experts[i * p.r.k + sub] = mine;
            p.r.weights[i * p.r.k + sub] = weight;
            if (mine >= 0) atomicAdd(&tally[mine], 1);
        }
#pragma unroll
        for (int j = 0; j < Row::kChunks; ++j) raw[j] = ahead[j];
    }
    __syncthreads();
    if (tid < p.r.n_experts) p.r.counts[(int64_t)blockIdx.x * p.r.n_experts + tid] = tally[tid];
}

// The rows that k_scored_quick has marked, 64 bits for all of a row's experts; the chunk's counts with theirs
constexpr int kRestThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kRestThreads) k_scored_rest(ScoredArgs p) {
    __shared__ int32_t rows[kRestThreads], left;
    const int tid = threadIdx.x, sub = tid % 64;   // (a wavefront a row: there are few, and the way of one is what the kernel takes)
    const int64_t first = (int64_t)blockIdx.x * p.r.chunk, stop = first + p.r.chunk < p.r.n ? first + p.r.chunk : p.r.n;
    for (int64_t i0 = first; i0 < stop; i0 += kRestThreads) {
        if (tid == 0) left = 0;
        __syncthreads();
        if (i0 + tid < stop && p.r.experts[(i0 + tid) * p.r.k] == kLeft) rows[atomicAdd(&left, 1)] = tid;
        __syncthreads();
        const int32_t all = left;
        for (int32_t at = tid / 64; at < all; at += kRestThreads / 64) {   // (in any order: each row by itself)
            const int64_t i = i0 + rows[at];
            int32_t expert[kMaxK];
            const float weight = score_row<double, T, 64, kMaxK, false>((const T*)p.r.logits + i * p.r.stride, p, sub, expert);
            int32_t mine = -1;
#pragma unroll
            for (int j = 0; j < kMaxK; ++j)
                if (sub == j) mine = expert[j];
            if (sub < p.r.k) {
                p.r.experts[i * p.r.k + sub] = mine;
                p.r.weights[i * p.r.k + sub] = weight;
                if (mine >= 0) atomicAdd(&p.r.counts[(int64_t)blockIdx.x * p.r.n_experts + mine], 1);
            }
        }
        __syncthreads();
    }
}

template <typename T, int LANES, int K, bool VEC>
__global__ void __launch_bounds__(kPickThreads) k_scored_pick(ScoredArgs p) {
    extern __shared__ int32_t tally[];
    const int tid = threadIdx.x, sub = tid % LANES;
    for (int32_t e = tid; e < p.r.n_experts; e += kPickThreads) tally[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * p.r.chunk, stop = first + p.r.chunk < p.r.n ? first + p.r.chunk : p.r.n;
    for (int64_t i = first + tid / LANES; i < stop; i += kPickThreads / LANES) {
        int32_t expert[K];
        const float weight = score_row<float, T, LANES, K, VEC>((const T*)p.r.logits + i * p.r.stride, p, sub, expert);
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (j < p.r.k && sub == j) {
                p.r.experts[i * p.r.k + j] = expert[j];
                p.r.weights[i * p.r.k + j] = weight;
                if (expert[j] >= 0) atomicAdd(&tally[expert[j]], 1);
            }
    }
    __syncthreads();
    for (int32_t e = tid; e < p.r.n_experts; e += kPickThreads) p.r.counts[(int64_t)blockIdx.x * p.r.n_experts + e] = tally[e];
}

template <typename T, int LANES, int K, bool VEC>
__global__ void __launch_bounds__(kSmallThreads) k_scored_small(ScoredArgs p) {
    extern __shared__ int32_t next[];   // [n_experts], behind it the experts of the slots [n k]
    int32_t* slots = next + p.r.n_experts;
    const int tid = threadIdx.x, sub = tid % LANES;
    for (int32_t e = tid; e < p.r.n_experts; e += kSmallThreads) next[e] = 0;
    __syncthreads();
    for (int64_t i = tid / LANES; i < p.r.n; i += kSmallThreads / LANES) {
        int32_t expert[K];
        const float weight = score_row<float, T, LANES, K, VEC>((const T*)p.r.logits + i * p.r.stride, p, sub, expert);
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (j < p.r.k && sub == j) {
                p.r.experts[i * p.r.k + j] = expert[j];
                p.r.weights[i * p.r.k + j] = weight;
                slots[i * p.r.k + j] = expert[j];
                if (expert[j] >= 0) atomicAdd(&next[expert[j]], 1);
            }
    }
    __syncthreads();
    place_few(p.r, next, slots, tid);
}

struct ScoredGradientArgs {
    RouteGradientArgs r;
    float scale;
    int32_t sigmoid;
};

// Through the logarithms of the chosen scores: d log s_j / d l_j = 1 - s_j = 1 / (1 + e^l_j) of a sigmoid, 1 of a softmax among the chosen;
// a softmax over all experts as in k_route_gradient
template <typename T, int LANES, int K, bool VEC>
__global__ void __launch_bounds__(256) k_scored_gradient(ScoredGradientArgs p) {
    const int sub = threadIdx.x % LANES;
    const int64_t i = block_number() * (256 / LANES) + threadIdx.x / LANES;
    if (i >= p.r.n) return;   // (whole rows leave; the others' lanes stay together)
    constexpr int epc = VEC ? 16 / (int)sizeof(T) : 1;
    const T* row = (const T*)p.r.logits + i * p.r.stride;
    int32_t expert[K];
    float weight[K], given[K], inner = 0.f;
#pragma unroll
    for (int j = 0; j < K; ++j) {   // (all loads at once, no branches: their way is what a row takes)
        const int64_t at = i * p.r.k + (j < p.r.k ? j : 0);
        expert[j] = p.r.experts[at];
        weight[j] = p.r.weights[at];
        given[j] = p.r.dweights[at];
    }
#pragma unroll
    for (int j = 0; j < K; ++j) {
        if (j >= p.r.k || expert[j] >= p.r.n_experts) expert[j] = -1;
        weight[j] = expert[j] < 0 ? 0.f : weight[j];
        given[j] = expert[j] < 0 ? 0.f : given[j];
        inner += (p.r.normalize ? weight[j] / p.scale : weight[j]) * given[j];   // (a share, exactly 1 of one expert alone, whose gradient is 0)
    }
    T* out = (T*)p.r.dlogits + i * p.r.n_experts;
    if (p.sigmoid || p.r.normalize || expert[0] < 0) {
#pragma unroll
        for (int j = 0; j < K; ++j) {
            given[j] = weight[j] * (given[j] - (p.r.normalize ? inner : 0.f));
            if (p.sigmoid && expert[j] >= 0) given[j] /= 1.f + expf(value_of(row[expert[j]]));
        }
        for (int32_t c = sub * epc; c < p.r.n_experts; c += LANES * epc) {
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
    float top = -INFINITY, sum = 0.f;
    each<T, LANES, VEC>(row, p.r.n_experts, sub, [&](float v, uint32_t) { top = fmaxf(top, v); });
    top = reduce<LANES>(top, [](float a, float b) { return fmaxf(a, b); });
    each<T, LANES, VEC>(row, p.r.n_experts, sub, [&](float v, uint32_t) { sum += expf(v - top); });
    sum = reduce<LANES>(sum, [](float a, float b) { return a + b; });
    for (int32_t c = sub * epc; c < p.r.n_experts; c += LANES * epc) {
        T in[epc], part[epc];
        if (VEC) *(uint4*)in = *(const uint4*)(row + c);
        else in[0] = row[c];
#pragma unroll
        for (int t = 0; t < epc; ++t) {
            float v = -inner;
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (expert[j] == c + t) v += p.scale * given[j];
            part[t] = (T)(expf(value_of(in[t]) - top) / sum * v);
        }
        store_chunk<T, VEC>(out + c, part);
    }
}

// The same where a row's gradient is 0 but for its experts: lane j of a row has the j-th, puts it into the row in LDS, and the row leaves whole (a
// comparison of every expert with every chosen one took 300,000 rows of 256 in bfloat16, k = 8, 114 us)
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_scored_gradient_rows(ScoredGradientArgs p) {
    extern __shared__ uint4 rows[];
    constexpr int epc = VEC ? 16 / (int)sizeof(T) : 1;
    const int sub = threadIdx.x % 16, line = threadIdx.x / 16;
    const int64_t i = block_number() * 16 + line;
    if (i >= p.r.n) return;   // (whole rows leave, and a row's lanes are of one wavefront: nothing here waits for others)
    const int32_t chunks = (p.r.n_experts * (int32_t)sizeof(T) + 15) / 16;
    uint4* held = rows + line * chunks;
    int32_t expert = -1;
    float weight = 0.f, given = 0.f;
    if (sub < p.r.k) {
        const int64_t at = i * p.r.k + sub;
        expert = p.r.experts[at];
        weight = p.r.weights[at];
        given = p.r.dweights[at];
        if (expert >= p.r.n_experts) expert = -1;
    }
    for (int32_t c = sub; c < chunks; c += 16) held[c] = make_uint4(0, 0, 0, 0);
    const float inner = fold<16>(expert < 0 || !p.r.normalize ? 0.f : weight / p.scale * given, [](float a, float b) { return a + b; });
    float value = weight * (given - inner);
    if (expert >= 0 && p.sigmoid) value /= 1.f + expf(value_of(((const T*)p.r.logits)[i * p.r.stride + expert]));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (expert >= 0) ((T*)held)[expert] = (T)value;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    T* out = (T*)p.r.dlogits + i * p.r.n_experts;
    for (int32_t c = sub * epc; c < p.r.n_experts; c += 16 * epc) store_chunk<T, VEC>(out + c, (const T*)held + c);
}

// bias + rate where an expert has fewer rows than the mean, - rate where it has more
static __global__ void __launch_bounds__(256) k_balance_bias(const float* bias, const int32_t* offsets, int32_t n_experts, float rate, float* out) {
    const int32_t e = blockIdx.x * 256 + threadIdx.x;
    if (e >= n_experts) return;
    const int64_t off = (int64_t)offsets[n_experts] - ((int64_t)offsets[e + 1] - offsets[e]) * n_experts;
    out[e] = bias[e] + (off > 0 ? rate : off < 0 ? -rate : 0.f);
}

}  // namespace nomad_router
