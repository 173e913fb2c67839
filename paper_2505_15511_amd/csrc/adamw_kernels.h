// AdamW over many tensors in one launch (gfx950), states in float32 or in 8 bits.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = (1 - lr wd) p - (lr / c1) m / (sqrt(v) / sqrt(c2) + eps)
//
// One pass over the elements, eight neighbouring ones a lane: bound by their bytes (28 an element in float32, 10 with 16-bit
// parameters and 8-bit states), and with 8-bit states nearly as much by the arithmetic of decoding and encoding.  97 M elements, one step after
// the other: in bfloat16 with 8-bit states 232 us, 4.2 TB/s of the 5.4 of a large copy; float32 287 (5.4 TB/s); 32-bit states 512 and, in
// bfloat16, 408 (5.3 and 5.2).
//
// 8 bits: blocks of 256 elements (the 32 lanes of half a wavefront) have one float32 scale s, their largest magnitude.
// m = s (c / 127) |c / 127| and v = s (c / 255)^4: codes are denser near zero, where most of a block's averages are (v spans
// 2.4e-10 of its block's largest; a linear code would round the small ones to zero and their steps to m / eps).  A code is the
// whole number c with (c - 1/2)^2 <= t < (c + 1/2)^2 for t = |m| (127^2 / s), to the fourth power for v with t = v (255^4 / s), for
// any scale of at least 2^-126 (small ones are multiplied by a power of two first, which changes no t);
// v's is 0 only where v is.  The averages round every operation once, without fused ones, and borders are compared in float32: the
// codes are the same whatever computes them.  The step's root and quotient are rounded correctly; only where parameters of 16 bits have
// states of 8 the hardware's root and reciprocal stand in (one unit in the last place each, 2^-15 and less of what the parameter's own
// rounding is; 97 M elements 232 us, 272 with the others, which cost nothing where more bytes move), and not for denormal numbers,
// which that root takes for zero.
//
// Nearest codes hold an average where it is as long as a step changes it by less than half the way to the next code: v falls only
// with its block's largest where 1 - beta2 is below 0.8 % (c = 255; more below), and rises on gradients far above its own.  Dithered
// codes are right on average instead: the border between c and c + 1 lies at c^2 + u ((c + 1)^2 - c^2) (fourth powers for v), u drawn
// evenly from (0, 1) for every element and step, so that the value that a code stands for is the average in expectation, and so are all
// that follow from it.  u: 16 bits of Philox(counter = (element / 8, 0 for m or 1 for v), key = step); nothing is kept for it.  97 M elements
// in bfloat16 252 us against 232 with nearest codes, in float32 318 against 287.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "philox.h"

namespace nomad_adamw {

constexpr int kTensors = 64;              // a launch: their addresses are its arguments (under 4 KB)
constexpr int kThreads = 256, kPer = 8;   // lanes a workgroup, elements a lane
constexpr int kChunk = kThreads * kPer;   // elements a workgroup takes (four times as many: 97 M elements with 8-bit states and the averages read
                                          // back 377 us, 370 so; with 32-bit states 522 and 509)
constexpr int kBlock = 256;               // elements a scale
constexpr int kLanes = kBlock / kPer;

struct Tensor {
    void* p;
    const void* g;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    int64_t n;
};
struct Scalars {
    float keep, rate, b1, c1, b2, c2, root, eps;
    uint32_t step_low, step_high;
    const float* grad_scale;   // NULL: 1
};
struct Batch {
    Tensor t[kTensors];
    uint32_t first[kTensors + 1];   // workgroup of each tensor
    int32_t count;
    Scalars s;
};

template <typename T, bool WHOLE>
__device__ __forceinline__ void load8(const T* from, int n, T (&v)[kPer]) {
    struct alignas(sizeof(T) * 4 < 16 ? sizeof(T) * kPer : 16) Part { T v[kPer]; };
    if (WHOLE) {
        *(Part*)v = *(const Part*)from;
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = i < n ? from[i] : (T)0;
    }
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void store8(T* to, int n, const T (&v)[kPer]) {
    struct alignas(sizeof(T) * 4 < 16 ? sizeof(T) * kPer : 16) Part { T v[kPer]; };
    if (WHOLE) {
        *(Part*)to = *(const Part*)v;
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (i < n) to[i] = v[i];
    }
}

// scales below kSmall are lifted by kLift: 255^4 / kSmall is finite, and a lifted scale is a normal number far from either end
constexpr float kSmall = 0x1p-90f, kLift = 0x1p64f;

__device__ __forceinline__ float decode_first(int c, float s) {
#pragma clang fp contract(off)
    const float t = (float)c * (1.f / 127.f);
    return (t * fabsf(t)) * s;
}
__device__ __forceinline__ float decode_second(uint32_t c, float s) {
#pragma clang fp contract(off)
    float t = (float)c * (1.f / 255.f);
    t = t * t;
    return (t * t) * s;
}
// largest magnitude of the block's 32 lanes, as bits: a NaN is larger than every number
__device__ __forceinline__ uint32_t block_most(uint32_t bits) {
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)bits, d);
        bits = o > bits ? o : bits;
    }
    return bits;
}
// (a NaN or an infinity makes the scale NaN, and so the block's values: they do not disappear)
__device__ __forceinline__ float scale_of(uint32_t bits) {
    return bits < 0x00800000u ? 0.f : __uint_as_float(bits < 0x7f800000u ? bits : 0x7fc00000u);
}
// Roots by the hardware, whose last place may be off by one: `off` collects how far they lie from their whole numbers, and where none
// is nearer to a border than that error reaches (kSure: 128 2^-23, and one and a half times that of 255 for the fourth root
// and 2^-26 for its border), the whole numbers are the codes.  Otherwise, for one wavefront in nine, borders are compared.
// (fmaxf makes a NaN, whose scale is one already, 0.)
constexpr float kSureFirst = 0.49997f, kSureSecond = 0.49992f;
__device__ __forceinline__ float root_first(float m, float factor, float& off) {
#pragma clang fp contract(off)
    const float r = __builtin_amdgcn_sqrtf(fabsf(m) * factor), c = rintf(r);
    off = fmaxf(off, fabsf(r - c));
    return fmaxf(c, 0.f);
}
__device__ __forceinline__ float root_second(float v, float factor, float& off) {
#pragma clang fp contract(off)
    const float r = __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(v * factor)), c = rintf(r);
    off = fmaxf(off, fabsf(r - c));
    return fmaxf(c, 0.f);
}
// the code of |m| factor = t from a whole number that is one off at most (c = 0 has no lower border)
__device__ __forceinline__ float border_first(float c, float m, float factor) {
#pragma clang fp contract(off)
    const float t = fabsf(m) * factor, up = c + 0.5f, down = fmaxf(c - 0.5f, 0.f);
    return c + (t >= up * up ? 1.f : 0.f) - (t < down * down ? 1.f : 0.f);
}
__device__ __forceinline__ float border_second(float c, float v, float factor) {
#pragma clang fp contract(off)
    const float t = v * factor;
    float up = c + 0.5f, down = fmaxf(c - 0.5f, 0.f);
    up = up * up;
    down = down * down;
    return c + (t >= up * up ? 1.f : 0.f) - (t < down * down ? 1.f : 0.f);
}

constexpr float kRootNormal = 0x1p-96f;   // far enough above the smallest normal number
// eight numbers of (0, 1), 16 bits each, for elements at .. at + 7
__device__ __forceinline__ void draw8(int64_t at, uint32_t which, const Scalars& s, float (&u)[kPer]) {
    uint32_t words[4];
    const uint64_t eighth = (uint64_t)at / kPer;
    philox4x32_10((uint32_t)eighth, (uint32_t)(eighth >> 32), which, 0u, s.step_low, s.step_high, words);
#pragma unroll
    for (int i = 0; i < kPer; ++i) u[i] = ((float)(words[i / 2] >> i % 2 * 16 & 0xffffu) + 0.5f) * 0x1p-16f;
}
// (a t within a rounding of a whole number's power may have that number or the one below for c: the border is next to it either way.
// fminf makes a NaN, whose scale is one, the largest code)
__device__ __forceinline__ float drawn_first(float m, float factor, float u) {
    const float t = fabsf(m) * factor, c = fminf(floorf(__builtin_amdgcn_sqrtf(t)), 127.f);
    return fminf(c + (t >= c * c + u * (2.f * c + 1.f) ? 1.f : 0.f), 127.f);
}
__device__ __forceinline__ float drawn_second(float v, float factor, float u) {
    const float t = v * factor, c = fminf(floorf(__builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(t))), 255.f);
    float low = c * c, up = (c + 1.f) * (c + 1.f);
    low = low * low;
    up = up * up;
    return fminf(c + (t >= low + u * (up - low) ? 1.f : 0.f), 255.f);
}

template <typename P, typename G, bool EIGHT, bool DITHER, bool WHOLE>
__device__ __forceinline__ void step8(const Tensor& t, const Scalars& s, int64_t at, int n) {
#pragma clang fp contract(off)
    P p[kPer];
    G g[kPer];
    float m[kPer], v[kPer];
    load8<P, WHOLE>((const P*)t.p + at, n, p);
    load8<G, WHOLE>((const G*)t.g + at, n, g);
    if (EIGHT) {
        int8_t mc[kPer];
        uint8_t vc[kPer];
        load8<int8_t, WHOLE>((const int8_t*)t.m + at, n, mc);
        load8<uint8_t, WHOLE>((const uint8_t*)t.v + at, n, vc);
        float ms = 0.f, vs = 0.f;
        if (n > 0) { ms = t.m_scale[at / kBlock]; vs = t.v_scale[at / kBlock]; }
#pragma unroll
        for (int i = 0; i < kPer; ++i) { m[i] = decode_first(mc[i], ms); v[i] = decode_second(vc[i], vs); }
    } else {
        load8<float, WHOLE>((const float*)t.m + at, n, m);
        load8<float, WHOLE>((const float*)t.v + at, n, v);
    }
    const float scale = s.grad_scale ? *s.grad_scale : 1.f;
    float least = __builtin_inff();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const float d = (float)g[i] * scale;
        m[i] = m[i] * s.b1 + d * s.c1;
        v[i] = v[i] * s.b2 + (d * d) * s.c2;
        least = fminf(least, v[i]);
    }
    if (!EIGHT || sizeof(P) == 4 || __any(least < kRootNormal)) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) p[i] = (P)((float)p[i] * s.keep - (m[i] * s.rate) / (sqrtf(v[i]) * s.root + s.eps));
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            p[i] = (P)((float)p[i] * s.keep - (m[i] * s.rate) * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[i]) * s.root + s.eps));
    }
    store8<P, WHOLE>((P*)t.p + at, n, p);
    if (EIGHT) {
        uint32_t m_most = 0, v_most = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint32_t mb = i < n ? __float_as_uint(m[i]) & 0x7fffffffu : 0u, vb = i < n ? __float_as_uint(v[i]) & 0x7fffffffu : 0u;
            m_most = mb > m_most ? mb : m_most;
            v_most = vb > v_most ? vb : v_most;
        }
        const float ms = scale_of(block_most(m_most)), vs = scale_of(block_most(v_most));
        // 127^2 / s and 255^4 / s have to be numbers: small averages and their scale are first multiplied by the same power of two
        const float m_lift = ms < kSmall ? kLift : 1.f, v_lift = vs < kSmall ? kLift : 1.f;
        const float mf = ms == 0.f ? 0.f : 16129.f / (ms * m_lift), vf = vs == 0.f ? 0.f : 4228250625.f / (vs * v_lift);
        if (__any(m_lift != 1.f || v_lift != 1.f))
#pragma unroll
            for (int i = 0; i < kPer; ++i) { m[i] *= m_lift; v[i] *= v_lift; }
        float mr[kPer], vr[kPer];
        if (DITHER) {
            float u[kPer];
            draw8(at, 0u, s, u);
#pragma unroll
            for (int i = 0; i < kPer; ++i) mr[i] = drawn_first(m[i], mf, u[i]);
            draw8(at, 1u, s, u);
#pragma unroll
            for (int i = 0; i < kPer; ++i) vr[i] = drawn_second(v[i], vf, u[i]);
        } else {
            float off_first = 0.f, off_second = 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) { mr[i] = root_first(m[i], mf, off_first); vr[i] = root_second(v[i], vf, off_second); }
            if (__any(off_first > kSureFirst || off_second > kSureSecond))
#pragma unroll
                for (int i = 0; i < kPer; ++i) { mr[i] = border_first(mr[i], m[i], mf); vr[i] = border_second(vr[i], v[i], vf); }
        }
        const float least = vs > 0.f ? 0.f : __builtin_inff();   // what v is above where its code is at least 1
        int8_t mc[kPer];
        uint8_t vc[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            mc[i] = (int8_t)(int)copysignf(mr[i], m[i]);
            vc[i] = (uint8_t)(uint32_t)fmaxf(vr[i], v[i] > least ? 1.f : 0.f);
        }
        store8<int8_t, WHOLE>((int8_t*)t.m + at, n, mc);
        store8<uint8_t, WHOLE>((uint8_t*)t.v + at, n, vc);
        if (n > 0 && at % kBlock == 0) { t.m_scale[at / kBlock] = ms; t.v_scale[at / kBlock] = vs; }
    } else {
        store8<float, WHOLE>((float*)t.m + at, n, m);
        store8<float, WHOLE>((float*)t.v + at, n, v);
    }
}

__device__ __forceinline__ bool aligned(const void* p, uintptr_t bytes) { return (uintptr_t)p % bytes == 0; }

template <typename P, typename G, bool EIGHT, bool DITHER>
__global__ void __launch_bounds__(kThreads) k_adamw(Batch b) {
    int lo = 0, hi = b.count;   // the tensor of this workgroup
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (b.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid;
    }
    const Tensor t = b.t[lo];
    const bool borders = aligned(t.p, sizeof(P) * 4 < 16 ? sizeof(P) * kPer : 16) && aligned(t.g, sizeof(G) * 4 < 16 ? sizeof(G) * kPer : 16) &&
                         aligned(t.m, EIGHT ? 8 : 16) && aligned(t.v, EIGHT ? 8 : 16);
    const int64_t first = (int64_t)(blockIdx.x - b.first[lo]) * kChunk, at = first + (int64_t)threadIdx.x * kPer;
    if (borders && first + kChunk <= t.n) step8<P, G, EIGHT, DITHER, true>(t, b.s, at, kPer);
    else step8<P, G, EIGHT, DITHER, false>(t, b.s, at, (int)(t.n - at > kPer ? kPer : t.n - at));   // (every lane stays: the block's largest is found by all)
}

// 8-bit states as the values they stand for
struct ValuesBatch {
    struct { const void* codes; const float* scale; float* out; int64_t n; } t[kTensors];
    uint32_t first[kTensors + 1];
    int32_t count;
};
template <bool SECOND>
__global__ void __launch_bounds__(kThreads) k_adamw_values(ValuesBatch b) {
    int lo = 0, hi = b.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (b.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid;
    }
    const auto t = b.t[lo];
    const int64_t first = (int64_t)(blockIdx.x - b.first[lo]) * kChunk;
#pragma unroll
    for (int part = 0; part < kPer / 4; ++part) {   // four elements a lane at a time: a wavefront's stores are one run
        const int64_t at = first + part * (kThreads * 4) + threadIdx.x * 4;
        if (at >= t.n) return;
        const float s = t.scale[at / kBlock];
        const bool whole = at + 4 <= t.n && aligned(t.codes, 4) && aligned(t.out, 16);
        uint8_t c[4] = {};
        if (whole) *(uint32_t*)c = *(const uint32_t*)((const uint8_t*)t.codes + at);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (at + i < t.n) c[i] = ((const uint8_t*)t.codes)[at + i];
        float4 v;
        float* x = (float*)&v;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = SECOND ? decode_second(c[i], s) : decode_first((int8_t)c[i], s);
        if (whole) *(float4*)(t.out + at) = v;
        else
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (at + i < t.n) t.out[at + i] = x[i];
    }
}

}  // namespace nomad_adamw
