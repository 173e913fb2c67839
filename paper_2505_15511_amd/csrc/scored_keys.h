// libnomad: what a lane keeps of its experts' keys while a row's best are chosen, plain C++ (the kernels use it on the device, a test compiles it with
// the host compiler).  A key is never 0, and those of different experts differ.
#pragma once
#include <stdint.h>

#if defined(__HIP__)
#define NOMAD_LANE __device__ __forceinline__
#else
#define NOMAD_LANE inline
#endif

namespace nomad_router {

NOMAD_LANE void order(uint32_t& a, uint32_t& b) {   // the larger first
    const uint32_t m = a > b ? a : b;
    b = a > b ? b : a;
    a = m;
}
template <int N>
NOMAD_LANE void bitonic(uint32_t (&v)[N]) {   // a sequence that rises and falls -> descending
#pragma unroll
    for (int d = N / 2; d > 0; d /= 2)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if ((i & d) == 0) order(v[i], v[i + d]);
}
template <int N>
NOMAD_LANE void sorted(uint32_t (&v)[N]) {   // descending
#pragma unroll
    for (int size = 2; size <= N; size *= 2)
#pragma unroll
        for (int d = size / 2; d > 0; d /= 2)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if ((i & d) == 0) {
                    if ((i & size) == 0) order(v[i], v[i + d]);
                    else order(v[i + d], v[i]);
                }
}
// the L largest of N, descending; returns the largest of the others (0: there are none)
template <int L, int N>
NOMAD_LANE uint32_t largest(const uint32_t (&v)[N], uint32_t (&out)[L]) {
    uint32_t gone = 0u;
#pragma unroll
    for (int i = 0; i < L; ++i) out[i] = i < N ? v[i] : 0u;
    sorted(out);
#pragma unroll
    for (int at = L; at < N; at += L) {
        uint32_t more[L];
#pragma unroll
        for (int i = 0; i < L; ++i) more[i] = at + i < N ? v[at + i] : 0u;
        sorted(more);
#pragma unroll
        for (int i = 0; i < L; ++i) {
            uint32_t less = more[L - 1 - i];
            order(out[i], less);
            gone = less > gone ? less : gone;
        }
        bitonic(out);
    }
    return gone;
}

// The keys that a lane of CAP experts has kept, while up to K of the row are given away, best first.  A lane does not run out of them while it has
// others: whatever it let go is below the last key given
template <int CAP, int K>
struct Kept {
    static constexpr int kList = K == 2 ? 4 : 8;
    uint32_t list[kList];                          // descending; 0: no key
    uint32_t gone;                                 // the largest that found no place in it; 0: all did

    NOMAD_LANE void keep(const uint32_t (&key)[CAP], bool open) {
        gone = largest(key, list);
        gone = open ? gone : 0u;
#pragma unroll
        for (int i = 0; i < kList; ++i) list[i] = open ? list[i] : 0u;
    }
    // the row's best key leaves the lane that has it
    NOMAD_LANE void give(uint32_t best) {
        if (list[0] != best) return;
#pragma unroll
        for (int i = 0; i + 1 < kList; ++i) list[i] = list[i + 1];
        list[kList - 1] = 0u;
    }
    // Whether the lane has an expert that may be better than the last one given (0: fewer were given than asked for): one whose key is within `apart` steps, of 2^bits
    // each, of the last one's, unless same(last, its key).  Of those that it let go it knows the largest alone: that near, it may be any of them
    template <typename F>
    NOMAD_LANE bool unsure(uint32_t last, uint32_t apart, int bits, F same) const {
        if (last == 0) return false;
        const auto close = [&](uint32_t key) { return key != 0 && (last >> bits) - (key >> bits) <= apart; };
        bool may = close(gone);
        if (close(list[0]))
#pragma unroll
            for (int i = 0; i < kList; ++i)
                if (close(list[i]) && !same(last, list[i])) may = true;
        return may;
    }
};

}  // namespace nomad_router
