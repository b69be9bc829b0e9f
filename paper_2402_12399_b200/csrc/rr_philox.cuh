// Dropout masks from a counter: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy
// as 1, 2, 3", SC 2011).  The mask of a tensor is a function of (seed, offset, flat element index) alone, so it
// is never stored: the backward pass, and any kernel with another tiling, computes the same bits again.
//   key     = seed (low word, high word)
//   counter = (i / 8 low, i / 8 high, offset low, offset high)       for element i of the tensor, row-major
// One block of four 32-bit words serves eight elements with 16 bits each: element i takes the (i % 8)-th
// 16-bit piece, low half first.  Sixteen bits instead of 32 halve the integer work, which is what a kernel
// that also moves data at the HBM rate has to hide; the drop probability is rounded to 1/65536 for it, and the
// factor of the kept elements uses the rounded probability, so the expectation is exact.
#pragma once
#include <stdint.h>

namespace rr {

struct DropoutParams {
    const unsigned long long *rng;  // dev: {seed, offset}; null without dropout
    uint32_t drop;                  // an element is dropped when its 16-bit piece is below this (0..65536)
    float factor;                   // of the kept elements: 65536 / (65536 - drop), 0 when all are dropped
};

// probability in [0, 1] -> thresholds (the caller has checked the range)
inline DropoutParams dropout_params(float p, const void *rng)
{
    DropoutParams d;
    d.drop = (uint32_t)((double)p * 65536.0 + 0.5);
    d.rng = d.drop ? static_cast<const unsigned long long *>(rng) : nullptr;
    d.factor = d.drop < 65536u ? (float)(65536.0 / (65536.0 - d.drop)) : 0.0f;
    return d;
}

struct PhiloxKey {
    uint32_t k0, k1, o0, o1;
};
__device__ __forceinline__ PhiloxKey philox_key(const unsigned long long *rng)
{
    const unsigned long long seed = rng[0], offset = rng[1];
    return {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)offset, (uint32_t)(offset >> 32)};
}

// The generator's words for G groups of eight elements, `group`, `group` + stride, ..., in lockstep: the groups share the key
// schedule and hide each other's latency.  They are set so that keep() below is false for every piece when all is dropped.
template <int G>
__device__ __forceinline__ void philox_words(const PhiloxKey &key, unsigned long long group, uint32_t drop, uint32_t (&w)[G][4],
                                             unsigned long long stride = 1)
{
    uint32_t k0 = key.k0, k1 = key.k1;
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const unsigned long long c = group + g * stride;
        w[g][0] = (uint32_t)c;
        w[g][1] = (uint32_t)(c >> 32);
        w[g][2] = key.o0;
        w[g][3] = key.o1;
    }
#pragma unroll
    for (int r = 0; r < 10; ++r) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const uint64_t p0 = (uint64_t)w[g][0] * 0xD2511F53u, p1 = (uint64_t)w[g][2] * 0xCD9E8D57u;
            w[g][0] = (uint32_t)(p1 >> 32) ^ w[g][1] ^ k0;
            w[g][2] = (uint32_t)(p0 >> 32) ^ w[g][3] ^ k1;
            w[g][1] = (uint32_t)p1;
            w[g][3] = (uint32_t)p0;
        }
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    if (drop > 65535u) {
#pragma unroll
        for (int g = 0; g < G; ++g) w[g][0] = w[g][1] = w[g][2] = w[g][3] = 0u;
    }
}
// `drop` as the bound of keep(): the pieces are compared in the upper halves of words, one comparison each
__device__ __forceinline__ uint32_t keep_bound(uint32_t drop) { return drop > 65535u ? 0xffffffffu : drop << 16; }
// is element j of the group kept?
__device__ __forceinline__ bool keep(const uint32_t (&w)[4], int j, uint32_t bound)
{
    return ((j & 1) ? w[j >> 1] : w[j >> 1] << 16) >= bound;
}

}  // namespace rr
