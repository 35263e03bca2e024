// Dropout masks from a counter-based generator: what is kept is computed where it is needed and never stored.
//
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) maps a 64-bit key
// and a 128-bit counter to 128 random bits.  The key is the step's seed, read from device memory, so that a captured
// graph draws new masks when the caller changes it.  The counter's upper half tells the places of one step apart, its
// lower half is the number of a vector of eight neighbouring columns, each of which takes 16 of the bits.
//
// 16 bits per element make the drop rate a multiple of 2^-16; kept values are scaled by the reciprocal of the actual
// keep rate, so the expectation is right whatever p was rounded to.  (32 bits per element would double the
// generator's cost, which already is what bounds bf16: 16384 x 4096 55 us instead of the 41 that its bytes take.)
#pragma once

#include <stdint.h>

#include "adasum_operators.cuh"

namespace adasum {

struct Dropout {
    const uint64_t* seed;      // device; nullptr: nothing is dropped
    uint64_t site;
    uint32_t threshold;        // of 65536: bits below it drop an element (65536 drops all)
    float factor;              // of kept elements
};

// p = 0 needs no seed.
inline adasum_status_t plan_dropout(float p, const void* seed, uint64_t site, Dropout* d)
{
    if (!(p >= 0.0f && p <= 1.0f))
        return fail(ADASUM_ERR_ARG, "drop probability %g is not between 0 and 1", (double)p);
    d->threshold = (uint32_t)(p * 65536.0f + 0.5f);
    d->factor = d->threshold < 65536 ? (float)(65536.0 / (65536.0 - d->threshold)) : 0.0f;
    d->site = site;
    d->seed = nullptr;
    if (d->threshold == 0)
        return ADASUM_OK;
    if (!seed)
        return fail(ADASUM_ERR_NULL, "seed is NULL");
    if (!aligned_to(seed, 8))
        return fail(ADASUM_ERR_ARG, "seed is not 8-byte aligned");
    d->seed = static_cast<const uint64_t*>(seed);
    return ADASUM_OK;
}

// The random bits of N vectors, `word` j holding those of columns 2 j (low half) and 2 j + 1.
template <int N>
__device__ __forceinline__ void random_words(const Dropout& d, uint64_t seed, const uint64_t (&vector)[N], uint32_t (&word)[N][4])
{
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        word[n][0] = (uint32_t)vector[n];
        word[n][1] = (uint32_t)(vector[n] >> 32);
        word[n][2] = (uint32_t)d.site;
        word[n][3] = (uint32_t)(d.site >> 32);
    }
#pragma unroll
    for (int round = 0; round < 10; ++round) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint64_t a = (uint64_t)word[n][0] * 0xD2511F53u, b = (uint64_t)word[n][2] * 0xCD9E8D57u;
            word[n][0] = (uint32_t)(b >> 32) ^ word[n][1] ^ k0;
            word[n][2] = (uint32_t)(a >> 32) ^ word[n][3] ^ k1;
            word[n][1] = (uint32_t)b;
            word[n][3] = (uint32_t)a;
        }
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

// x of a vector with its dropped elements replaced by zero (whatever they hold) and the others scaled.  16 bits are
// compared as the upper half of a word; what the lower half holds makes no difference.
__device__ __forceinline__ void drop(const Dropout& d, const uint32_t (&word)[4], float (&x)[8])
{
    const uint32_t limit = d.threshold << 16;
    if (d.threshold >= 65536u) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = 0.0f;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = i & 1 ? word[i / 2] : word[i / 2] << 16;
        x[i] = bits >= limit ? x[i] * d.factor : 0.0f;
    }
}

}  // namespace adasum
