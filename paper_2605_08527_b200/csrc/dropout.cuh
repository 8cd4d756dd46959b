// Masks of the adapters' dropout: 16 random bits per element from a counter-based generator, so that every kernel that needs an
// element's mask computes it anew and none is stored.  Philox-4x32 of seven rounds (Salmon, Moraes, Dror and Shaw, "Parallel
// random numbers: as easy as 1, 2, 3", 2011, who name seven as the fewest that pass their tests) on the counter
// (column / 8, token, offset) under the seed gives 128 bits: eight columns of a token.
#pragma once

#include "internal.cuh"

namespace marlaas {

__device__ __forceinline__ uint4 drop_bits(const DropKey& k, uint32_t vec, uint32_t token) {
    uint32_t c0 = vec, c1 = token, c2 = k.o0, c3 = k.o1, k0 = k.k0, k1 = k.k1;
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// Of 65536 numbers, how many drop an element at rate p: none for a rate that is not above 0, or a NaN.
__device__ __forceinline__ uint32_t drop_limit(float p) { return p > 0.f ? (uint32_t)rintf(fminf(p, 1.f) * 65536.f) : 0u; }
// s / (1 - p), of the rate as it is rounded; 0 where everything is dropped.
__device__ __forceinline__ float drop_scale(float s, uint32_t limit) { return limit < 65536u ? s * (65536.f / (float)(65536u - limit)) : 0.f; }

// Eight bf16 elements with the dropped ones (16 bits below `limit`) set to 0, whatever they hold.  The comparisons are made in the
// upper halves of 32-bit words, where the lower halves' bits cannot matter.
__device__ __forceinline__ uint4 drop_apply(uint4 x, const uint4& bits, uint32_t limit) {
    if (limit >= 65536u) return make_uint4(0u, 0u, 0u, 0u);
    const uint32_t l = limit << 16;
    uint32_t* v = &x.x;
    const uint32_t* b = &bits.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((b[i] << 16) < l) v[i] &= 0xffff0000u;
        if (b[i] < l) v[i] &= 0x0000ffffu;
    }
    return x;
}

// Threads more in a shrink kernel whose streamed rows are masked in shared memory: four warps, beside the four that also write its
// results.
constexpr int DROP_EXTRA_THREADS = 128;

}  // namespace marlaas
