// Counter-based random bits: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011).
#pragma once
#include <stdint.h>

namespace mpode {

__device__ __forceinline__ uint4 philox4x32(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p = (uint64_t)c.x * 0xD2511F53u, q = (uint64_t)c.z * 0xCD9E8D57u;
        c = make_uint4((uint32_t)(q >> 32) ^ c.y ^ k0, (uint32_t)q, (uint32_t)(p >> 32) ^ c.w ^ k1, (uint32_t)p);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}

// What a launch's dropout is made of: the caller's two words {seed, step} in device memory (a captured graph reads them again at every replay),
// the call's own number, and the probability in 65536ths (0: no dropout).
struct Dropout {
    const unsigned long long* rng;
    uint32_t site, threshold;
    float scale;                   // 65536 / (65536 - threshold): the kept elements' factor, exactly what the rounded probability asks for
};
inline Dropout make_dropout(float p, const void* rng, uint32_t site) {
    Dropout d{(const unsigned long long*)rng, site, 0u, 1.f};
    d.threshold = (uint32_t)((double)p * 65536.0 + 0.5);
    d.scale = d.threshold < 65536u ? (float)(65536.0 / (65536.0 - d.threshold)) : 0.f;
    return d;
}

// The masks of eight neighbouring columns 8 j .. 8 j + 7 of a row, bit i set where column 8 j + i is kept: one counter a group, 16 bits an
// element, so that the generator's ten rounds cost about 13 instructions an element (32 bits an element would be twice that and more than the
// time the element's bytes take).  group = row * ceil(width / 8) + j.
__device__ __forceinline__ uint32_t keep_bits(uint64_t group, uint64_t seed, uint64_t step, uint32_t site, uint32_t threshold) {
    const uint4 w = philox4x32(make_uint4((uint32_t)group, (uint32_t)(group >> 32), (uint32_t)step, site), (uint32_t)seed, (uint32_t)(seed >> 32));
    const uint32_t r[4] = {w.x, w.y, w.z, w.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m |= ((r[i] & 0xffffu) >= threshold ? 1u : 0u) << (2 * i);
        m |= ((r[i] >> 16) >= threshold ? 1u : 0u) << (2 * i + 1);
    }
    return m;
}

}  // namespace mpode
