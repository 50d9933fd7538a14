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
// the call's own number, and the probability in 65536ths (0: no dropout) as `above`, see Kept.
struct Dropout {
    const unsigned long long* rng;
    uint32_t site, above;
    float scale;                   // 65536 / (65536 - threshold): the kept elements' factor, exactly what the rounded probability asks for
    bool on;
};
inline Dropout make_dropout(float p, const void* rng, uint32_t site) {
    const uint32_t threshold = (uint32_t)((double)p * 65536.0 + 0.5);
    Dropout d{(const unsigned long long*)rng, site, 0u, 1.f, threshold != 0};
    d.above = threshold * 65536u - 1u;                                   // (65536: 2^32 - 1, which nothing is above)
    d.scale = threshold < 65536u ? (float)(65536.0 / (65536.0 - threshold)) : 0.f;
    return d;
}

// Which of the eight neighbouring columns 8 j .. 8 j + 7 of a row are kept: one counter a group, 16 bits an element, so that the generator's ten
// rounds cost about 8 instructions an element (with 32 bits an element they would be more than the time the element's bytes take).
// Bits are kept when they are at least the threshold: placed in the upper half of a word (with anything in the lower one), when the word is above
// 65536 threshold - 1.
struct Kept {
    uint4 w;
    uint32_t above;
    __device__ __forceinline__ Kept() {}
    // group = row * ceil(width / 8) + j
    __device__ __forceinline__ Kept(const Dropout& d, uint64_t group, uint64_t seed, uint64_t step) : above(d.above) {
        w = philox4x32(make_uint4((uint32_t)group, (uint32_t)(group >> 32), (uint32_t)step, d.site), (uint32_t)seed, (uint32_t)(seed >> 32));
    }
    __device__ __forceinline__ bool operator[](int i) const {
        const uint32_t r = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w;
        return (i & 1 ? r : r << 16) > above;
    }
};

}  // namespace mpode
