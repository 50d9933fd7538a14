// Eight neighbouring elements of a row at a time, as float32: 16-byte accesses (VEC: the caller has checked alignment, and all eight exist or
// none does) or single elements, of which the first n exist.
#pragma once
#include <type_traits>

#include "common.cuh"

namespace mpode {

template <typename T> struct Pair;
template <> struct Pair<__nv_bfloat16> {
    static __device__ __forceinline__ float2 get(uint32_t w) {
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t put(float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};
template <> struct Pair<__half> {
    static __device__ __forceinline__ float2 get(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
    static __device__ __forceinline__ uint32_t put(float a, float b) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};

template <typename T, bool VEC> __device__ __forceinline__ void load8(const T* p, int n, float (&f)[8]) {
    if constexpr (VEC) {
        if (n <= 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = 0.f;
            return;
        }
        if constexpr (sizeof(T) == 4) {
            const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
            f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
            f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(p);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 t = Pair<T>::get(w[i]);
                f[2 * i] = t.x; f[2 * i + 1] = t.y;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < n ? Low<T>::to_f(p[i]) : 0.f;
    }
}

// returns whether a value that was written is not finite
template <typename T, bool VEC> __device__ __forceinline__ bool store8(T* p, int n, const float (&f)[8]) {
    bool bad = false;
    if constexpr (VEC) {
        if (n <= 0) return false;
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
            reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
#pragma unroll
            for (int i = 0; i < 8; ++i) bad |= Low<float>::nonfinite(f[i]);
        } else {
            uint32_t w[4];
            const uint32_t lo = sizeof(T) == 2 && std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u, hi = lo << 16;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = Pair<T>::put(f[2 * i], f[2 * i + 1]);
                bad |= (w[i] & lo) == lo || (w[i] & hi) == hi;
            }
            *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) {
                const T t = Low<T>::from_f(f[i]);
                bad |= Low<T>::nonfinite(t);
                p[i] = t;
            }
    }
    return bad;
}

}  // namespace mpode
