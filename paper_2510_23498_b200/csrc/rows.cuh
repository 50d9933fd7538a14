// Eight neighbouring elements of a row at a time: as they lie in memory (Raw8), and as four pairs of float32 (Oct), on which one instruction works on two.
#pragma once
#include <type_traits>

#include "common.cuh"

namespace mpode {

template <typename T> struct Pair;
template <> struct Pair<__nv_bfloat16> {
    static __device__ __forceinline__ float2 get(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
    static __device__ __forceinline__ uint32_t put(float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static constexpr uint32_t infinity = 0x7F80u;
};
template <> struct Pair<__half> {
    static __device__ __forceinline__ float2 get(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
    static __device__ __forceinline__ uint32_t put(float a, float b) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static constexpr uint32_t infinity = 0x7C00u;
};

struct Oct {
    float2 v[4];
    __device__ __forceinline__ void fill(float f) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = make_float2(f, f);
    }
};

// VEC: 16-byte accesses, for which the caller has checked alignment, and all eight elements exist or none does; else single elements of which the first n
// exist.  Elements that do not exist read as zero.
template <typename T> struct Raw8 { uint32_t w[sizeof(T) * 2]; };
template <typename T, bool VEC> __device__ __forceinline__ void load_raw(const T* p, int n, Raw8<T>& r) {
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) * 2; ++j) r.w[j] = 0u;
    if constexpr (VEC) {
        if (n <= 0) return;
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j) {
            const uint4 a = reinterpret_cast<const uint4*>(p)[j];
            r.w[4 * j] = a.x; r.w[4 * j + 1] = a.y; r.w[4 * j + 2] = a.z; r.w[4 * j + 3] = a.w;
        }
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) r.w[i] = __float_as_uint(p[i]);
    } else {
        const uint16_t* const h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) r.w[i / 2] |= (uint32_t)h[i] << (16 * (i & 1));
    }
}
template <typename T> __device__ __forceinline__ void unpack(const Raw8<T>& r, Oct& o) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) o.v[j] = make_float2(__uint_as_float(r.w[2 * j]), __uint_as_float(r.w[2 * j + 1]));
        else o.v[j] = Pair<T>::get(r.w[j]);
    }
}
template <typename T> __device__ __forceinline__ void pack(const Oct& o, Raw8<T>& r) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) { r.w[2 * j] = __float_as_uint(o.v[j].x); r.w[2 * j + 1] = __float_as_uint(o.v[j].y); }
        else r.w[j] = Pair<T>::put(o.v[j].x, o.v[j].y);
    }
}
template <typename T, bool VEC> __device__ __forceinline__ void load8(const T* p, int n, Oct& o) {
    Raw8<T> r;
    load_raw<T, VEC>(p, n, r);
    unpack<T>(r, o);
}
template <typename T, bool VEC> __device__ __forceinline__ void store_raw(T* p, int n, const Raw8<T>& r) {
    if constexpr (VEC) {
        if (n <= 0) return;
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j) reinterpret_cast<uint4*>(p)[j] = make_uint4(r.w[4 * j], r.w[4 * j + 1], r.w[4 * j + 2], r.w[4 * j + 3]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = __uint_as_float(r.w[i]);
    } else {
        uint16_t* const h = reinterpret_cast<uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) h[i] = (uint16_t)(r.w[i / 2] >> (16 * (i & 1)));
    }
}

// Four neighbouring elements (a half of the above): as pairs of float32, and their accesses
struct Quad { float2 v[2]; };
template <typename T, bool VEC> __device__ __forceinline__ Quad load4(const T* p, int n) {
    Quad q;
    if constexpr (VEC) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = *reinterpret_cast<const float4*>(p);
            q.v[0] = make_float2(a.x, a.y); q.v[1] = make_float2(a.z, a.w);
        } else {
            const uint2 a = *reinterpret_cast<const uint2*>(p);
            q.v[0] = Pair<T>::get(a.x); q.v[1] = Pair<T>::get(a.y);
        }
    } else {
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = i < n ? Low<T>::to_f(p[i]) : 0.f;
        q.v[0] = make_float2(f[0], f[1]); q.v[1] = make_float2(f[2], f[3]);
    }
    return q;
}
template <typename T, bool VEC> __device__ __forceinline__ void store4(T* p, int n, const Quad& q) {
    if constexpr (VEC) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = make_float4(q.v[0].x, q.v[0].y, q.v[1].x, q.v[1].y);
        else *reinterpret_cast<uint2*>(p) = make_uint2(Pair<T>::put(q.v[0].x, q.v[0].y), Pair<T>::put(q.v[1].x, q.v[1].y));
    } else {
        const float f[4] = {q.v[0].x, q.v[0].y, q.v[1].x, q.v[1].y};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = Low<T>::from_f(f[i]);
    }
}

// Largest magnitude of the low-format values seen, as bits (infinities and NaN above every number): two instructions a word
template <typename T> struct Largest {
    uint32_t m = 0;
    __device__ __forceinline__ void see(uint32_t w) {
        if constexpr (sizeof(T) == 4) m = max(m, w & 0x7fffffffu);
        else m = __vmaxu2(m, w & 0x7fff7fffu);
    }
    __device__ __forceinline__ void see(const Raw8<T>& r, int n) {
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) * 2; ++j)
            if (j * 4 < n * (int)sizeof(T)) {
                const bool half = sizeof(T) == 2 && j * 2 + 1 == n;          // an odd row's last word holds one element
                see(half ? r.w[j] & 0xffffu : r.w[j]);
            }
    }
    // of four elements as they are stored
    __device__ __forceinline__ void see(const Quad& q, int n) {
        if constexpr (sizeof(T) == 4) {
            const float f[4] = {q.v[0].x, q.v[0].y, q.v[1].x, q.v[1].y};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) see(__float_as_uint(f[i]));
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t w = Pair<T>::put(q.v[i].x, q.v[i].y);
                if (2 * i < n) see(2 * i + 1 < n ? w : w & 0xffffu);
            }
        }
    }
    __device__ __forceinline__ bool nonfinite() const {
        if constexpr (sizeof(T) == 4) return m >= 0x7f800000u;
        else return (m & 0xffffu) >= Pair<T>::infinity || (m >> 16) >= Pair<T>::infinity;
    }
};

}  // namespace mpode
