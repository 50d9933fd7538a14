// Backward pass of the residual step: adjoint, cotangents and the weights' gradients of a row in one pass.
#include "residual.cuh"

namespace mpode {
namespace {

// A thread's own pieces of the rows y', dy', dz, u and gate (0 .. 4).  VEC: copied to shared memory by asynchronous copies some rows ahead; a thread reads
// what it has copied itself, so that nothing has to be waited for but its own copies.  Else loaded into registers when the row starts.
template <typename T, bool VEC, int threads> struct Rows;
template <typename T, int threads> struct Rows<T, true, threads> {
    static constexpr int kStages = sizeof(T) == 4 ? 2 : 3, kLow = sizeof(T) / 2, kPieces = 4 + 3 * kLow;
    uint4* at;
    __device__ __forceinline__ void bind(char* smem, int n) {
        at = reinterpret_cast<uint4*>(smem) + threadIdx.x;
        if (n <= 0)                                         // columns that do not exist are zero
            for (int i = 0; i < kStages * kPieces; ++i) at[i * threads] = make_uint4(0u, 0u, 0u, 0u);
    }
    static __device__ __forceinline__ constexpr int first(int k) { return k < 2 ? 2 * k : 4 + (k - 2) * kLow; }
    template <typename E> __device__ __forceinline__ void request(int stage, int k, const E* from, int n) {
        if (n <= 0) return;
#pragma unroll
        for (int j = 0; j < (int)sizeof(E) / 2; ++j)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_of(at + (stage * kPieces + first(k) + j) * threads)), "l"(reinterpret_cast<const uint4*>(from) + j) : "memory");
    }
    __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory"); }
    template <typename E> __device__ __forceinline__ void raw(int stage, int k, Raw8<E>& r) const {
#pragma unroll
        for (int j = 0; j < (int)sizeof(E) / 2; ++j) {
            const uint4 v = at[(stage * kPieces + first(k) + j) * threads];
            r.w[4 * j] = v.x; r.w[4 * j + 1] = v.y; r.w[4 * j + 2] = v.z; r.w[4 * j + 3] = v.w;
        }
    }
    __device__ __forceinline__ void get(int stage, int k, Oct& o) const {
        if (k < 2) {
            Raw8<float> r;
            raw<float>(stage, k, r);
            unpack<float>(r, o);
        } else {
            Raw8<T> r;
            raw<T>(stage, k, r);
            unpack<T>(r, o);
        }
    }
};
template <typename T, int threads> struct Rows<T, false, threads> {
    static constexpr int kStages = 1;
    Raw8<float> wide[2];
    Raw8<T> low[3];
    __device__ __forceinline__ void bind(char*, int) {}
    template <typename E> __device__ __forceinline__ void request(int, int k, const E* from, int n) {
        if constexpr (std::is_same<E, T>::value && !std::is_same<T, float>::value) load_raw<T, false>(from, n, low[k - 2]);
        else if (k < 2) load_raw<float, false>((const float*)from, n, wide[k]);
        else load_raw<T, false>((const T*)from, n, low[k - 2]);
    }
    __device__ __forceinline__ void commit() {}
    __device__ __forceinline__ void wait() {}
    __device__ __forceinline__ void raw(int, int k, Raw8<T>& r) const { r = low[k - 2]; }
    __device__ __forceinline__ void get(int, int k, Oct& o) const {
        if (k < 2) unpack<float>(wide[k], o);
        else unpack<T>(low[k - 2], o);
    }
};

// With n' the normalised y', n that of u, and t the cotangent of the step's term:
//   a = dy' + r' (w dz - n' mean(w dz n') - mean(w dz)),  dw_pre += dz n';   t = drop(a), dscale += h t v sig, with v = w_post n;
//   t <- h scale t, dgate = t v sig', t <- t sig, dw_post += t n, du = r (w t - n mean(w t n) - mean(w t)); the means of w dz and w t only for MEANVAR
template <typename T, bool VEC, bool CENTER, int WARPS, bool CLUSTER>
__global__ void __launch_bounds__(Lane<WARPS, CLUSTER>::kThreads, WARPS == 16 ? 1 : 512 / Lane<WARPS, CLUSTER>::kThreads) residual_backward_kernel(const ResArgs p, const int blocks) {
    constexpr int N = CENTER ? 2 : 1;
    using Sum = RowSum<N, WARPS, CLUSTER>;
    extern __shared__ __align__(16) char staged[];
    __shared__ typename Sum::Shared shared;
    const Lane<WARPS, CLUSTER> q(p.width, blocks);
    Sum sum(shared, blocks);
    const uint64_t seed = p.drop.on ? p.drop.rng[0] : 0, step = p.drop.on ? p.drop.rng[1] : 0;
    const int groups_row = (p.width + 7) / 8;
    const float inv = 1.f / (float)p.width;
    const bool exists = q.n > 0;
    Oct gw_post, gscale, gw_pre;
    gw_post.fill(0.f); gscale.fill(0.f); gw_pre.fill(0.f);
    Largest<T> largest;
    int row = q.first;
    Rows<T, VEC, Lane<WARPS, CLUSTER>::kThreads> in;
    in.bind(staged, q.n);
    float4 stats = make_float4(0.f, 1.f, 0.f, 1.f);
    auto request = [&](long long r, int stage) {
        if (r < p.rows) {
            if (p.dz != nullptr) {
                in.request(stage, 0, p.y + r * p.ld_y + q.col, q.n);
                in.request(stage, 2, (const T*)p.dz + r * p.ld_z + q.col, q.n);
            }
            if (p.dy != nullptr) in.request(stage, 1, p.dy + r * p.ld_y + q.col, q.n);
            if (p.u != nullptr) in.request(stage, 3, (const T*)p.u + r * p.ld_u + q.col, q.n);
            if (p.gate != nullptr) in.request(stage, 4, (const T*)p.gate + r * p.ld_gate + q.col, q.n);
        }
        in.commit();
    };
    if (VEC)
        for (int k = 0; k < in.kStages; ++k) request(row + (long long)k * q.step, k);
    if (p.stats != nullptr && row < p.rows) stats = reinterpret_cast<const float4*>(p.stats)[row];
    int stage = 0;
    while (row < p.rows) {
        const int next = q.step < p.rows - row ? row + q.step : p.rows;
        const float4 st = stats;
        if (p.stats != nullptr && next < p.rows) stats = reinterpret_cast<const float4*>(p.stats)[next];
        if (!VEC) request(row, 0);
        in.wait();
        Oct a, y, d, w;
        Raw8<T> un, gn;                                     // unpacked where they are used
        if (p.dy != nullptr) in.get(stage, 1, a);
        else a.fill(0.f);
        if (p.dz != nullptr) {
            in.get(stage, 0, y);
            in.get(stage, 2, d);
        }
        if (p.u != nullptr) in.raw(stage, 3, un);
        if (p.gate != nullptr) in.raw(stage, 4, gn);
        if (p.dz != nullptr) {
            load_weights<VEC>(p.w_pre, q.col, q.n, w);
            float2 m0 = pair(0.f), m1 = pair(0.f);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (CENTER) y.v[j] = __fadd2_rn(y.v[j], pair(-st.z));
                y.v[j] = __fmul2_rn(y.v[j], pair(st.w));
                d.v[j] = __fmul2_rn(d.v[j], pair(p.cot_in));
                gw_pre.v[j] = __ffma2_rn(d.v[j], y.v[j], gw_pre.v[j]);
                d.v[j] = __fmul2_rn(d.v[j], w.v[j]);
                m0 = __ffma2_rn(d.v[j], y.v[j], m0);
                if (CENTER) m1 = __fadd2_rn(m1, d.v[j]);
            }
            if (p.pre != MPODE_NORM_NONE) {
                float m[N];
                m[0] = m0.x + m0.y;
                if (CENTER) m[N - 1] = m1.x + m1.y;
                sum(m, q);
                m0 = pair(-m[0] * inv);
                m1 = pair(CENTER && p.pre == MPODE_NORM_MEANVAR ? -m[N - 1] * inv : 0.f);
            } else m0 = m1 = pair(0.f);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (CENTER) d.v[j] = __fadd2_rn(d.v[j], m1);
                a.v[j] = __ffma2_rn(__ffma2_rn(y.v[j], m0, d.v[j]), pair(st.w), a.v[j]);
            }
        }
        store8<float, VEC>(p.dy_out + row * p.ld_y + q.col, q.n, a);
        if (p.u != nullptr) {
        Oct u, g, c;
        unpack<T>(un, u);
        if (p.gate != nullptr) unpack<T>(gn, g);
        Kept keep;
        if (p.drop.on) keep = Kept(p.drop, (uint64_t)row * groups_row + q.col / 8, seed, step);
        load_weights<VEC>(p.w_post, q.col, q.n, w);
        load_weights<VEC>(p.scale, q.col, q.n, c);
        float2 m0 = pair(0.f), m1 = pair(0.f);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (CENTER) u.v[j] = __fadd2_rn(u.v[j], pair(-st.x));
            u.v[j] = __fmul2_rn(u.v[j], pair(st.y));
            float2 t = __fmul2_rn(a.v[j], pair(p.h * p.drop.scale));
            if (p.drop.on) {
                if (!keep[2 * j]) t.x = 0.f;
                if (!keep[2 * j + 1]) t.y = 0.f;
            }
            if (VEC ? !exists : 2 * j >= q.n) t.x = 0.f;    // columns that do not exist add nothing to the sums
            if (VEC ? !exists : 2 * j + 1 >= q.n) t.y = 0.f;
            const float2 v = __fmul2_rn(u.v[j], w.v[j]);
            if (p.gate != nullptr) {
                float2 slope;
                const float2 sig = gate_of<T, true>(g.v[j], slope);
                gscale.v[j] = __ffma2_rn(t, __fmul2_rn(v, sig), gscale.v[j]);
                t = __fmul2_rn(t, c.v[j]);
                g.v[j] = __fmul2_rn(__fmul2_rn(t, v), __fmul2_rn(slope, pair(p.cot_out)));
                t = __fmul2_rn(t, sig);
            } else {
                gscale.v[j] = __ffma2_rn(t, v, gscale.v[j]);
                t = __fmul2_rn(t, c.v[j]);
            }
            gw_post.v[j] = __ffma2_rn(t, u.v[j], gw_post.v[j]);
            a.v[j] = __fmul2_rn(t, w.v[j]);
            m0 = __ffma2_rn(a.v[j], u.v[j], m0);
            if (CENTER) m1 = __fadd2_rn(m1, a.v[j]);
        }
        Raw8<T> out;
        if (p.dgate != nullptr) {
            pack<T>(g, out);
            if (p.flag != nullptr) largest.see(out, q.n);
            store_raw<T, VEC>((T*)p.dgate + row * p.ld_gate + q.col, q.n, out);
        }
        if (p.post != MPODE_NORM_NONE) {
            float m[N];
            m[0] = m0.x + m0.y;
            if (CENTER) m[N - 1] = m1.x + m1.y;
            sum(m, q);
            m0 = pair(-m[0] * inv);
            m1 = pair(CENTER && p.post == MPODE_NORM_MEANVAR ? -m[N - 1] * inv : 0.f);
        } else m0 = m1 = pair(0.f);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (CENTER) a.v[j] = __fadd2_rn(a.v[j], m1);
            a.v[j] = __fmul2_rn(__fmul2_rn(__ffma2_rn(u.v[j], m0, a.v[j]), pair(st.y)), pair(p.cot_out));
        }
        pack<T>(a, out);
        if (p.flag != nullptr) largest.see(out, q.n);
        store_raw<T, VEC>((T*)p.du + row * p.ld_u + q.col, q.n, out);
        }
        if (VEC) {                                          // this row's pieces have been used: its stage is free
            request(row + (long long)in.kStages * q.step, stage);
            stage = stage + 1 < in.kStages ? stage + 1 : 0;
        }
        row = next;
    }
    warp_flag_or(p.flag, largest.nonfinite());
    if (p.partial != nullptr) {
        float* out = p.partial + (long long)q.first * 3 * p.width + q.col;
        store8<float, VEC>(out, q.n, gw_post);
        store8<float, VEC>(out + p.width, q.n, gscale);
        store8<float, VEC>(out + 2 * p.width, q.n, gw_pre);
    }
    sum.end();
}

}  // namespace

cudaError_t launch_residual_backward(mpode_dtype dt, const ResArgs& a, const ResShape& s, bool vec, bool center, cudaStream_t st) {
    return with_low(dt, [&](auto t) {
        using T = decltype(t);
        return with_shape(s, [&](auto warps, auto cluster) {
            constexpr int W = warps.value;
            constexpr bool C = cluster.value;
            using R = Rows<T, true, Lane<W, C>::kThreads>;
            const size_t smem = (size_t)Lane<W, C>::kThreads * R::kStages * R::kPieces * 16;
            if (!vec) {
                if constexpr (W == 2 || W == 4) return cudaErrorInvalidValue;
                else return launch_rows(residual_backward_kernel<T, false, true, W, C>, a, s, 0, st);
            }
            return center ? launch_rows(residual_backward_kernel<T, true, true, W, C>, a, s, smem, st)
                          : launch_rows(residual_backward_kernel<T, true, false, W, C>, a, s, smem, st);
        });
    });
}

}  // namespace mpode
