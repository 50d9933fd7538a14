// Gated linear recurrence along a sequence, forward and backward: the time loop of a linear relaxation equation as a scan.
//
// With b = sigmoid(g) and a = 1 - b, per channel: y_i = a y_{i-1} + b x_i (coupled: one implicit Euler step of y' = lambda (x - y),
// g = log(h lambda)) or y_i = a y_{i-1} + x_i.  Backward: l_i = dy_i + r_i, r_{i-1} = a_i l_i, from r behind the last step; coupled dx = b l,
// dg = l (x - y_{i-1}) a b, else dx = l, dg = -l y_{i-1} a b.
//
// Every step is an affine map y -> A y + u.  A block holds 32 lanes of channels and W warps along the time axis; a warp's steps lie in its
// registers.  First each warp composes its own steps, the blocks of a cluster exchange their products through distributed shared memory, and
// then every warp runs its steps again from the state in front of them: the data is read once and written once, nothing is kept in device
// memory and no block waits for another but at the cluster's barrier.
//
// Precision: b is formed with a relative error (no cancellation for g << 0), and every decay is written y - b y in one rounding, so that memories of
// a million steps (b = 1e-6) decay at the right rate, where a rounded a = 1 - b would not, and b = 1 forgets everything, exactly.  For the same reason a
// composed map is kept as y -> y - C y + u with C = 1 - A.
#include <stdarg.h>
#include <stdio.h>

#include <math.h>

#include "operators.h"
#include "rows.cuh"

namespace mpode {
namespace {

struct RecArgs {
    const void *x, *gate, *y, *dy;     // y, dy: backward only
    const float* y0;                   // [n_seq, width] or null (zero)
    const float* dyT;                  // backward: [n_seq, width] or null
    const int* lengths;                // [n_seq] or null
    void *out, *out2;                  // forward: y; backward: dx, dgate
    float* last;                       // forward: y_T; backward: dy0; may be null
    unsigned* flag;
    long long in_seq, in_step, out_seq, out_step;
    int n_seq, n_steps, width;
};

// V channels of a row as one access: two (a 32-bit word, or 64 bits of float32), or one where widths or addresses are odd
template <typename T, int V> struct Word;
template <> struct Word<float, 1> {
    using type = float;
    static __device__ __forceinline__ void get(type w, float (&f)[1]) { f[0] = w; }
    static __device__ __forceinline__ type put(const float (&f)[1]) { return f[0]; }
    static __device__ __forceinline__ type negate(type w) { return -w; }
};
template <> struct Word<float, 2> {
    using type = float2;
    static __device__ __forceinline__ void get(type w, float (&f)[2]) { f[0] = w.x; f[1] = w.y; }
    static __device__ __forceinline__ type put(const float (&f)[2]) { return make_float2(f[0], f[1]); }
    static __device__ __forceinline__ type negate(type w) { return make_float2(-w.x, -w.y); }
};
template <> struct Word<__nv_bfloat16, 1> {
    using type = __nv_bfloat16;
    static __device__ __forceinline__ void get(type w, float (&f)[1]) { f[0] = __bfloat162float(w); }
    static __device__ __forceinline__ type put(const float (&f)[1]) { return __float2bfloat16_rn(f[0]); }
    static __device__ __forceinline__ type negate(type w) { return __hneg(w); }
};
template <> struct Word<__half, 1> {
    using type = __half;
    static __device__ __forceinline__ void get(type w, float (&f)[1]) { f[0] = __half2float(w); }
    static __device__ __forceinline__ type put(const float (&f)[1]) { return __float2half_rn(f[0]); }
    static __device__ __forceinline__ type negate(type w) { return __hneg(w); }
};
template <typename T> struct Word<T, 2> {
    using type = uint32_t;
    static __device__ __forceinline__ void get(type w, float (&f)[2]) { const float2 t = Pair<T>::get(w); f[0] = t.x; f[1] = t.y; }
    static __device__ __forceinline__ type put(const float (&f)[2]) { return Pair<T>::put(f[0], f[1]); }
    static __device__ __forceinline__ type negate(type w) { return w ^ 0x80008000u; }
};
template <typename T, int V> __device__ __forceinline__ typename Word<T, V>::type word_of(float v) {
    float f[V];
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = v;
    return Word<T, V>::put(f);
}
template <typename T, int V> __device__ __forceinline__ bool word_nonfinite(typename Word<T, V>::type w) {
    float f[V];
    Word<T, V>::get(w, f);
    bool bad = false;
#pragma unroll
    for (int v = 0; v < V; ++v) bad |= Low<float>::nonfinite(f[v]);
    return bad;
}

// a b + c and a + b on all channels of a lane; two of them are one instruction
template <int V> struct Ops {
    static __device__ __forceinline__ void fma(float (&d)[V], const float (&a)[V], const float (&b)[V], const float (&c)[V]) {
        if constexpr (V == 2) {
            asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}"
                : "=f"(d[0]), "=f"(d[1]) : "f"(a[0]), "f"(a[1]), "f"(b[0]), "f"(b[1]), "f"(c[0]), "f"(c[1]));
        } else d[0] = fmaf(a[0], b[0], c[0]);
    }
    static __device__ __forceinline__ void add(float (&d)[V], const float (&a)[V], const float (&b)[V]) {
        if constexpr (V == 2) {
            asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
                : "=f"(d[0]), "=f"(d[1]) : "f"(a[0]), "f"(a[1]), "f"(b[0]), "f"(b[1]));
        } else d[0] = a[0] + b[0];
    }
    static __device__ __forceinline__ void mul(float (&d)[V], const float (&a)[V], const float (&b)[V]) {
        if constexpr (V == 2) {
            asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
                : "=f"(d[0]), "=f"(d[1]) : "f"(a[0]), "f"(a[1]), "f"(b[0]), "f"(b[1]));
        } else d[0] = a[0] * b[0];
    }
};

// -sigmoid(g) = -b and the slope b (1 - b), which is e b^2 with e = exp(-g).  16-bit gates: the device's approximate power and quotient (2^-22
// relative, and the argument's rounding adds |g| 2^-24), which cost 5 instructions where the accurate ones of float32 cost 15; the exponent is
// kept below 2^126, so that e b^2 is finite: b is 1e-38 instead of less, which no float32 state feels.
template <typename T> __device__ __forceinline__ void negated_gate(float g, float& nb, float& slope) {
    float e;
    if constexpr (sizeof(T) == 4) {
        e = expf(-g);
        const float b = __fdividef(1.f, 1.f + e);
        nb = -b;
        slope = b * (e > 1.f ? 1.f - b : e * b);
    } else {
        asm("min.NaN.f32 %0, %1, %2;" : "=f"(e) : "f"(g * -1.4426950408889634f), "f"(126.f));
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(nb) : "f"(-1.f - e));
        slope = e * nb * nb;
    }
}

// one step, nb = -b; x is negated when coupled
template <bool COUPLED, int V> __device__ __forceinline__ void step_forward(float (&y)[V], const float (&nb)[V], const float (&x)[V]) {
    float kept[V];
    Ops<V>::fma(kept, nb, y, y);
    if constexpr (COUPLED) Ops<V>::fma(y, nb, x, kept);
    else Ops<V>::add(y, kept, x);
}
// The composed map y -> A y + u of some steps, C = 1 - A: A exact to its last bits where it is small (a reset leaves A = 0), C where the steps
// forget little.  Kept per lane as A, -C and u.
template <int V> struct Map {
    float A[V], nC[V], u[V];
    __device__ __forceinline__ Map() {
#pragma unroll
        for (int v = 0; v < V; ++v) { A[v] = 1.f; nC[v] = 0.f; u[v] = 0.f; }
    }
    __device__ __forceinline__ void decay(const float (&nb)[V]) {
        float one[V], left[V];
#pragma unroll
        for (int v = 0; v < V; ++v) one[v] = 1.f;
        Ops<V>::fma(A, nb, A, A);
        Ops<V>::add(left, one, nC);
        Ops<V>::fma(nC, nb, left, nC);
    }
};
struct Affine { float A, C, u; };
__device__ __forceinline__ float apply(const Affine& m, float y) { return (m.A < 0.5f ? m.A * y : fmaf(-m.C, y, y)) + m.u; }
// first m, then n
__device__ __forceinline__ Affine compose(const Affine& m, const Affine& n) {
    return {m.A * n.A, fmaf(n.C, 1.f - m.C, m.C), apply(n, m.u)};
}

__device__ __forceinline__ unsigned smem_of(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ unsigned peer_of(unsigned local, unsigned rank) {
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(rank));
    return r;
}
__device__ __forceinline__ void peer_store(unsigned at, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

constexpr int kMaxWarps = 8, kMaxCluster = 8;

// Shared memory of the exchange: products of the block's warps and of the cluster's blocks, two sets used in turn (a set is written again
// only behind the next barrier, which nobody passes before the set has been read)
template <int V> struct Exchange {
    float warp[2][kMaxWarps][3][32 * V];
    float block[2][kMaxCluster][3][32 * V];
};
template <int V> __device__ __forceinline__ Affine fetch(const float (&t)[3][32 * V], int i) { return {t[0][i], t[1][i], t[2][i]}; }

// The state in front of this warp's steps, from the state in front of all of this round's steps (`carry`, replaced by the one behind them).
// Called by all threads of the cluster with the same number of blocks.
template <int V> __device__ __forceinline__ void exchange(Exchange<V>& ex, int set, const Map<V>& own, float (&carry)[V], float (&start)[V],
                                                          int blocks, int rank) {
    const int lane = threadIdx.x, warp = threadIdx.y, warps = blockDim.y;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        ex.warp[set][warp][0][v * 32 + lane] = own.A[v];
        ex.warp[set][warp][1][v * 32 + lane] = -own.nC[v];
        ex.warp[set][warp][2][v * 32 + lane] = own.u[v];
    }
    __syncthreads();
    if (blocks == 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float y = carry[v];
            for (int w = 0; w < warps; ++w) {
                if (w == warp) start[v] = y;
                y = apply(fetch<V>(ex.warp[set][w], v * 32 + lane), y);
            }
            carry[v] = y;
        }
        return;
    }
    if (warp < blocks) {                                                    // this block's product goes to every block, one warp to each
#pragma unroll
        for (int v = 0; v < V; ++v) {
            Affine m = fetch<V>(ex.warp[set][0], v * 32 + lane);
            for (int w = 1; w < warps; ++w) m = compose(m, fetch<V>(ex.warp[set][w], v * 32 + lane));
            for (int to = warp; to < blocks; to += warps) {
                peer_store(peer_of(smem_of(&ex.block[set][rank][0][v * 32 + lane]), to), m.A);
                peer_store(peer_of(smem_of(&ex.block[set][rank][1][v * 32 + lane]), to), m.C);
                peer_store(peer_of(smem_of(&ex.block[set][rank][2][v * 32 + lane]), to), m.u);
            }
        }
    }
    cluster_arrive();
    cluster_wait();
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float y = carry[v];
        for (int r = 0; r < blocks; ++r) {
            if (r == rank) start[v] = y;
            y = apply(fetch<V>(ex.block[set][r], v * 32 + lane), y);
        }
        carry[v] = y;
        y = start[v];
        for (int w = 0; w < warp; ++w) y = apply(fetch<V>(ex.warp[set][w], v * 32 + lane), y);
        start[v] = y;
    }
}

// which channels and steps a thread works on
struct Place { int seq, col, len, rank; bool on; };
template <int V> __device__ __forceinline__ Place place(const RecArgs& p, int blocks) {
    const int tiles = (p.width + 32 * V - 1) / (32 * V), tile = blockIdx.x / blocks;
    Place q;
    q.rank = blockIdx.x - tile * blocks;
    q.seq = tile / tiles;
    q.col = (tile - q.seq * tiles) * 32 * V + threadIdx.x * V;
    q.on = q.col < p.width;
    q.len = p.n_steps;
    if (p.lengths != nullptr) q.len = min(max(p.lengths[q.seq], 0), p.n_steps);
    return q;
}

// A warp's tile of one array: L steps of V channels a lane, from step t0 on (step: the stride; negative backwards in time), `n` of which exist; the
// others hold `fill`
template <typename T, int V, int L> __device__ __forceinline__ void load_tile(typename Word<T, V>::type (&w)[L], const T* p, long long step, int n, float fill) {
    using word = typename Word<T, V>::type;
    if (n >= L) {
#pragma unroll
        for (int i = 0; i < L; ++i, p += step) w[i] = *(const word*)p;
    } else {
        const word none = word_of<T, V>(fill);
#pragma unroll
        for (int i = 0; i < L; ++i, p += step) {
            w[i] = none;
            if (i < n) w[i] = *(const word*)p;
        }
    }
}

template <typename T, int V, bool COUPLED, int L>
__global__ void __launch_bounds__(32 * kMaxWarps, 2) recurrence_forward_kernel(const RecArgs p, const int blocks) {
    using W = Word<T, V>;
    using word = typename W::type;
    __shared__ Exchange<V> ex;
    const Place q = place<V>(p, blocks);
    if (blocks > 1) cluster_arrive();                       // nobody writes into a block that has not started
    const T* x = (const T*)p.x + q.seq * p.in_seq + q.col;
    const T* g = (const T*)p.gate + q.seq * p.in_seq + q.col;
    T* out = (T*)p.out + q.seq * p.out_seq + q.col;
    const bool alone = blocks == 1 && blockDim.y == 1;
    const int stride = blocks * (int)blockDim.y * L;
    float carry[V];
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = p.y0 != nullptr && q.on ? p.y0[(long long)q.seq * p.width + q.col + v] : 0.f;
    long long t0 = (q.rank * (int)blockDim.y + (int)threadIdx.y) * L;
    // steps that do not exist keep the state: x = 0, gate = -inf
    int n = q.on ? (int)max(0ll, min((long long)L, q.len - t0)) : 0;
    word xw[L], gw[L];
    load_tile<T, V, L>(xw, x + t0 * p.in_step, p.in_step, n, 0.f);
    load_tile<T, V, L>(gw, g + t0 * p.in_step, p.in_step, n, -INFINITY);
    if (blocks > 1) cluster_wait();
    int set = 0;
    for (long long base = 0; base < q.len; base += stride, set ^= 1) {
        float nb[L][V], start[V];
        word now[L];
#pragma unroll
        for (int i = 0; i < L; ++i) {
            float f[V], slope;
            W::get(gw[i], f);
#pragma unroll
            for (int v = 0; v < V; ++v) negated_gate<T>(f[v], nb[i][v], slope);
            now[i] = COUPLED ? W::negate(xw[i]) : xw[i];
        }
        // the next round's steps are on their way while this one's are summed
        const int m = n;
        T* const o = out + t0 * p.out_step;
        t0 += stride;
        n = q.on ? (int)max(0ll, min((long long)L, q.len - t0)) : 0;
        load_tile<T, V, L>(xw, x + t0 * p.in_step, p.in_step, n, 0.f);
        load_tile<T, V, L>(gw, g + t0 * p.in_step, p.in_step, n, -INFINITY);
#pragma unroll
        for (int v = 0; v < V; ++v) start[v] = carry[v];
        if (!alone) {
            Map<V> own;
#pragma unroll
            for (int i = 0; i < L; ++i) {
                float xs[V];
                W::get(now[i], xs);
                own.decay(nb[i]);
                step_forward<COUPLED, V>(own.u, nb[i], xs);
            }
            exchange<V>(ex, set, own, carry, start, blocks, q.rank);
        }
        T* to = o;
#pragma unroll
        for (int i = 0; i < L; ++i, to += p.out_step) {
            float xs[V];
            W::get(now[i], xs);
            step_forward<COUPLED, V>(start, nb[i], xs);
            if (i < m) *(word*)to = W::put(start);
        }
        if (alone) {
#pragma unroll
            for (int v = 0; v < V; ++v) carry[v] = start[v];
        }
    }
    if (p.last != nullptr && q.on && q.rank == 0 && threadIdx.y == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) p.last[(long long)q.seq * p.width + q.col + v] = carry[v];
    }
}

// Steps counted from the end: step i of a warp is time t0 - i
template <typename T, int V, bool COUPLED, int L>
__global__ void __launch_bounds__(32 * kMaxWarps, 2) recurrence_backward_kernel(const RecArgs p, const int blocks) {
    using W = Word<T, V>;
    using word = typename W::type;
    __shared__ Exchange<V> ex;
    const Place q = place<V>(p, blocks);
    if (blocks > 1) cluster_arrive();
    const long long in0 = q.seq * p.in_seq + q.col, out0 = q.seq * p.out_seq + q.col, w0 = (long long)q.seq * p.width + q.col;
    const T *x = (const T*)p.x + in0, *g = (const T*)p.gate + in0, *y = (const T*)p.y + out0, *dy = (const T*)p.dy + out0;
    T *dx = (T*)p.out + in0, *dg = (T*)p.out2 + in0;
    const bool alone = blocks == 1 && blockDim.y == 1;
    const int stride = blocks * (int)blockDim.y * L;
    float carry[V];
    bool bad = false;
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = p.dyT != nullptr && q.on ? p.dyT[w0 + v] : 0.f;
    long long t0 = (long long)q.len - 1 - (q.rank * (int)blockDim.y + (int)threadIdx.y) * L;
    int n = q.on ? (int)max(0ll, min((long long)L, t0 + 1)) : 0;
    word xw[L], gw[L], dw[L], yw[L];
    auto load = [&]() {
        load_tile<T, V, L>(gw, g + t0 * p.in_step, -p.in_step, n, -INFINITY);
        load_tile<T, V, L>(dw, dy + t0 * p.out_step, -p.out_step, p.dy != nullptr ? n : 0, 0.f);
        if (COUPLED) load_tile<T, V, L>(xw, x + t0 * p.in_step, -p.in_step, n, 0.f);
        load_tile<T, V, L>(yw, y + (t0 - 1) * p.out_step, -p.out_step, (int)min((long long)n, t0), 0.f);      // the states in front of the steps
    };
    load();
    if (blocks > 1) cluster_wait();
    int set = 0;
    for (long long base = 0; base < q.len; base += stride, set ^= 1) {
        float nb[L][V], slope[L][V], start[V];
        word now[L], before[L], given[L];
#pragma unroll
        for (int i = 0; i < L; ++i) {
            float f[V];
            W::get(gw[i], f);
#pragma unroll
            for (int v = 0; v < V; ++v) negated_gate<T>(f[v], nb[i][v], slope[i][v]);
            now[i] = xw[i]; before[i] = yw[i]; given[i] = dw[i];
        }
        const int m = n, first = t0 < L ? (int)t0 : L;                       // index of time 0
        const long long at = t0 * p.in_step;
        t0 -= stride;
        n = q.on ? (int)max(0ll, min((long long)L, t0 + 1)) : 0;
        load();
#pragma unroll
        for (int v = 0; v < V; ++v) start[v] = carry[v];
        if (!alone) {
            Map<V> own;
#pragma unroll
            for (int i = 0; i < L; ++i) {
                float d[V], l[V];
                W::get(given[i], d);
                own.decay(nb[i]);
                Ops<V>::add(l, own.u, d);
                Ops<V>::fma(own.u, nb[i], l, l);
            }
            exchange<V>(ex, set, own, carry, start, blocks, q.rank);
        }
        T *ox = dx + at, *og = dg + at;
#pragma unroll
        for (int i = 0; i < L; ++i, ox -= p.in_step, og -= p.in_step) {
            float xs[V], ys[V], d[V], l[V], gx[V], gg[V];
            W::get(given[i], d);
            W::get(before[i], ys);
            if (i == first && p.y0 != nullptr && q.on) {
#pragma unroll
                for (int v = 0; v < V; ++v) ys[v] = p.y0[w0 + v];
            }
            Ops<V>::add(l, start, d);
            Ops<V>::fma(start, nb[i], l, l);
            if (COUPLED) W::get(now[i], xs);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                gx[v] = COUPLED ? -nb[i][v] * l[v] : l[v];
                gg[v] = slope[i][v] * l[v] * (COUPLED ? xs[v] - ys[v] : -ys[v]);
            }
            if (i < m) {
                const word wx = W::put(gx), wg = W::put(gg);
                bad |= word_nonfinite<T, V>(wx) || word_nonfinite<T, V>(wg);
                *(word*)ox = wx;
                *(word*)og = wg;
            }
        }
        if (alone) {
#pragma unroll
            for (int v = 0; v < V; ++v) carry[v] = start[v];
        }
    }
    if (p.last != nullptr && q.on && q.rank == 0 && threadIdx.y == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) p.last[w0 + v] = carry[v];
    }
    warp_flag_or(p.flag, bad);
}

// How a call is spread over the GPU: warps along the time axis of a block, then blocks of a cluster, until every SM has its warps or no steps are left
struct Shape { int warps, blocks; long long tiles; };
Shape shape_of(const mpode_recurrence_desc& d, int lanes_width, int steps_of_warp) {
    Shape s;
    s.tiles = (long long)d.n_seq * ((d.width + lanes_width - 1) / lanes_width);
    s.warps = s.blocks = 1;
    while (s.warps < kMaxWarps && (long long)s.warps * steps_of_warp < d.n_steps) s.warps *= 2;
    while (s.blocks < kMaxCluster && s.tiles * s.blocks < 148 && (long long)s.blocks * s.warps * steps_of_warp < d.n_steps) s.blocks *= 2;
    return s;
}

cudaError_t launch(void (*kernel)(const RecArgs, const int), const RecArgs& a, const Shape& s, cudaStream_t st) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(s.tiles * s.blocks));
    cfg.blockDim = dim3(32, s.warps);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)s.blocks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = s.blocks > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, a, s.blocks);
}

template <typename T, int V> constexpr int kForwardSteps = sizeof(T) * V > 4 ? 8 : 16;
template <typename T, int V> constexpr int kBackwardSteps = sizeof(T) * V > 4 ? 4 : 8;

template <typename T, int V> cudaError_t run_forward(const mpode_recurrence_desc& d, const RecArgs& a, cudaStream_t st) {
    constexpr int L = kForwardSteps<T, V>;
    const Shape s = shape_of(d, 32 * V, L);
    return d.coupled ? launch(recurrence_forward_kernel<T, V, true, L>, a, s, st) : launch(recurrence_forward_kernel<T, V, false, L>, a, s, st);
}
template <typename T, int V> cudaError_t run_backward(const mpode_recurrence_desc& d, const RecArgs& a, cudaStream_t st) {
    constexpr int L = kBackwardSteps<T, V>;
    const Shape s = shape_of(d, 32 * V, L);
    return d.coupled ? launch(recurrence_backward_kernel<T, V, true, L>, a, s, st) : launch(recurrence_backward_kernel<T, V, false, L>, a, s, st);
}

// the checks that both directions share; fills in strides that are zero
mpode_status check(const mpode_recurrence_desc* d, RecArgs& a) {
    if (d == nullptr) return operator_fail(MPODE_ERR_INVALID_ARG, "recurrence: null descriptor");
    if (!known_dtype(d->low)) return operator_fail(MPODE_ERR_INVALID_ARG, "recurrence: unknown format %d", (int)d->low);
    if (d->n_seq < 0 || d->n_steps < 0 || d->width < 1)
        return operator_fail(MPODE_ERR_INVALID_ARG, "recurrence: n_seq %d, n_steps %d, width %d", d->n_seq, d->n_steps, d->width);
    if ((long long)d->n_seq * (((long long)d->width + 31) / 32) * kMaxCluster > 0x7fffffffll)
        return operator_fail(MPODE_ERR_UNSUPPORTED, "recurrence: %d sequences of width %d are more than one launch holds", d->n_seq, d->width);
    const long long lo = (long long)d->width, seq = lo * d->n_steps;
    a.in_step = d->in_step_stride ? d->in_step_stride : lo;
    a.in_seq = d->in_seq_stride ? d->in_seq_stride : seq;
    a.out_step = d->out_step_stride ? d->out_step_stride : lo;
    a.out_seq = d->out_seq_stride ? d->out_seq_stride : seq;
    if ((d->n_steps > 1 && (a.in_step < lo || a.out_step < lo)) || (d->n_seq > 1 && d->n_steps > 0 && (a.in_seq < lo || a.out_seq < lo)))
        return operator_fail(MPODE_ERR_INVALID_ARG, "recurrence: a stride is smaller than the width %d", d->width);
    // (the last element of one sequence lies before the first of the next, or the last sequence of one step before the first of the next)
    const long long S = d->n_seq - 1, N = d->n_steps - 1;
    if (S > 0 && N > 0 && ((a.in_seq <= N * a.in_step + lo - 1 && a.in_step <= S * a.in_seq + lo - 1) ||
                           (a.out_seq <= N * a.out_step + lo - 1 && a.out_step <= S * a.out_seq + lo - 1)))
        return operator_fail(MPODE_ERR_INVALID_ARG, "recurrence: the strides make rows overlap");
    a.n_seq = d->n_seq; a.n_steps = d->n_steps; a.width = d->width;
    return MPODE_OK;
}
// two channels an access need even widths and strides and rows aligned to two elements
bool words_fit(const mpode_recurrence_desc& d, const RecArgs& a) {
    if (d.width & 1) return false;
    if ((a.in_step | a.in_seq | a.out_step | a.out_seq) & 1) return false;
    const void* const all[] = {a.x, a.gate, a.y, a.dy, a.out, a.out2};
    for (const void* q : all)
        if (misaligned(q, 2 * low_size(d.low))) return false;
    return true;
}
mpode_status check_pointers(const mpode_recurrence_desc& d, const RecArgs& a) {
    const void* const low[] = {a.x, a.gate, a.y, a.dy, a.out, a.out2};
    for (const void* q : low)
        if (misaligned(q, low_size(d.low))) return operator_fail(MPODE_ERR_INVALID_ARG, "recurrence: a pointer is not aligned to its elements");
    const void* const wide[] = {a.y0, a.dyT, a.lengths, a.last, a.flag};
    for (const void* q : wide)
        if (misaligned(q, 4)) return operator_fail(MPODE_ERR_INVALID_ARG, "recurrence: a pointer is not aligned to its elements");
    return MPODE_OK;
}

thread_local char tl_message[256] = "";

}  // namespace

mpode_status operator_fail(mpode_status s, const char* format, ...) {
    va_list ap;
    va_start(ap, format);
    vsnprintf(tl_message, sizeof(tl_message), format, ap);
    va_end(ap);
    return s;
}
mpode_status operator_launched(cudaError_t e, const char* entry) {
    if (e == cudaSuccess) return MPODE_OK;
    (void)cudaGetLastError();
    return operator_fail(MPODE_ERR_CUDA, "%s: %s", entry, cudaGetErrorString(e));
}

}  // namespace mpode

using namespace mpode;

extern "C" {

const char* mpode_operator_error(void) { return tl_message; }

mpode_status mpode_recurrence_forward(const mpode_recurrence_desc* desc, void* cuda_stream, const void* x_dev, const void* gate_dev,
                                      const float* y0_dev, const int* lengths_dev, void* y_dev, float* yT_dev) {
    RecArgs a{};
    const mpode_status bad = check(desc, a);
    if (bad != MPODE_OK) return bad;
    a.x = x_dev; a.gate = gate_dev; a.y0 = y0_dev; a.lengths = lengths_dev; a.out = y_dev; a.last = yT_dev;
    if (desc->n_seq == 0) return MPODE_OK;
    if (desc->n_steps > 0 && (!x_dev || !gate_dev || !y_dev)) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_recurrence_forward: null pointer argument");
    const mpode_status off = check_pointers(*desc, a);
    if (off != MPODE_OK) return off;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    if (desc->low == MPODE_F32) e = words_fit(*desc, a) ? run_forward<float, 2>(*desc, a, st) : run_forward<float, 1>(*desc, a, st);
    else if (desc->low == MPODE_BF16) e = words_fit(*desc, a) ? run_forward<__nv_bfloat16, 2>(*desc, a, st) : run_forward<__nv_bfloat16, 1>(*desc, a, st);
    else e = words_fit(*desc, a) ? run_forward<__half, 2>(*desc, a, st) : run_forward<__half, 1>(*desc, a, st);
    return operator_launched(e, "mpode_recurrence_forward");
}

mpode_status mpode_recurrence_backward(const mpode_recurrence_desc* desc, void* cuda_stream, const void* x_dev, const void* gate_dev,
                                       const float* y0_dev, const int* lengths_dev, const void* y_dev, const void* dL_dy_dev,
                                       const float* dL_dyT_dev, void* dL_dx_dev, void* dL_dgate_dev, float* dL_dy0_dev, unsigned* flag_dev) {
    RecArgs a{};
    const mpode_status bad = check(desc, a);
    if (bad != MPODE_OK) return bad;
    a.x = x_dev; a.gate = gate_dev; a.y0 = y0_dev; a.lengths = lengths_dev; a.y = y_dev; a.dy = dL_dy_dev; a.dyT = dL_dyT_dev;
    a.out = dL_dx_dev; a.out2 = dL_dgate_dev; a.last = dL_dy0_dev; a.flag = flag_dev;
    if (desc->n_seq == 0) return MPODE_OK;
    if (desc->n_steps > 0 && ((!x_dev && desc->coupled) || !gate_dev || !y_dev || !dL_dx_dev || !dL_dgate_dev))
        return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_recurrence_backward: null pointer argument");
    const mpode_status off = check_pointers(*desc, a);
    if (off != MPODE_OK) return off;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    if (desc->low == MPODE_F32) e = words_fit(*desc, a) ? run_backward<float, 2>(*desc, a, st) : run_backward<float, 1>(*desc, a, st);
    else if (desc->low == MPODE_BF16) e = words_fit(*desc, a) ? run_backward<__nv_bfloat16, 2>(*desc, a, st) : run_backward<__nv_bfloat16, 1>(*desc, a, st);
    else e = words_fit(*desc, a) ? run_backward<__half, 2>(*desc, a, st) : run_backward<__half, 1>(*desc, a, st);
    return operator_launched(e, "mpode_recurrence_backward");
}

}  // extern "C"
