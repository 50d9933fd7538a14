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
// Precision: the smaller one of a and b is formed without cancellation and kept with a sign that says which one it is (s = b >= +0, or s = -a <= -0),
// so that memories of a million steps (b = 1e-6) and resets (a = 0) are both exact to rounding.  A composed map keeps the product A of the a
// and, for slow channels, its complement C = 1 - A, which a product of numbers near one would lose.
#include <stdarg.h>
#include <stdio.h>

#include "operators.h"

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

// one 32-bit word of channels (two 16-bit ones or a float), or a single 16-bit channel where widths or addresses are odd
template <typename T, int V> struct Word;
template <> struct Word<float, 1> {
    using type = float;
    static __device__ __forceinline__ void get(float w, float* f) { f[0] = w; }
    static __device__ __forceinline__ float put(const float* f) { return f[0]; }
};
template <> struct Word<__nv_bfloat16, 1> {
    using type = __nv_bfloat16;
    static __device__ __forceinline__ void get(type w, float* f) { f[0] = __bfloat162float(w); }
    static __device__ __forceinline__ type put(const float* f) { return __float2bfloat16_rn(f[0]); }
};
template <> struct Word<__half, 1> {
    using type = __half;
    static __device__ __forceinline__ void get(type w, float* f) { f[0] = __half2float(w); }
    static __device__ __forceinline__ type put(const float* f) { return __float2half_rn(f[0]); }
};
template <> struct Word<__nv_bfloat16, 2> {
    using type = __nv_bfloat162;
    static __device__ __forceinline__ void get(type w, float* f) { float2 t = __bfloat1622float2(w); f[0] = t.x; f[1] = t.y; }
    static __device__ __forceinline__ type put(const float* f) { return __floats2bfloat162_rn(f[0], f[1]); }
};
template <> struct Word<__half, 2> {
    using type = __half2;
    static __device__ __forceinline__ void get(type w, float* f) { float2 t = __half22float2(w); f[0] = t.x; f[1] = t.y; }
    static __device__ __forceinline__ type put(const float* f) { return __floats2half2_rn(f[0], f[1]); }
};
template <typename T, int V> __device__ __forceinline__ bool word_nonfinite(typename Word<T, V>::type w) {
    float f[V];
    Word<T, V>::get(w, f);
    bool bad = false;
#pragma unroll
    for (int v = 0; v < V; ++v) bad |= Low<float>::nonfinite(f[v]);
    return bad;
}

// s = sigmoid(g) where that is at most a half, else -(1 - sigmoid(g)); the sign bit tells the two apart even at zero
__device__ __forceinline__ float signed_gate(float g) {
    const float e = expf(-fabsf(g));
    const float small = __fdividef(e, 1.f + e);
    return copysignf(small, -g);
}
__device__ __forceinline__ bool resets(float s) { return (int)__float_as_uint(s) < 0; }     // a is the smaller one

template <bool COUPLED> __device__ __forceinline__ float step_forward(float s, float x, float y) {
    if (COUPLED) return fmaf(s, x - y, resets(s) ? x : y);
    return fmaf(-s, y, (resets(s) ? 0.f : y) + x);
}
__device__ __forceinline__ float decay(float s, float l) { return fmaf(-s, l, resets(s) ? 0.f : l); }     // a l

// y -> A y + u, C = 1 - A
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
template <int V> __device__ __forceinline__ void exchange(Exchange<V>& ex, int set, const Affine (&own)[V], float (&carry)[V], float (&start)[V],
                                                          int blocks, int rank) {
    const int lane = threadIdx.x, warp = threadIdx.y, warps = blockDim.y;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        ex.warp[set][warp][0][v * 32 + lane] = own[v].A;
        ex.warp[set][warp][1][v * 32 + lane] = own[v].C;
        ex.warp[set][warp][2][v * 32 + lane] = own[v].u;
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
    if (blocks > 1) cluster_wait();
    int set = 0;
    for (long long base = 0; base < q.len; base += stride, set ^= 1) {
        const long long t0 = base + (q.rank * (int)blockDim.y + (int)threadIdx.y) * L;
        const int n = q.on ? (int)max(0ll, min((long long)L, q.len - t0)) : 0;
        word xw[L], gw[L];
#pragma unroll
        for (int i = 0; i < L; ++i)
            if (i < n) {
                xw[i] = *(const word*)(x + (t0 + i) * p.in_step);
                gw[i] = *(const word*)(g + (t0 + i) * p.in_step);
            }
        float s[L][V], xs[L][V], start[V];
        Affine own[V];
#pragma unroll
        for (int v = 0; v < V; ++v) { own[v] = {1.f, 0.f, 0.f}; start[v] = carry[v]; }
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if (i < n) {
                float gf[V];
                W::get(gw[i], gf);
                W::get(xw[i], xs[i]);
#pragma unroll
                for (int v = 0; v < V; ++v) s[i][v] = signed_gate(gf[v]);
                if (!alone) {
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const float sv = s[i][v];
                        own[v].A = decay(sv, own[v].A);
                        own[v].C = step_forward<true>(sv, 1.f, own[v].C);
                        own[v].u = step_forward<COUPLED>(sv, xs[i][v], own[v].u);
                    }
                }
            }
        }
        if (!alone) exchange<V>(ex, set, own, carry, start, blocks, q.rank);
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if (i < n) {
#pragma unroll
                for (int v = 0; v < V; ++v) start[v] = step_forward<COUPLED>(s[i][v], xs[i][v], start[v]);
                *(word*)(out + (t0 + i) * p.out_step) = W::put(start);
            }
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

// Steps counted from the end: step i of a warp is time t = len - 1 - (tau0 + i)
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
    if (blocks > 1) cluster_wait();
    int set = 0;
    for (long long base = 0; base < q.len; base += stride, set ^= 1) {
        const long long t0 = q.len - 1 - (base + (q.rank * (int)blockDim.y + (int)threadIdx.y) * L);
        const int n = q.on ? (int)max(0ll, min((long long)L, t0 + 1)) : 0;
        word xw[L], gw[L], dw[L], yw[L];
#pragma unroll
        for (int i = 0; i < L; ++i)
            if (i < n) {
                gw[i] = *(const word*)(g + (t0 - i) * p.in_step);
                if (p.dy != nullptr) dw[i] = *(const word*)(dy + (t0 - i) * p.out_step);
                if (COUPLED) xw[i] = *(const word*)(x + (t0 - i) * p.in_step);
                if (t0 - i > 0) yw[i] = *(const word*)(y + (t0 - i - 1) * p.out_step);
            }
        float s[L][V], ds[L][V], start[V];
        Affine own[V];
#pragma unroll
        for (int v = 0; v < V; ++v) { own[v] = {1.f, 0.f, 0.f}; start[v] = carry[v]; }
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if (i < n) {
                float gf[V];
                W::get(gw[i], gf);
#pragma unroll
                for (int v = 0; v < V; ++v) { s[i][v] = signed_gate(gf[v]); ds[i][v] = 0.f; }
                if (p.dy != nullptr) W::get(dw[i], ds[i]);
                if (!alone) {
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const float sv = s[i][v];
                        own[v].A = decay(sv, own[v].A);
                        own[v].C = step_forward<true>(sv, 1.f, own[v].C);
                        own[v].u = decay(sv, own[v].u + ds[i][v]);
                    }
                }
            }
        }
        if (!alone) exchange<V>(ex, set, own, carry, start, blocks, q.rank);
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if (i < n) {
                float before[V], xs[V], gx[V], gg[V];
#pragma unroll
                for (int v = 0; v < V; ++v) before[v] = xs[v] = 0.f;
                if (t0 - i > 0) W::get(yw[i], before);
                else if (p.y0 != nullptr) {
#pragma unroll
                    for (int v = 0; v < V; ++v) before[v] = p.y0[w0 + v];
                }
                if (COUPLED) W::get(xw[i], xs);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float sv = s[i][v], small = fabsf(sv), big = 1.f - small, l = start[v] + ds[i][v];
                    gx[v] = COUPLED ? (resets(sv) ? big : small) * l : l;
                    gg[v] = l * (small * big) * (COUPLED ? xs[v] - before[v] : -before[v]);
                    start[v] = decay(sv, l);
                }
                const word wx = W::put(gx), wg = W::put(gg);
                bad |= word_nonfinite<T, V>(wx) || word_nonfinite<T, V>(wg);
                *(word*)(dx + (t0 - i) * p.in_step) = wx;
                *(word*)(dg + (t0 - i) * p.in_step) = wg;
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

constexpr int kForwardSteps = 16, kBackwardSteps = 8;

template <typename T, int V> cudaError_t run_forward(const mpode_recurrence_desc& d, const RecArgs& a, cudaStream_t st) {
    const Shape s = shape_of(d, 32 * V, kForwardSteps);
    return d.coupled ? launch(recurrence_forward_kernel<T, V, true, kForwardSteps>, a, s, st)
                     : launch(recurrence_forward_kernel<T, V, false, kForwardSteps>, a, s, st);
}
template <typename T, int V> cudaError_t run_backward(const mpode_recurrence_desc& d, const RecArgs& a, cudaStream_t st) {
    const Shape s = shape_of(d, 32 * V, kBackwardSteps);
    return d.coupled ? launch(recurrence_backward_kernel<T, V, true, kBackwardSteps>, a, s, st)
                     : launch(recurrence_backward_kernel<T, V, false, kBackwardSteps>, a, s, st);
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
// 32-bit words of two channels need even widths and strides and 4-byte aligned rows
bool words_fit(const mpode_recurrence_desc& d, const RecArgs& a) {
    if (d.width & 1) return false;
    if ((a.in_step | a.in_seq | a.out_step | a.out_seq) & 1) return false;
    const void* const all[] = {a.x, a.gate, a.y, a.dy, a.out, a.out2};
    for (const void* q : all)
        if (misaligned(q, 4)) return false;
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
    if (desc->low == MPODE_F32) e = run_forward<float, 1>(*desc, a, st);
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
    if (desc->low == MPODE_F32) e = run_backward<float, 1>(*desc, a, st);
    else if (desc->low == MPODE_BF16) e = words_fit(*desc, a) ? run_backward<__nv_bfloat16, 2>(*desc, a, st) : run_backward<__nv_bfloat16, 1>(*desc, a, st);
    else e = words_fit(*desc, a) ? run_backward<__half, 2>(*desc, a, st) : run_backward<__half, 1>(*desc, a, st);
    return operator_launched(e, "mpode_recurrence_backward");
}

}  // extern "C"
