// One forward Euler step of the float32 state around a block that the caller evaluates, with the norms on both sides of the block:
//     n = N_post(u),  y' = y + h scale * drop(sigmoid(gate) * w_post n),  z = Q16(w_pre N_pre(y')),
// u the block's output and z the next block's input, and the step's backward pass.  N: none, v / sqrt(mean(v^2) + eps), or the same of v - mean(v).
//
// Bound by the bytes of its rows (16-bit formats: 14 an element forward, 22 backward): a row is read once, stays in registers while its sums are
// formed, and is written once.  Eight neighbouring columns a thread (16-byte accesses, one counter of the generator); a row takes one warp up to
// 256 columns and a block of up to 512 threads up to 4096, wider rows a cluster of up to four blocks whose partial sums meet in distributed
// shared memory.  All sums, statistics, gates and gradients are float32; what is stored in the low format is rounded once, when it is written.
#include "operators.h"
#include "philox.cuh"
#include "rows.cuh"

namespace mpode {
namespace {

constexpr int kMaxThreads = 512, kMaxBlocks = 4, kMaxWidth = kMaxThreads * 8 * kMaxBlocks;
constexpr int kMaxGroups = 8;             // rows in a block

struct ResArgs {
    const float *y, *w_post, *scale, *w_pre;      // y: forward the state before the step, backward the one behind it
    const void *u, *gate;
    float *y_out, *stats;                         // stats [rows][4]: mean and 1 / deviation of u, then of y'
    void* z;
    // backward
    const float* dy; const void* dz;
    float* dy_out; void *du, *dgate;
    float* partial;                               // [blocks * groups][3][width]: dw_post, dscale, dw_pre, or null when no weight gradient is asked for
    float cot_in, cot_out;                        // 2^-e, 2^e
    unsigned* flag;
    long long ld_y, ld_u, ld_gate, ld_z;
    int rows, width, post, pre;
    float eps, h;
    Dropout drop;
};

__device__ __forceinline__ unsigned smem_of(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }

// Where a thread stands: `group` of `groups` rows in the block (one warp each when there are several), first column, how many columns exist
struct Lane { int group, groups, threads, warp, warps, blocks, rank, col, n; };
__device__ __forceinline__ Lane lane_of(int width, int blocks) {
    Lane q;
    q.threads = blockDim.x; q.group = threadIdx.y; q.groups = blockDim.y;
    q.warp = threadIdx.x >> 5; q.warps = blockDim.x >> 5;
    q.blocks = blocks; q.rank = blocks > 1 ? (int)(blockIdx.x % blocks) : 0;
    q.col = (q.rank * q.threads + (int)threadIdx.x) * 8;
    q.n = min(8, width - q.col);
    return q;
}

// Sums over a row's threads, the same bits in all of them.  One warp: shuffles.  One block: partial sums of its warps in shared memory.
// A cluster: every warp's into every block's shared memory.  Two sets of partial sums in turn, so that one barrier a sum does.
constexpr int kSlots = kMaxBlocks * (kMaxThreads / 32);
template <int N> struct RowSum {
    float part[2][N][kSlots];
};
template <int N> __device__ __forceinline__ void row_sum(float (&v)[N], const Lane& q, RowSum<N>& s, int& set) {
    const int lane = threadIdx.x & 31;
    if constexpr (N == 1) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    } else {
        // both at once: the lower lanes take over the first sum, the upper ones the second
        const float give = lane < 16 ? v[1] : v[0];
        float mine = lane < 16 ? v[0] : v[1];
        mine += __shfl_xor_sync(0xffffffffu, give, 16);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
        const float other = __shfl_xor_sync(0xffffffffu, mine, 16);
        v[0] = lane < 16 ? mine : other;
        v[1] = lane < 16 ? other : mine;
    }
    if (q.warps * q.blocks == 1) return;
    const int slot = q.rank * q.warps + q.warp, slots = q.blocks * q.warps;
    if (q.blocks == 1) {
        if (lane < N) s.part[set][lane][slot] = N == 1 ? v[0] : lane == 0 ? v[0] : v[N - 1];
        __syncthreads();
    } else {
        if (lane < q.blocks) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                unsigned at;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_of(&s.part[set][i][slot])), "r"(lane));
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v[i]) : "memory");
            }
        }
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    // four at a time (the number of warps of a block is a power of two; a pair of them fills a half)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
    if (slots < 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = s.part[set][i][0] + s.part[set][i][1];
    } else {
#pragma unroll 4
        for (int k = 0; k < slots; k += 4)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float4 f = *reinterpret_cast<const float4*>(&s.part[set][i][k]);
                v[i] += (f.x + f.y) + (f.z + f.w);
            }
    }
    set ^= 1;
}

template <bool VEC> __device__ __forceinline__ void load_weights(const float* w, const Lane& q, Oct& o) {
    if (w == nullptr) o.fill(1.f);
    else load8<float, VEC>(w + q.col, q.n, o);
}
__device__ __forceinline__ float2 pair(float f) { return make_float2(f, f); }

// mean and 1 / deviation of a row whose elements lie in the threads' registers (zero where none exist)
template <bool CENTER> __device__ __forceinline__ void row_stats(const Oct& f, int kind, float eps, const Lane& q, int width, RowSum<1>& s, int& set, float& mean,
                                                                 float& rstd) {
    mean = 0.f;
    rstd = 1.f;
    if (kind == MPODE_NORM_NONE) return;
    const float inv = 1.f / (float)width;
    if (CENTER && kind == MPODE_NORM_MEANVAR) {
        float v[1] = {f.sum()};
        row_sum<1>(v, q, s, set);
        mean = v[0] * inv;
    }
    float2 sq = pair(0.f);
    const float2 less = pair(-mean);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float2 d = f.v[j];
        if (CENTER) {
            d = __fadd2_rn(d, less);
            if (2 * j >= q.n) d.x = 0.f;
            if (2 * j + 1 >= q.n) d.y = 0.f;
        }
        sq = __ffma2_rn(d, d, sq);
    }
    float v[1] = {sq.x + sq.y};
    row_sum<1>(v, q, s, set);
    rstd = rsqrtf(fmaf(v[0], inv, eps));
}

// sigmoid and its slope sig (1 - sig) = e sig^2 with e = exp(-g).  16-bit gates: the device's approximate power and reciprocal (2^-22 relative, and the
// argument's rounding adds |g| 2^-24); the exponent is kept below 2^126, so that e sig^2 is finite.
template <typename T, bool SLOPE> __device__ __forceinline__ float2 gate_of(float2 g, float2& slope) {
    float2 e, s;
    if constexpr (sizeof(T) == 4) {
        e = make_float2(expf(-g.x), expf(-g.y));
        s = make_float2(__fdividef(1.f, 1.f + e.x), __fdividef(1.f, 1.f + e.y));
        if (SLOPE) slope = make_float2(s.x * (e.x > 1.f ? 1.f - s.x : e.x * s.x), s.y * (e.y > 1.f ? 1.f - s.y : e.y * s.y));
    } else {
        e = __fmul2_rn(g, pair(-1.4426950408889634f));
        if (SLOPE) {
            asm("min.NaN.f32 %0, %0, %1;" : "+f"(e.x) : "f"(126.f));
            asm("min.NaN.f32 %0, %0, %1;" : "+f"(e.y) : "f"(126.f));
        }
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.x));
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.y));
        const float2 d = __fadd2_rn(e, pair(1.f));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s.x) : "f"(d.x));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s.y) : "f"(d.y));
        if (SLOPE) slope = __fmul2_rn(__fmul2_rn(s, s), e);
    }
    return s;
}

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// CENTER: one of the norms takes the mean away
template <typename T, bool VEC, bool CENTER> __global__ void __launch_bounds__(kMaxThreads) residual_forward_kernel(const ResArgs p, const int blocks) {
    __shared__ __align__(16) RowSum<1> sums;
    const Lane q = lane_of(p.width, blocks);
    int set = 0;
    if (blocks > 1) cluster_sync();                         // nobody writes into a block that has not started
    const long long step_rows = (long long)(gridDim.x / blocks) * q.groups;
    const uint64_t seed = p.drop.on ? p.drop.rng[0] : 0, step = p.drop.on ? p.drop.rng[1] : 0;
    const int groups_row = (p.width + 7) / 8;
    long long row = (long long)(blockIdx.x / blocks) * q.groups + q.group;
    // the next row is on its way while this one's sums meet
    Raw8<float> yr;
    Raw8<T> ur, gr;
    auto request = [&](long long r) {
        load_raw<float, VEC>(p.y + r * p.ld_y + q.col, q.n, yr);
        if (p.u != nullptr) load_raw<T, VEC>((const T*)p.u + r * p.ld_u + q.col, q.n, ur);
        if (p.gate != nullptr) load_raw<T, VEC>((const T*)p.gate + r * p.ld_gate + q.col, q.n, gr);
    };
    if (row < p.rows) request(row);
    for (; row < p.rows; row += step_rows) {
        float mean_u = 0.f, rstd_u = 1.f, mean_y = 0.f, rstd_y = 1.f;
        Oct y, u, g;
        unpack<float>(yr, y);
        if (p.u != nullptr) unpack<T>(ur, u);
        if (p.gate != nullptr) unpack<T>(gr, g);
        if (row + step_rows < p.rows) request(row + step_rows);
        if (p.u != nullptr) {
            Oct w, c;
            Kept keep;
            if (p.drop.on) keep = Kept(p.drop, (uint64_t)row * groups_row + q.col / 8, seed, step);
            row_stats<CENTER>(u, p.post, p.eps, q, p.width, sums, set, mean_u, rstd_u);
            load_weights<VEC>(p.w_post, q, w);
            load_weights<VEC>(p.scale, q, c);
            const float2 less = pair(-mean_u), r = pair(rstd_u), h = pair(p.h * p.drop.scale);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float2 v = u.v[j], slope;
                if (CENTER) v = __fadd2_rn(v, less);
                v = __fmul2_rn(__fmul2_rn(v, r), w.v[j]);
                if (p.gate != nullptr) v = __fmul2_rn(v, gate_of<T, false>(g.v[j], slope));
                const float2 k = __fmul2_rn(h, c.v[j]);
                if (p.drop.on) {
                    v = __fmul2_rn(v, k);
                    if (!keep[2 * j]) v.x = 0.f;
                    if (!keep[2 * j + 1]) v.y = 0.f;
                    y.v[j] = __fadd2_rn(y.v[j], v);
                } else y.v[j] = __ffma2_rn(v, k, y.v[j]);
            }
            if (!VEC) {                                      // columns that do not exist stay zero in the sums below
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (2 * j >= q.n) y.v[j].x = 0.f;
                    if (2 * j + 1 >= q.n) y.v[j].y = 0.f;
                }
            } else if (q.n <= 0) y.fill(0.f);
        }
        if (p.y_out != nullptr) store8<float, VEC>(p.y_out + row * p.ld_y + q.col, q.n, y);
        if (p.z != nullptr) {
            Oct w;
            row_stats<CENTER>(y, p.pre, p.eps, q, p.width, sums, set, mean_y, rstd_y);
            load_weights<VEC>(p.w_pre, q, w);
            const float2 less = pair(-mean_y), r = pair(rstd_y);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (CENTER) y.v[j] = __fadd2_rn(y.v[j], less);
                y.v[j] = __fmul2_rn(__fmul2_rn(y.v[j], r), w.v[j]);
            }
            store8<T, VEC>((T*)p.z + row * p.ld_z + q.col, q.n, y);
        }
        if (p.stats != nullptr && q.rank == 0 && threadIdx.x == 0)
            reinterpret_cast<float4*>(p.stats)[row] = make_float4(mean_u, rstd_u, mean_y, rstd_y);
    }
    if (blocks > 1) cluster_sync();                         // nobody leaves while its shared memory may be written
}

// A thread's own pieces of the rows y', dy', dz, u and gate (0 .. 4).  VEC: copied to shared memory by asynchronous copies some rows ahead; a thread reads
// what it has copied itself, so that nothing has to be waited for but its own copies.  Else loaded into registers when the row starts.
template <typename T, bool VEC> struct Rows;
template <typename T> struct Rows<T, true> {
    static constexpr int kStages = sizeof(T) == 4 ? 2 : 3, kLow = sizeof(T) / 2, kPieces = 4 + 3 * kLow;
    uint4* at;
    int threads;
    __device__ __forceinline__ void bind(char* smem, int n) {
        threads = blockDim.x * blockDim.y;
        at = reinterpret_cast<uint4*>(smem) + threadIdx.y * blockDim.x + threadIdx.x;
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
template <typename T> struct Rows<T, false> {
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
template <typename T, bool VEC, bool CENTER> __global__ void __launch_bounds__(kMaxThreads, 1) residual_backward_kernel(const ResArgs p, const int blocks) {
    constexpr int N = CENTER ? 2 : 1;
    extern __shared__ __align__(16) char staged[];
    __shared__ __align__(16) RowSum<N> sums;
    const Lane q = lane_of(p.width, blocks);
    int set = 0;
    if (blocks > 1) cluster_sync();
    const long long step_rows = (long long)(gridDim.x / blocks) * q.groups;
    const uint64_t seed = p.drop.on ? p.drop.rng[0] : 0, step = p.drop.on ? p.drop.rng[1] : 0;
    const int groups_row = (p.width + 7) / 8;
    const float inv = 1.f / (float)p.width;
    const bool exists = q.n > 0;
    Oct gw_post, gscale, gw_pre;
    gw_post.fill(0.f); gscale.fill(0.f); gw_pre.fill(0.f);
    Largest<T> largest;
    long long row = (long long)(blockIdx.x / blocks) * q.groups + q.group;
    Rows<T, VEC> in;
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
        for (int k = 0; k < in.kStages; ++k) request(row + k * step_rows, k);
    if (p.stats != nullptr && row < p.rows) stats = reinterpret_cast<const float4*>(p.stats)[row];
    int stage = 0;
    auto advance = [&]() {                                  // this row's pieces have been used: its stage is free
        if (VEC) request(row + in.kStages * step_rows, stage);
        row += step_rows;
        stage = stage + 1 < in.kStages ? stage + 1 : 0;
    };
    for (; row < p.rows; advance()) {
        const float4 st = stats;
        if (p.stats != nullptr && row + step_rows < p.rows) stats = reinterpret_cast<const float4*>(p.stats)[row + step_rows];
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
            load_weights<VEC>(p.w_pre, q, w);
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
                row_sum<N>(m, q, sums, set);
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
        if (p.u == nullptr) continue;
        Oct u, g, c;
        unpack<T>(un, u);
        if (p.gate != nullptr) unpack<T>(gn, g);
        Kept keep;
        if (p.drop.on) keep = Kept(p.drop, (uint64_t)row * groups_row + q.col / 8, seed, step);
        load_weights<VEC>(p.w_post, q, w);
        load_weights<VEC>(p.scale, q, c);
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
            row_sum<N>(m, q, sums, set);
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
    warp_flag_or(p.flag, largest.nonfinite());
    if (p.partial != nullptr) {
        float* out = p.partial + ((long long)(blockIdx.x / blocks) * q.groups + q.group) * 3 * p.width + q.col;
        store8<float, VEC>(out, q.n, gw_post);
        store8<float, VEC>(out + p.width, q.n, gscale);
        store8<float, VEC>(out + 2 * p.width, q.n, gw_pre);
    }
    if (blocks > 1) cluster_sync();
}

// out_k[c] (+)= sum over the partial rows, in a fixed order: 32 columns and 16 slices of the rows a block
struct FinishArgs { const float* partial; float* out[3]; int rows, width, accumulate; };
__global__ void __launch_bounds__(512) residual_finish_kernel(const FinishArgs p) {
    __shared__ float part[16][33];
    const int i = blockIdx.x * 32 + threadIdx.x;         // column of the three gradients side by side
    float s = 0.f;
    if (i < 3 * p.width)
        for (int r = threadIdx.y; r < p.rows; r += 16) s += p.partial[(long long)r * 3 * p.width + i];
    part[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y != 0 || i >= 3 * p.width) return;
    s = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) s += part[r][threadIdx.x];
    const int k = i / p.width;
    float* out = p.out[k];
    if (out == nullptr) return;
    out += i - k * p.width;
    *out = (p.accumulate ? *out : 0.f) + s;
}

// How rows are spread: threads of a row in a block, rows in a block, blocks of a row (a cluster), clusters
struct Shape { int threads, groups, blocks, clusters; };
Shape shape_of(int rows, int width, int clusters_at_once) {
    Shape s;
    s.blocks = 1;
    while (s.blocks * kMaxThreads * 8 < width) s.blocks *= 2;
    s.threads = 32;
    while (s.threads * s.blocks * 8 < width) s.threads *= 2;
    s.groups = s.threads == 32 ? kMaxGroups : 1;
    const int need = (rows + s.groups - 1) / s.groups;
    const int most = clusters_at_once * (s.threads <= 64 ? 4 : s.threads == 128 ? 2 : 1);
    s.clusters = (need < most ? need : most);
    s.clusters = s.blocks > 1 && s.clusters > (most + s.blocks - 1) / s.blocks ? (most + s.blocks - 1) / s.blocks : s.clusters;
    return s;
}
constexpr int kForwardBlocks = 148 * 4, kBackwardBlocks = 148 * 2;

cudaError_t launch(void (*kernel)(const ResArgs, const int), const ResArgs& a, const Shape& s, cudaStream_t st, size_t smem = 0) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(s.clusters * s.blocks));
    cfg.blockDim = dim3(s.threads, s.groups);
    cfg.stream = st;
    cfg.dynamicSmemBytes = smem;
    if (smem > 0) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)s.blocks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = s.blocks > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, a, s.blocks);
}

mpode_status check(const mpode_residual_desc* d, int rows, const char* who) {
    if (d == nullptr) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: null descriptor", who);
    if (!known_dtype(d->low)) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: unknown format %d", who, (int)d->low);
    for (int k : {(int)d->post_norm, (int)d->pre_norm})
        if (k < MPODE_NORM_NONE || k > MPODE_NORM_MEANVAR) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: unknown norm %d", who, k);
    if (d->width < 1 || rows < 0) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: %d rows of width %d", who, rows, d->width);
    if (d->width > kMaxWidth) return operator_fail(MPODE_ERR_UNSUPPORTED, "%s: width %d is above %d", who, d->width, kMaxWidth);
    if (!(d->eps > 0.f)) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: eps has to be positive", who);
    if (!(d->p_drop >= 0.f && d->p_drop <= 1.f)) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: p_drop = %g is not a probability", who, (double)d->p_drop);
    for (long long ld : {d->ld_y, d->ld_u, d->ld_gate, d->ld_z})
        if (ld != 0 && ld < d->width) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: rows overlap", who);
    return MPODE_OK;
}

ResArgs base_args(const mpode_residual_desc& d, int rows, const void* rng) {
    ResArgs a{};
    a.ld_y = d.ld_y ? d.ld_y : d.width;
    a.ld_u = d.ld_u ? d.ld_u : d.width;
    a.ld_gate = d.ld_gate ? d.ld_gate : d.width;
    a.ld_z = d.ld_z ? d.ld_z : d.width;
    a.rows = rows; a.width = d.width; a.post = d.post_norm; a.pre = d.pre_norm;
    a.eps = d.eps; a.h = d.h;
    a.drop = make_dropout(d.p_drop, rng, d.site);
    return a;
}
// 16-byte accesses everywhere?  Sets `torn` when a pointer is not even aligned to its elements.
bool vectors_fit(const mpode_residual_desc& d, const ResArgs& a, bool& torn) {
    const size_t es = low_size(d.low);
    const void* const wide[] = {a.y, a.w_post, a.scale, a.w_pre, a.y_out, a.dy, a.dy_out};
    const void* const low[] = {a.u, a.gate, a.z, a.dz, a.du, a.dgate};
    bool fit = d.width % 8 == 0 && a.ld_y % 4 == 0;
    torn = misaligned(a.stats, 16) || misaligned(a.flag, 4) || misaligned(a.drop.rng, 8);
    for (const void* p : wide) { fit = fit && !misaligned(p, 16); torn = torn || misaligned(p, 4); }
    for (const void* p : low) { fit = fit && !misaligned(p, 16); torn = torn || misaligned(p, es); }
    for (long long ld : {a.ld_u, a.ld_gate, a.ld_z}) fit = fit && (ld * es) % 16 == 0;
    return fit;
}

bool center(const mpode_residual_desc& d) { return d.post_norm == MPODE_NORM_MEANVAR || d.pre_norm == MPODE_NORM_MEANVAR; }

size_t partial_rows(int rows, int width) {
    const Shape s = shape_of(rows, width, kBackwardBlocks);
    return (size_t)s.clusters * s.groups;
}

}  // namespace
}  // namespace mpode

using namespace mpode;

extern "C" {

size_t mpode_residual_workspace_bytes(const mpode_residual_desc* desc, int rows) {
    if (check(desc, rows, "mpode_residual_workspace_bytes") != MPODE_OK || rows == 0) return 0;
    return partial_rows(rows, desc->width) * 3 * desc->width * sizeof(float);
}

mpode_status mpode_residual_forward(const mpode_residual_desc* desc, void* cuda_stream, int rows, const float* y_dev, const void* u_dev,
                                    const void* gate_dev, const float* w_post_dev, const float* scale_dev, const float* w_pre_dev,
                                    const void* rng_dev, float* y_out_dev, void* z_dev, float* stats_dev) {
    const mpode_status bad = check(desc, rows, "mpode_residual_forward");
    if (bad != MPODE_OK) return bad;
    if (rows == 0) return MPODE_OK;
    ResArgs a = base_args(*desc, rows, rng_dev);
    if (u_dev == nullptr) a.drop.on = false;
    if (!y_dev || (u_dev && !y_out_dev) || (!u_dev && !z_dev)) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_residual_forward: null pointer argument");
    if (gate_dev && !u_dev) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_residual_forward: a gate without a block output");
    if (a.drop.on && !rng_dev) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_residual_forward: dropout without its {seed, step}");
    a.y = y_dev; a.u = u_dev; a.gate = gate_dev; a.w_post = w_post_dev; a.scale = scale_dev; a.w_pre = w_pre_dev;
    a.y_out = y_out_dev; a.z = z_dev; a.stats = stats_dev;
    bool torn;
    const bool vec = vectors_fit(*desc, a, torn);
    if (torn) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_residual_forward: a pointer is not aligned to its elements (stats_dev: 16 bytes)");
    const Shape s = shape_of(rows, desc->width, kForwardBlocks);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    return operator_launched(with_low(desc->low, [&](auto t) {
        using T = decltype(t);
        if (center(*desc)) return vec ? launch(residual_forward_kernel<T, true, true>, a, s, st) : launch(residual_forward_kernel<T, false, true>, a, s, st);
        return vec ? launch(residual_forward_kernel<T, true, false>, a, s, st) : launch(residual_forward_kernel<T, false, false>, a, s, st);
    }), "mpode_residual_forward");
}

mpode_status mpode_residual_backward(const mpode_residual_desc* desc, void* cuda_stream, int rows, const float* y_new_dev, const void* u_dev,
                                     const void* gate_dev, const float* w_post_dev, const float* scale_dev, const float* w_pre_dev,
                                     const void* rng_dev, const float* stats_dev, const float* dL_dy_new_dev, const void* dL_dz_dev, int scale_exp,
                                     float* dL_dy_dev, void* dL_du_dev, void* dL_dgate_dev, float* dL_dw_post_dev, float* dL_dscale_dev,
                                     float* dL_dw_pre_dev, int accumulate, unsigned* flag_dev, void* workspace_dev, size_t workspace_bytes) {
    const char* const who = "mpode_residual_backward";
    const mpode_status bad = check(desc, rows, who);
    if (bad != MPODE_OK) return bad;
    if (scale_exp < -100 || scale_exp > 100) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: scale exponent %d", who, scale_exp);
    ResArgs a = base_args(*desc, rows, rng_dev);
    if (u_dev == nullptr) a.drop.on = false;
    a.y = y_new_dev; a.u = u_dev; a.gate = gate_dev; a.w_post = w_post_dev; a.scale = scale_dev; a.w_pre = w_pre_dev;
    a.stats = const_cast<float*>(stats_dev);
    a.dy = dL_dy_new_dev; a.dz = dL_dz_dev; a.dy_out = dL_dy_dev; a.du = dL_du_dev; a.dgate = dL_dgate_dev;
    a.cot_in = ldexpf(1.f, -scale_exp); a.cot_out = ldexpf(1.f, scale_exp);
    a.flag = flag_dev;
    const bool weights = dL_dw_post_dev || dL_dscale_dev || dL_dw_pre_dev;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    if (rows > 0) {
        if (!dL_dy_dev || (dL_dz_dev && !y_new_dev) || (u_dev && !dL_du_dev) || (gate_dev && !dL_dgate_dev))
            return operator_fail(MPODE_ERR_INVALID_ARG, "%s: null pointer argument", who);
        if (!u_dev && (gate_dev || dL_du_dev)) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: a gate or a cotangent without a block output", who);
        if (dL_dgate_dev && !gate_dev) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: a cotangent for a gate that is not there", who);
        if (!stats_dev && ((u_dev && desc->post_norm != MPODE_NORM_NONE) || (dL_dz_dev && desc->pre_norm != MPODE_NORM_NONE)))
            return operator_fail(MPODE_ERR_INVALID_ARG, "%s: norms need the forward pass's statistics", who);
        if (a.drop.on && !rng_dev) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: dropout without its {seed, step}", who);
        bool torn;
        const bool vec = vectors_fit(*desc, a, torn);
        torn = torn || misaligned(dL_dw_post_dev, 4) || misaligned(dL_dscale_dev, 4) || misaligned(dL_dw_pre_dev, 4);
        if (torn) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: a pointer is not aligned to its elements (stats_dev: 16 bytes)", who);
        if (weights) {
            if (!workspace_dev) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: weight gradients need a workspace", who);
            if (misaligned(workspace_dev, 256)) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: misaligned workspace", who);
            if (workspace_bytes < mpode_residual_workspace_bytes(desc, rows)) return operator_fail(MPODE_ERR_WORKSPACE_TOO_SMALL, "%s: workspace too small", who);
            a.partial = (float*)workspace_dev;
        }
        const Shape s = shape_of(rows, desc->width, kBackwardBlocks);
        const mpode_status ran = operator_launched(with_low(desc->low, [&](auto t) {
            using T = decltype(t);
            using R = Rows<T, true>;
            const size_t smem = (size_t)s.threads * s.groups * R::kStages * R::kPieces * 16;
            if (center(*desc)) return vec ? launch(residual_backward_kernel<T, true, true>, a, s, st, smem) : launch(residual_backward_kernel<T, false, true>, a, s, st);
            return vec ? launch(residual_backward_kernel<T, true, false>, a, s, st, smem) : launch(residual_backward_kernel<T, false, false>, a, s, st);
        }), who);
        if (ran != MPODE_OK || !weights) return ran;
    }
    if (!weights) return MPODE_OK;
    FinishArgs f{a.partial, {dL_dw_post_dev, dL_dscale_dev, dL_dw_pre_dev}, rows > 0 ? (int)partial_rows(rows, desc->width) : 0, desc->width, accumulate};
    residual_finish_kernel<<<(3 * desc->width + 31) / 32, dim3(32, 16), 0, st>>>(f);
    return operator_launched(cudaGetLastError(), who);
}

}  // extern "C"
