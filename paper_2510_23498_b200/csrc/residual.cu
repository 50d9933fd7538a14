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
template <int N> struct RowSum {
    float part[2][kMaxBlocks * (kMaxThreads / 32)][N];
};
template <int N> __device__ __forceinline__ void row_sum(float (&v)[N], const Lane& q, RowSum<N>& s, int& set) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (q.warps * q.blocks == 1) return;
    const int lane = threadIdx.x & 31, slot = q.rank * q.warps + q.warp, slots = q.blocks * q.warps;
    if (q.blocks == 1) {
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) s.part[set][slot][i] = v[i];
        }
        __syncthreads();
    } else {
        if (lane < q.blocks) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                unsigned at;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_of(&s.part[set][slot][i])), "r"(lane));
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v[i]) : "memory");
            }
        }
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = lane < slots ? s.part[set][lane][i] : 0.f;
        if (lane + 32 < slots) v[i] += s.part[set][lane + 32][i];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    set ^= 1;
}

template <bool VEC> __device__ __forceinline__ void load_weights(const float* w, int col, int n, float (&f)[8]) {
    if (w == nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = 1.f;
    } else load8<float, VEC>(w + col, n, f);
}

// mean and 1 / deviation of a row whose elements lie in the threads' registers (zero where none exist)
__device__ __forceinline__ void row_stats(const float (&f)[8], int kind, float eps, const Lane& q, int width, RowSum<1>& s, int& set, float& mean, float& rstd) {
    mean = 0.f;
    rstd = 1.f;
    if (kind == MPODE_NORM_NONE) return;
    const float inv = 1.f / (float)width;
    if (kind == MPODE_NORM_MEANVAR) {
        float v[1] = {0.f};
#pragma unroll
        for (int i = 0; i < 8; ++i) v[0] += f[i];
        row_sum<1>(v, q, s, set);
        mean = v[0] * inv;
    }
    float v[1] = {0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float d = i < q.n ? f[i] - mean : 0.f;
        v[0] = fmaf(d, d, v[0]);
    }
    row_sum<1>(v, q, s, set);
    rstd = rsqrtf(fmaf(v[0], inv, eps));
}

// sigmoid and its slope, both without cancellation
__device__ __forceinline__ float gate_of(float g, float& slope) {
    const float e = expf(-fabsf(g)), big = __fdividef(1.f, 1.f + e), small = e * big;
    slope = small * big;
    return g < 0.f ? small : big;
}

template <typename T, bool VEC> __global__ void __launch_bounds__(kMaxThreads) residual_forward_kernel(const ResArgs p, const int blocks) {
    __shared__ RowSum<1> sums;
    const Lane q = lane_of(p.width, blocks);
    int set = 0;
    if (blocks > 1) {                                       // nobody writes into a block that has not started
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    const long long step_rows = (long long)(gridDim.x / blocks) * q.groups;
    const uint64_t seed = p.drop.threshold ? p.drop.rng[0] : 0, step = p.drop.threshold ? p.drop.rng[1] : 0;
    const int groups_row = (p.width + 7) / 8;
    for (long long row = (long long)(blockIdx.x / blocks) * q.groups + q.group; row < p.rows; row += step_rows) {
        float y[8], mean_u = 0.f, rstd_u = 1.f, mean_y, rstd_y;
        load8<float, VEC>(p.y + row * p.ld_y + q.col, q.n, y);
        if (p.u != nullptr) {
            float u[8], w[8], c[8];
            load8<T, VEC>((const T*)p.u + row * p.ld_u + q.col, q.n, u);
            float g[8];
            if (p.gate != nullptr) load8<T, VEC>((const T*)p.gate + row * p.ld_gate + q.col, q.n, g);
            row_stats(u, p.post, p.eps, q, p.width, sums, set, mean_u, rstd_u);
            load_weights<VEC>(p.w_post, q.col, q.n, w);
            load_weights<VEC>(p.scale, q.col, q.n, c);
            uint32_t keep = 0xffu;
            if (p.drop.threshold) keep = keep_bits((uint64_t)row * groups_row + q.col / 8, seed, step, p.drop.site, p.drop.threshold);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v = (u[i] - mean_u) * rstd_u * w[i], slope;
                if (p.gate != nullptr) v *= gate_of(g[i], slope);
                v *= p.h * p.drop.scale * c[i];
                if ((keep >> i) & 1u) y[i] += v;
            }
        }
        if (p.y_out != nullptr) store8<float, VEC>(p.y_out + row * p.ld_y + q.col, q.n, y);
        mean_y = 0.f; rstd_y = 1.f;
        if (p.z != nullptr) {
            float w[8];
            row_stats(y, p.pre, p.eps, q, p.width, sums, set, mean_y, rstd_y);
            load_weights<VEC>(p.w_pre, q.col, q.n, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = (y[i] - mean_y) * rstd_y * w[i];
            store8<T, VEC>((T*)p.z + row * p.ld_z + q.col, q.n, y);
        }
        if (p.stats != nullptr && q.rank == 0 && threadIdx.x == 0)
            reinterpret_cast<float4*>(p.stats)[row] = make_float4(mean_u, rstd_u, mean_y, rstd_y);
    }
    if (blocks > 1) {                                       // nobody leaves while its shared memory may be written
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}

// With n' the normalised y', n that of u, and t the cotangent of the step's term:
//   a = dy' + r' (w dz - n' mean(w dz n') - mean(w dz)),  dw_pre += dz n';   t = drop(a), dscale += h t v sig, with v = w_post n;
//   t <- h scale t, dgate = t v sig', t <- t sig, dw_post += t n, du = r (w t - n mean(w t n) - mean(w t)); the means of w dz and w t only for MEANVAR
template <typename T, bool VEC> __global__ void __launch_bounds__(kMaxThreads, 1) residual_backward_kernel(const ResArgs p, const int blocks) {
    __shared__ RowSum<2> sums;
    const Lane q = lane_of(p.width, blocks);
    int set = 0;
    if (blocks > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    const long long step_rows = (long long)(gridDim.x / blocks) * q.groups;
    const uint64_t seed = p.drop.threshold ? p.drop.rng[0] : 0, step = p.drop.threshold ? p.drop.rng[1] : 0;
    const int groups_row = (p.width + 7) / 8;
    const float inv = 1.f / (float)p.width;
    float gw_post[8], gscale[8], gw_pre[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) gw_post[i] = gscale[i] = gw_pre[i] = 0.f;
    bool bad = false;
    for (long long row = (long long)(blockIdx.x / blocks) * q.groups + q.group; row < p.rows; row += step_rows) {
        float a[8], w[8], st[4] = {0.f, 1.f, 0.f, 1.f};
        if (p.stats != nullptr) {
            const float4 f = reinterpret_cast<const float4*>(p.stats)[row];
            st[0] = f.x; st[1] = f.y; st[2] = f.z; st[3] = f.w;
        }
        float u[8], g[8];
        if (p.u != nullptr) {
            load8<T, VEC>((const T*)p.u + row * p.ld_u + q.col, q.n, u);
            if (p.gate != nullptr) load8<T, VEC>((const T*)p.gate + row * p.ld_gate + q.col, q.n, g);
        }
        if (p.dy != nullptr) load8<float, VEC>(p.dy + row * p.ld_y + q.col, q.n, a);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = 0.f;
        }
        if (p.dz != nullptr) {
            float y[8], d[8], m[2] = {0.f, 0.f};
            load8<float, VEC>(p.y + row * p.ld_y + q.col, q.n, y);
            load8<T, VEC>((const T*)p.dz + row * p.ld_z + q.col, q.n, d);
            load_weights<VEC>(p.w_pre, q.col, q.n, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[i] = (y[i] - st[2]) * st[3];
                d[i] *= p.cot_in;
                gw_pre[i] = fmaf(d[i], y[i], gw_pre[i]);
                d[i] *= w[i];
                m[0] = fmaf(d[i], y[i], m[0]);
                m[1] += d[i];
            }
            if (p.pre != MPODE_NORM_NONE) {
                row_sum<2>(m, q, sums, set);
                m[0] *= inv;
                m[1] = p.pre == MPODE_NORM_MEANVAR ? m[1] * inv : 0.f;
            } else m[0] = m[1] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] += st[3] * (d[i] - y[i] * m[0] - m[1]);
        }
        store8<float, VEC>(p.dy_out + row * p.ld_y + q.col, q.n, a);
        if (p.u != nullptr) {
            float c[8], m[2] = {0.f, 0.f};
            load_weights<VEC>(p.w_post, q.col, q.n, w);
            load_weights<VEC>(p.scale, q.col, q.n, c);
            uint32_t keep = 0xffu;
            if (p.drop.threshold) keep = keep_bits((uint64_t)row * groups_row + q.col / 8, seed, step, p.drop.site, p.drop.threshold);
            if (q.n < 8) keep &= (1u << max(q.n, 0)) - 1u;          // (columns that do not exist add nothing to the sums)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                u[i] = (u[i] - st[0]) * st[1];
                float slope = 0.f, sig = 1.f;
                if (p.gate != nullptr) sig = gate_of(g[i], slope);
                float t = (keep >> i) & 1u ? a[i] * (p.h * p.drop.scale) : 0.f;
                const float v = u[i] * w[i];
                gscale[i] = fmaf(t, v * sig, gscale[i]);
                t *= c[i];
                g[i] = t * v * slope * p.cot_out;
                t *= sig;
                gw_post[i] = fmaf(t, u[i], gw_post[i]);
                a[i] = t * w[i];
                m[0] = fmaf(a[i], u[i], m[0]);
                m[1] += a[i];
            }
            if (p.dgate != nullptr) bad |= store8<T, VEC>((T*)p.dgate + row * p.ld_gate + q.col, q.n, g);
            if (p.post != MPODE_NORM_NONE) {
                row_sum<2>(m, q, sums, set);
                m[0] *= inv;
                m[1] = p.post == MPODE_NORM_MEANVAR ? m[1] * inv : 0.f;
            } else m[0] = m[1] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = st[1] * (a[i] - u[i] * m[0] - m[1]) * p.cot_out;
            bad |= store8<T, VEC>((T*)p.du + row * p.ld_u + q.col, q.n, a);
        }
    }
    warp_flag_or(p.flag, bad);
    if (p.partial != nullptr) {
        float* out = p.partial + ((long long)(blockIdx.x / blocks) * q.groups + q.group) * 3 * p.width + q.col;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < q.n) {
                out[i] = gw_post[i];
                out[p.width + i] = gscale[i];
                out[2 * p.width + i] = gw_pre[i];
            }
    }
    if (blocks > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
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

cudaError_t launch(void (*kernel)(const ResArgs, const int), const ResArgs& a, const Shape& s, cudaStream_t st) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(s.clusters * s.blocks));
    cfg.blockDim = dim3(s.threads, s.groups);
    cfg.stream = st;
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
    if (u_dev == nullptr) a.drop.threshold = 0;
    if (!y_dev || (u_dev && !y_out_dev) || (!u_dev && !z_dev)) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_residual_forward: null pointer argument");
    if (gate_dev && !u_dev) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_residual_forward: a gate without a block output");
    if (a.drop.threshold != 0 && !rng_dev) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_residual_forward: dropout without its {seed, step}");
    a.y = y_dev; a.u = u_dev; a.gate = gate_dev; a.w_post = w_post_dev; a.scale = scale_dev; a.w_pre = w_pre_dev;
    a.y_out = y_out_dev; a.z = z_dev; a.stats = stats_dev;
    bool torn;
    const bool vec = vectors_fit(*desc, a, torn);
    if (torn) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_residual_forward: a pointer is not aligned to its elements (stats_dev: 16 bytes)");
    const Shape s = shape_of(rows, desc->width, kForwardBlocks);
    return operator_launched(with_low(desc->low, [&](auto t) {
        using T = decltype(t);
        return vec ? launch(residual_forward_kernel<T, true>, a, s, (cudaStream_t)cuda_stream)
                   : launch(residual_forward_kernel<T, false>, a, s, (cudaStream_t)cuda_stream);
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
    if (u_dev == nullptr) a.drop.threshold = 0;
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
        if (a.drop.threshold != 0 && !rng_dev) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: dropout without its {seed, step}", who);
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
            return vec ? launch(residual_backward_kernel<T, true>, a, s, st) : launch(residual_backward_kernel<T, false>, a, s, st);
        }), who);
        if (ran != MPODE_OK || !weights) return ran;
    }
    if (!weights) return MPODE_OK;
    FinishArgs f{a.partial, {dL_dw_post_dev, dL_dscale_dev, dL_dw_pre_dev}, rows > 0 ? (int)partial_rows(rows, desc->width) : 0, desc->width, accumulate};
    residual_finish_kernel<<<(3 * desc->width + 31) / 32, dim3(32, 16), 0, st>>>(f);
    return operator_launched(cudaGetLastError(), who);
}

}  // extern "C"
