// What the two directions of the residual step share: arguments, how rows lie on threads, row sums.
#pragma once
#include <atomic>

#include "cluster.cuh"
#include "operators.h"
#include "philox.cuh"
#include "rows.cuh"
#include "tensormap.h"

namespace mpode {

struct ResArgs {
    const float *y, *w_post, *scale, *w_pre;      // y: forward the state before the step, backward the one behind it
    const void *u, *gate;
    float *y_out, *stats;                         // stats [rows][4]: mean and 1 / deviation of u, then of y'
    void* z;
    // backward
    const float* dy; const void* dz;
    float* dy_out; void *du, *dgate;
    float* partial;                               // [rows of blocks][2][width]: see residual_backward.cu; null when no weight gradient is asked for
    float cot_in, cot_out;                        // 2^-e, 2^e
    unsigned* flag;
    long long ld_y, ld_u, ld_gate, ld_z;
    int rows, width, post, pre;
    float eps, h;
    Dropout drop;
};

// How rows are spread: warps of a row in a block, rows in a block, blocks of a row (a cluster), clusters
struct ResShape { int warps, groups, blocks, clusters; };
constexpr int kResWarps = 8, kResBlocks = 8, kResMaxWidth = kResWarps * 256 * kResBlocks, kResGroups = 8;

cudaError_t launch_residual_forward(mpode_dtype dt, const ResArgs& a, const ResShape& s, bool vec, bool center, cudaStream_t st);
cudaError_t launch_residual_backward(mpode_dtype dt, const ResArgs& a, const ResShape& s, bool vec, bool center, cudaStream_t st);
// clusters of `blocks` blocks that the current device holds at once, asked once for each format width
int residual_forward_room(mpode_dtype dt, int blocks);
int residual_backward_room(mpode_dtype dt, int blocks);

#ifdef __CUDACC__
__device__ __forceinline__ float2 pair(float f) { return make_float2(f, f); }

// Where a thread stands.  WARPS warps a row; one warp: eight rows a block.  CLUSTER: the row goes on in the other blocks of the cluster.
// A thread has two times four neighbouring columns, the second four half a block's columns further on, so that the lanes' accesses lie side by side (eight
// neighbouring columns a thread had twice the shared-memory cycles).
template <int WARPS, bool CLUSTER> struct Lane {
    static constexpr int kGroups = WARPS == 1 ? kResGroups : 1, kThreads = 32 * WARPS * kGroups;
    // base, cols: the block's part of a row; at: the thread's first column in it; first row and distance of the rows
    int group, warp, blocks, rank, base, cols, at, first, step;
    static constexpr int kHalf = 128 * WARPS;
    __device__ __forceinline__ Lane(int width, int blocks_) {
        const int t = threadIdx.x;
        group = WARPS == 1 ? t >> 5 : 0;
        warp = WARPS == 1 ? 0 : t >> 5;
        blocks = CLUSTER ? blocks_ : 1;
        const int cluster = CLUSTER ? (int)(blockIdx.x / blocks) : (int)blockIdx.x;
        rank = CLUSTER ? (int)(blockIdx.x - cluster * blocks) : 0;
        const int part = CLUSTER ? (width + 8 * blocks - 1) / (8 * blocks) * 8 : width;
        base = rank * part;
        cols = max(0, min(part, width - base));
        at = (WARPS == 1 ? t & 31 : t) * 4;
        first = cluster * kGroups + group;
        step = (CLUSTER ? (int)(gridDim.x / blocks) : (int)gridDim.x) * kGroups;
    }
    __device__ __forceinline__ int col(int h) const { return base + at + h * kHalf; }        // first column of the thread's quad h
    __device__ __forceinline__ int n(int h) const { return cols - at - h * kHalf; }          // columns that exist from there on, or less than one
};

// Sums over a row's threads, the same bits in all of them.  One warp: shuffles.  One block: partial sums of its warps in shared memory.  A cluster: every
// warp's into every block's shared memory.  Two sets of partial sums in turn, so that one barrier a sum does: a sum is complete only when every warp has sent,
// and each of them sends behind its own reads of the sum before, so that the set of the one before that is free.
template <int N, int WARPS, bool CLUSTER> struct RowSum {
    static constexpr int kSlots = WARPS * (CLUSTER ? kResBlocks : 1);
    struct __align__(16) Shared {
        float part[2][N][kSlots];
        unsigned long long bar[2];
    };
    Shared& s;
    unsigned round = 0;
    bool broken = false;
    __device__ __forceinline__ RowSum(Shared& shared, int blocks) : s(shared) {
        if (!CLUSTER) return;
        for (int i = threadIdx.x; i < 2 * N * kSlots; i += blockDim.x) (&s.part[0][0][0])[i] = 0.f;      // (places of blocks that do not exist)
        if (threadIdx.x == 0) sets_begin(s.bar, 2);
        cluster_arrive();                                    // nobody writes into a block that has not started
        cluster_wait();
    }
    __device__ __forceinline__ void end() {
        if (!CLUSTER) return;
        cluster_arrive();                                    // nobody leaves while its shared memory may be written
        cluster_wait();
    }
    template <int W, bool C> __device__ __forceinline__ void operator()(float (&v)[N], const Lane<W, C>& q) {
        const int lane = threadIdx.x & 31;
        if constexpr (N == 1) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
        } else {
            // both at once: the lower lanes take over the first sum, the upper ones the second
            float mine = lane < 16 ? v[0] : v[1];
            mine += __shfl_xor_sync(0xffffffffu, lane < 16 ? v[1] : v[0], 16);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
            const float other = __shfl_xor_sync(0xffffffffu, mine, 16);
            v[0] = lane < 16 ? mine : other;
            v[1] = lane < 16 ? other : mine;
        }
        if constexpr (kSlots > 1) {
            const int set = round & 1;
            if constexpr (!CLUSTER) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (lane == i) s.part[set][i][q.warp] = v[i];
                __syncthreads();
            } else {
                const unsigned bar = smem_of(&s.bar[set]);
                if (threadIdx.x == 0) set_expects(bar, q.blocks * WARPS * N * 4);
                if (lane < q.blocks) {
#pragma unroll
                    for (int i = 0; i < N; ++i) send(peer_of(smem_of(&s.part[set][i][q.rank * WARPS + q.warp]), lane), v[i], peer_of(bar, lane));
                }
                __syncwarp();
                wait_set(bar, (round >> 1) & 1, broken);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float* const f = s.part[set][i];
                if constexpr (kSlots == 2) v[i] = f[0] + f[1];
                else {
                    float2 t = make_float2(0.f, 0.f);
#pragma unroll
                    for (int k = 0; k < kSlots; k += 4) {
                        const float4 x = *reinterpret_cast<const float4*>(f + k);
                        t = __fadd2_rn(t, __fadd2_rn(make_float2(x.x, x.y), make_float2(x.z, x.w)));
                    }
                    v[i] = t.x + t.y;
                }
                if (CLUSTER && broken) v[i] = __int_as_float(0x7fffffff);
            }
            ++round;
        }
    }
};

// Where a thread reads its rows (arrays 0 .. N - 1: WIDE float32 ones, then low ones), four columns at a time and as often as it needs them.
//   VEC:  whole rows are copied to shared memory by bulk copies, kStages rows ahead; one thread of the row asks for them.
//   else: from global memory.
template <typename T, bool VEC, int WARPS, bool CLUSTER, int WIDE, int LOW> struct Rows;
template <typename T, int WARPS, bool CLUSTER, int WIDE, int LOW> struct Rows<T, true, WARPS, CLUSTER, WIDE, LOW> {
    using L = Lane<WARPS, CLUSTER>;
    static constexpr int kStages = 2, kCols = WARPS * 256, kWide = kCols * 4, kLow = kCols * (int)sizeof(T), kStage = WIDE * kWide + LOW * kLow;
    static constexpr size_t kBytes = (size_t)L::kGroups * (kStages * kStage + 16);
    unsigned mine, at_wide, at_low;      // this row's stages, the thread's columns of the first wide and the first low array in the first one
    unsigned bar, bytes_wide, bytes_low, parity = 0;
    int stage = 0;
    bool broken = false, leader;
    __device__ __forceinline__ Rows(char* smem, const L& q) {
        char* const rows = smem + q.group * kStages * kStage;
        mine = smem_of(rows);
        bar = smem_of(smem + L::kGroups * kStages * kStage) + q.group * 16;
        bytes_wide = q.cols * 4; bytes_low = q.cols * (unsigned)sizeof(T);
        at_wide = mine + q.at * 4;
        at_low = mine + WIDE * kWide + q.at * (unsigned)sizeof(T);
        leader = WARPS == 1 ? (threadIdx.x & 31) == 0 : threadIdx.x == 0;
        for (int h = 0; h < 2; ++h)
            if (q.n(h) <= 0)                         // columns that do not exist are zero
                for (int s = 0; s < kStages; ++s) {
                    const int at = q.at + h * L::kHalf;
                    for (int k = 0; k < WIDE; ++k)
                        for (int i = 0; i < 4; ++i) reinterpret_cast<float*>(rows + s * kStage + k * kWide)[at + i] = 0.f;
                    for (int k = 0; k < LOW; ++k)
                        for (int i = 0; i < 4; ++i) reinterpret_cast<T*>(rows + s * kStage + WIDE * kWide + k * kLow)[at + i] = Low<T>::from_f(0.f);
                }
        if (leader)
            for (int s = 0; s < kStages; ++s) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar + 8 * s) : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        sync();
    }
    __device__ __forceinline__ void sync() const {
        if (WARPS == 1) __syncwarp();
        else __syncthreads();
    }
    __device__ __forceinline__ void touch(const void* const (&)[WIDE + LOW]) const {}
    // by the leader, for the arrays that are there: from[k] is the row's first column of this block, or null
    __device__ __forceinline__ void request(int s, const void* const (&from)[WIDE + LOW]) {
        unsigned bytes = 0;
#pragma unroll
        for (int k = 0; k < WIDE + LOW; ++k)
            if (from[k] != nullptr) bytes += k < WIDE ? bytes_wide : bytes_low;          // (none in a block without columns)
        set_expects(bar + 8 * s, bytes);
#pragma unroll
        for (int k = 0; k < WIDE + LOW; ++k)
            if (from[k] != nullptr && bytes > 0)
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                             ::"r"(mine + s * kStage + (k < WIDE ? k * kWide : WIDE * kWide + (k - WIDE) * kLow)), "l"(from[k]),
                               "r"(k < WIDE ? bytes_wide : bytes_low), "r"(bar + 8 * s) : "memory");
    }
    __device__ __forceinline__ void wait() { wait_set(bar + 8 * stage, parity, broken); }
    __device__ __forceinline__ int slot() const { return stage; }
    __device__ __forceinline__ void done() {
        if (++stage == kStages) { stage = 0; parity ^= 1; }
    }
    template <int K> __device__ __forceinline__ Quad get(int h) const {
        Quad q;
        if constexpr (K < WIDE || sizeof(T) == 4) {
            const unsigned a = (K < WIDE ? at_wide + K * kWide : at_low + (K - WIDE) * kLow) + stage * kStage + L::kHalf * 4 * h;
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(q.v[0].x), "=f"(q.v[0].y), "=f"(q.v[1].x), "=f"(q.v[1].y) : "r"(a));
        } else {
            uint32_t x, y;
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x), "=r"(y) : "r"(at_low + (K - WIDE) * kLow + stage * kStage + L::kHalf * 2 * h));
            q.v[0] = Pair<T>::get(x);
            q.v[1] = Pair<T>::get(y);
        }
        return q;
    }
};
template <typename T, int WARPS, bool CLUSTER, int WIDE, int LOW> struct Rows<T, false, WARPS, CLUSTER, WIDE, LOW> {
    using L = Lane<WARPS, CLUSTER>;
    static constexpr int kStages = 0;
    static constexpr size_t kBytes = 0;
    const void* row[WIDE + LOW];
    int at, n;
    bool broken = false, leader = false;
    __device__ __forceinline__ Rows(char*, const L& q) : at(q.at), n(q.n(0)) {}
    __device__ __forceinline__ void sync() const {}
    // The row after this one: all its arrays are on their way to the cache at once, a row ahead of the phases that read them
    __device__ __forceinline__ void touch(const void* const (&from)[WIDE + LOW]) const {
#pragma unroll
        for (int k = 0; k < WIDE + LOW; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (from[k] != nullptr && n > L::kHalf * h)
                    asm volatile("prefetch.global.L1 [%0];" ::"l"((const char*)from[k] + (at + L::kHalf * h) * (k < WIDE ? 4 : (int)sizeof(T))));
    }
    __device__ __forceinline__ void request(int, const void* const (&from)[WIDE + LOW]) {
#pragma unroll
        for (int k = 0; k < WIDE + LOW; ++k) row[k] = from[k];
    }
    __device__ __forceinline__ void wait() {}
    __device__ __forceinline__ int slot() const { return 0; }
    __device__ __forceinline__ void done() {}
    template <int K> __device__ __forceinline__ Quad get(int h) const {
        if constexpr (K < WIDE) return load4<float, false>((const float*)row[K] + at + L::kHalf * h, n - L::kHalf * h);
        else return load4<T, false>((const T*)row[K] + at + L::kHalf * h, n - L::kHalf * h);
    }
};

// weights of the thread's columns, ones where there are none
template <bool VEC, int W, bool C> __device__ __forceinline__ Oct weights_of(const float* w, const Lane<W, C>& q) {
    Oct o;
    o.fill(w == nullptr ? 1.f : 0.f);
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (w != nullptr && q.n(h) > 0) {
            const Quad f = load4<float, VEC>(w + q.col(h), q.n(h));
            o.v[2 * h] = f.v[0];
            o.v[2 * h + 1] = f.v[1];
        }
    return o;
}
template <typename T, bool VEC, int W, bool C> __device__ __forceinline__ void store_row(T* row, const Lane<W, C>& q, const Oct& o) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (q.n(h) > 0) store4<T, VEC>(row + q.col(h), q.n(h), Quad{{o.v[2 * h], o.v[2 * h + 1]}});
}
// Which of the thread's columns dropout keeps.  Two neighbouring lanes need a half each of the same two counters' words: each works one of them out and
// gives the other lane its half.
struct KeptRow {
    uint32_t w[2][2], above;
    template <int W, bool C> __device__ __forceinline__ void draw(const Dropout& d, uint64_t first, const Lane<W, C>& q, uint64_t seed, uint64_t step) {
        const bool odd = threadIdx.x & 1;
        above = d.above;
        const Kept k(d, first + (q.col(0) + (odd ? q.kHalf : 0)) / 8, seed, step);
        const uint32_t x = __shfl_xor_sync(0xffffffffu, odd ? k.w.x : k.w.z, 1), y = __shfl_xor_sync(0xffffffffu, odd ? k.w.y : k.w.w, 1);
        w[0][0] = odd ? x : k.w.x; w[0][1] = odd ? y : k.w.y;
        w[1][0] = odd ? k.w.z : x; w[1][1] = odd ? k.w.w : y;
    }
    // element i of the thread's eight
    __device__ __forceinline__ bool operator[](int i) const {
        const uint32_t r = w[i >> 2][(i >> 1) & 1];
        return (i & 1 ? r : r << 16) > above;
    }
};

// sigmoid and its slope sig (1 - sig) = (e sig) sig with e = exp(-g), in this order: e sig is 1 - sig, where sig sig would leave float32's range below
// g = -44.  16-bit gates: the device's approximate power and reciprocal (2^-22 relative, and the argument's rounding adds |g| 2^-24).  A sigmoid below
// 2^-126 is zero there (the reciprocal has no smaller numbers); for the slope the exponent is kept at 2^127, so that e sig is then zero too.
template <typename T, bool SLOPE> __device__ __forceinline__ float2 gate_of(float2 g, float2& slope) {
    float2 e, s;
    if constexpr (sizeof(T) == 4) {
        e = make_float2(expf(-g.x), expf(-g.y));
        s = make_float2(__fdividef(1.f, 1.f + e.x), __fdividef(1.f, 1.f + e.y));
        if (SLOPE) slope = make_float2(s.x * (e.x > 1.f ? 1.f - s.x : e.x * s.x), s.y * (e.y > 1.f ? 1.f - s.y : e.y * s.y));
    } else {
        e = __fmul2_rn(g, pair(-1.4426950408889634f));
        if (SLOPE) {
            asm("min.NaN.f32 %0, %0, %1;" : "+f"(e.x) : "f"(127.f));
            asm("min.NaN.f32 %0, %0, %1;" : "+f"(e.y) : "f"(127.f));
        }
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.x));
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.y));
        const float2 d = __fadd2_rn(e, pair(1.f));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s.x) : "f"(d.x));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s.y) : "f"(d.y));
        if (SLOPE) slope = __fmul2_rn(__fmul2_rn(e, s), s);
    }
    return s;
}

#endif

inline cudaError_t launch_rows(void (*kernel)(const ResArgs, const int), const ResArgs& a, const ResShape& s, size_t smem, cudaStream_t st) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(s.clusters * s.blocks));
    cfg.blockDim = dim3(32 * s.warps * s.groups);
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
// the kernel's room, kept per device, format width and cluster size
template <typename K> int room_of(std::atomic<int> (&known)[kMaxDevices][2][kResBlocks + 1], K kernel16, K kernel32, size_t smem16, size_t smem32, mpode_dtype dt, int blocks) {
    const bool wide = dt == MPODE_F32;
    std::atomic<int>& slot = known[current_device()][wide ? 1 : 0][blocks];
    int n = slot.load(std::memory_order_relaxed);
    if (n > 0) return n - 1;
    n = clusters_at_once((const void*)(wide ? kernel32 : kernel16), dim3(32 * kResWarps), wide ? smem32 : smem16, blocks);
    if (n < 0) return 0;                                    // (asked again by the next call)
    slot.store(n + 1, std::memory_order_relaxed);
    return n;
}
// Calls f with the shape as types: f(WARPS, CLUSTER)
template <int N> struct Int { static constexpr int value = N; };
template <bool B> struct Bool { static constexpr bool value = B; };
template <typename F> cudaError_t with_shape(const ResShape& s, F&& f) {
    if (s.blocks > 1) return f(Int<8>(), Bool<true>());
    if (s.warps == 8) return f(Int<8>(), Bool<false>());
    if (s.warps == 4) return f(Int<4>(), Bool<false>());
    if (s.warps == 2) return f(Int<2>(), Bool<false>());
    return f(Int<1>(), Bool<false>());
}

}  // namespace mpode
