// Gated linear recurrence along a sequence, forward and backward: the time loop of a linear relaxation equation as a scan.
//
// With b = sigmoid(g) and a = 1 - b, per channel: y_i = a y_{i-1} + b x_i (coupled: one implicit Euler step of y' = lambda (x - y),
// g = log(h lambda)) or y_i = a y_{i-1} + x_i.  Backward: l_i = dy_i + r_i, r_{i-1} = a_i l_i, from r behind the last step; coupled dx = b l,
// dg = l (x - y_{i-1}) a b, else dx = l, dg = -l y_{i-1} a b.
//
// Every step is an affine map y -> A y + u.  A block holds 32 lanes of channels, two each, and some warps along the time axis; a warp's steps of a round
// lie in its registers or its part of shared memory.  First each warp composes its own steps, then the warps' maps are exchanged, and every warp runs its
// steps again from the state in front of them: the data is read once and written once, and nothing is kept in device memory.  Where a batch has too few
// channels for the GPU, the blocks of a cluster share a sequence and exchange their maps through distributed shared memory; one more warp of each block does
// that while the others are at the next round's first half.
//
// Precision: b is formed with a relative error (no cancellation for g << 0), and every decay is written y - b y in one rounding, so that memories of
// a million steps (b = 1e-6) decay at the right rate, where a rounded a = 1 - b would not, and b = 1 forgets everything, exactly.  For the same reason a
// composed map is kept as y -> y - C y + u with C = 1 - A.
#include <stdarg.h>
#include <stddef.h>
#include <stdio.h>

#include <math.h>

#include <atomic>

#include <type_traits>

#include "cluster.cuh"
#include "operators.h"
#include "recurrence_tiles.h"
#include "rows.cuh"
#include "tensormap.h"

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
    int stages;                        // STAGED, PIPED: rounds in shared memory
    int zero_behind;                   // what lies behind a sequence's length is set to zero
    int time_major;                    // STAGED: the maps' coordinates are (channel, sequence, step) instead of (channel, step, sequence)
};
// STAGED: tensor maps of gate and x (forward), of gate, dL/dy, y and x (backward)
struct RecMaps { CUtensorMap m[4]; };

constexpr int V = 2;                   // channels of a lane
// Two channels of a row: a pair of 16-bit values in 32 bits, or of float32
template <typename T> struct Word {
    using type = uint32_t;
    static __device__ __forceinline__ void get(type w, float (&f)[2]) { const float2 t = Pair<T>::get(w); f[0] = t.x; f[1] = t.y; }
    static __device__ __forceinline__ type put(const float (&f)[2]) { return Pair<T>::put(f[0], f[1]); }
    static __device__ __forceinline__ type negate(type w) { return w ^ 0x80008000u; }
};
template <> struct Word<float> {
    using type = float2;
    static __device__ __forceinline__ void get(type w, float (&f)[2]) { f[0] = w.x; f[1] = w.y; }
    static __device__ __forceinline__ type put(const float (&f)[2]) { return make_float2(f[0], f[1]); }
    static __device__ __forceinline__ type negate(type w) { return make_float2(-w.x, -w.y); }
};
template <typename T> __device__ __forceinline__ void see(Largest<T>& m, const typename Word<T>::type& w) {
    if constexpr (sizeof(T) == 2) m.see(w);
    else { m.see(__float_as_uint(w.x)); m.see(__float_as_uint(w.y)); }
}

// a b + c, a + b and a b on a lane's channels, one instruction each
struct Ops {
    static __device__ __forceinline__ void fma(float (&d)[V], const float (&a)[V], const float (&b)[V], const float (&c)[V]) {
        const float2 r = __ffma2_rn(make_float2(a[0], a[1]), make_float2(b[0], b[1]), make_float2(c[0], c[1]));
        d[0] = r.x; d[1] = r.y;
    }
    static __device__ __forceinline__ void add(float (&d)[V], const float (&a)[V], const float (&b)[V]) {
        const float2 r = __fadd2_rn(make_float2(a[0], a[1]), make_float2(b[0], b[1]));
        d[0] = r.x; d[1] = r.y;
    }
    static __device__ __forceinline__ void mul(float (&d)[V], const float (&a)[V], const float (&b)[V]) {
        const float2 r = __fmul2_rn(make_float2(a[0], a[1]), make_float2(b[0], b[1]));
        d[0] = r.x; d[1] = r.y;
    }
};

// -sigmoid(g) = -b, and the slope b (1 - b), which is (e b) b with e = exp(-g), in this order: e b is 1 - b, where b b would leave float32's range below
// g = -44.  16-bit gates: the device's approximate power and quotient (2^-22 relative, and the argument's rounding adds |g| 2^-24), which cost 3 instructions
// a channel where the accurate ones of float32 cost 15.  A b below 2^-126 is zero there (the quotient has no smaller numbers); for the slope the exponent
// is kept at 2^127, so that e b is then zero too.
template <typename T, bool SLOPE> __device__ __forceinline__ void negated_gate(const float (&g)[V], float (&nb)[V], float (&slope)[V]) {
    float e[V];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            e[v] = expf(-g[v]);
            const float b = __fdividef(1.f, 1.f + e[v]);
            nb[v] = -b;
            if (SLOPE) slope[v] = b * (e[v] > 1.f ? 1.f - b : e[v] * b);
        }
    } else {
        float k[V], d[V];
#pragma unroll
        for (int v = 0; v < V; ++v) k[v] = -1.4426950408889634f;
        Ops::mul(e, g, k);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (SLOPE) asm("min.NaN.f32 %0, %0, %1;" : "+f"(e[v]) : "f"(127.f));
            asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e[v]));
            k[v] = -1.f;
        }
        Ops::fma(d, e, k, k);
#pragma unroll
        for (int v = 0; v < V; ++v) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(nb[v]) : "f"(d[v]));
        if (SLOPE) {
            Ops::mul(slope, e, nb);
            Ops::mul(slope, slope, nb);
        }
    }
}

// -b of a step that does not exist, and 1 - A of the identity map, negative: s + kKeep s is s for every float32 number in one rounding, and infinity for an
// infinite s, where 0 s would be a NaN
constexpr float kKeep = 1.17549435e-38f;

// One step of the state s, nb = -b.  The coupled forward pass runs on s = -y, where b x is taken away without a change of sign: s - b s - b x.
template <bool COUPLED> __device__ __forceinline__ void step_forward(float (&s)[V], const float (&nb)[V], const float (&x)[V]) {
    float kept[V];
    Ops::fma(kept, nb, s, s);
    if constexpr (COUPLED) Ops::fma(s, nb, x, kept);
    else Ops::add(s, kept, x);
}
// The composed map s -> A s + u of some steps, C = 1 - A: A exact to its last bits where it is small (a reset leaves A = 0), C where the steps
// forget little.  Kept per lane as A, -C and u.
struct Map {
    float A[V], nC[V], u[V];
    __device__ __forceinline__ Map() {
#pragma unroll
        for (int v = 0; v < V; ++v) { A[v] = 1.f; nC[v] = kKeep; u[v] = 0.f; }
    }
    __device__ __forceinline__ void decay(const float (&nb)[V]) {
        float one[V], left[V];
#pragma unroll
        for (int v = 0; v < V; ++v) one[v] = 1.f;
        Ops::fma(A, nb, A, A);
        Ops::add(left, one, nC);
        Ops::fma(nC, nb, left, nC);
    }
};
// As the warps and blocks exchange it: s -> m s + (k s + u), with (m, k) = (A, 0) or (-C, 1), whichever is the smaller one
struct Affine {
    float m[V], k[V], u[V];
    __device__ __forceinline__ void from(const Map& p) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const bool fast = p.A[v] < 0.5f;
            m[v] = fast ? p.A[v] : p.nC[v]; k[v] = fast ? 0.f : 1.f; u[v] = p.u[v];
        }
    }
    __device__ __forceinline__ void apply(float (&s)[V]) const {
        float t[V];
        Ops::fma(t, k, s, u);
        Ops::fma(s, m, s, t);
    }
    // p, then this map
    __device__ __forceinline__ void follow(Map& p) const {
        float t[V], one[V], k1[V];
#pragma unroll
        for (int v = 0; v < V; ++v) { one[v] = 1.f; k1[v] = k[v] - 1.f; }
        Ops::mul(t, k, p.A);
        Ops::fma(p.A, m, p.A, t);
        Ops::add(t, one, p.nC);
        Ops::fma(p.nC, k, p.nC, k1);              // -C - c (1 - C) with c = -m, or 1 - m: -1 + m (1 - C)
        Ops::fma(p.nC, m, t, p.nC);
        apply(p.u);
    }
};

constexpr int kMaxWarps = 8, kPipedWarps = 11, kMaxCluster = 16;

// Shared memory of the exchange inside a block or a cluster: maps of the block's warps and of the cluster's blocks, two sets in turn.  Places of warps and
// blocks that do not exist hold the identity, so that the loops over them have fixed lengths and their loads go ahead of the arithmetic.
// A set is written again two rounds later: a block sends its map of round k + 1 when it has those of round k from all blocks, and each of them sends behind a
// barrier of its warps, which have then read those of round k - 1.
struct __align__(16) Exchange {
    float warp[2][kMaxWarps][3][32 * V];
    unsigned long long bytes[2];                // counts the bytes of a set's block maps
    float block[2][kMaxCluster][3][32 * V];     // (not there where the kernel is launched without clusters)
};
constexpr size_t kBlockExchange = offsetof(Exchange, block);
// The same with a warp that scans: also the states in front of the warps' steps, and barriers that count the warps' maps and the states.  A warp writes its
// map of round k + 2 behind its second half of round k, for which the maps of round k had been read; states of round k + 2 are written when all maps of
// it are there, behind the reads of round k's.
struct __align__(16) Scan {
    float warp[2][kPipedWarps][3][32 * V];
    float block[2][kMaxCluster][3][32 * V];
    float start[2][kPipedWarps][32 * V];
    unsigned long long maps[2], bytes[2], starts[2];
};
__device__ __forceinline__ void lds(float (&f)[V], const float* p) {
    const float2 t = *reinterpret_cast<const float2*>(p);
    f[0] = t.x; f[1] = t.y;
}
__device__ __forceinline__ void sts(float* p, const float (&f)[V]) {
    *reinterpret_cast<float2*>(p) = make_float2(f[0], f[1]);
}
__device__ __forceinline__ void fetch(Affine& a, const float (&t)[3][32 * V]) {
    lds(a.m, &t[0][threadIdx.x * V]); lds(a.k, &t[1][threadIdx.x * V]); lds(a.u, &t[2][threadIdx.x * V]);
}
__device__ __forceinline__ void put(float (&t)[3][32 * V], const Affine& a) {
    sts(&t[0][threadIdx.x * V], a.m); sts(&t[1][threadIdx.x * V], a.k); sts(&t[2][threadIdx.x * V], a.u);
}

__device__ __forceinline__ void exchange_begin(Exchange& ex, int warps, int blocks) {
    Affine id;
#pragma unroll
    for (int v = 0; v < V; ++v) { id.m[v] = kKeep; id.k[v] = 1.f; id.u[v] = 0.f; }
    for (int set = 0; set < 2; ++set) {
        for (int w = warps + threadIdx.y; w < kMaxWarps; w += warps) put(ex.warp[set][w], id);
        if (blocks > 1)
            for (int r = blocks + threadIdx.y; r < kMaxCluster; r += warps) put(ex.block[set][r], id);
    }
    if (blocks == 1) return;
    if (threadIdx.x == 0 && threadIdx.y == 0) sets_begin(ex.bytes, 2);
    cluster_arrive();                       // nobody writes into a block that has not started
}
// A round's exchange has two halves.  publish: this warp's map to the block, the block's map to every block of the cluster; returns the map of the steps of the
// block that lie in front of this warp's.  collect: from the state in front of all of the round's steps (`carry`, replaced by the one behind them) the
// state in front of this warp's.  Called by all threads of the cluster in the same order.
__device__ __forceinline__ void publish(Exchange& ex, unsigned round, const Map& own, Affine& before, int blocks, int rank) {
    const int warp = threadIdx.y, set = round & 1;
    Affine a;
    a.from(own);
    put(ex.warp[round & 1][warp], a);
    __syncthreads();
    if (blocks == 1) return;
    const unsigned bar = smem_of(&ex.bytes[set]);
    if (warp == 0 && threadIdx.x == 0) set_expects(bar, blocks * 3 * 32 * V * 4);
    Map all;
#pragma unroll
    for (int w = 0; w < kMaxWarps; ++w) {
        if (w == warp) before.from(all);
        fetch(a, ex.warp[round & 1][w]);
        a.follow(all);
    }
    a.from(all);
    const unsigned at = smem_of(&ex.block[set][rank][0][threadIdx.x * V]);
    for (int to = warp; to < blocks; to += (int)blockDim.y) {               // a warp to each block
        const unsigned there = peer_of(at, to), count = peer_of(bar, to);
        send(there, a.m[0], a.m[1], count);
        send(there + 32 * V * 4, a.k[0], a.k[1], count);
        send(there + 64 * V * 4, a.u[0], a.u[1], count);
    }
}
__device__ __forceinline__ void collect(Exchange& ex, unsigned round, const Affine& before, float (&carry)[V], float (&start)[V],
                                                                   int blocks, int rank, bool& broken) {
    const int warp = threadIdx.y, set = round & 1;
    Affine a;
    if (blocks == 1) {
#pragma unroll
        for (int w = 0; w < kMaxWarps; ++w) {
            if (w == warp) {
#pragma unroll
                for (int v = 0; v < V; ++v) start[v] = carry[v];
            }
            fetch(a, ex.warp[round & 1][w]);
            a.apply(carry);
        }
        return;
    }
    wait_set(smem_of(&ex.bytes[set]), (round >> 1) & 1, broken);
    if (broken) {
#pragma unroll
        for (int v = 0; v < V; ++v) carry[v] = __int_as_float(0x7fffffff);
    }
    for (int r0 = 0; r0 < blocks; r0 += 4) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (r0 + r == rank) {
#pragma unroll
                for (int v = 0; v < V; ++v) start[v] = carry[v];
            }
            fetch(a, ex.block[set][r0 + r]);
            a.apply(carry);
        }
    }
    before.apply(start);
}

__device__ __forceinline__ void exchange_begin(Scan& ex, int warps, int) {
    if (threadIdx.x == 0 && threadIdx.y == 0) {
        for (int i = 0; i < 2; ++i) {
            bar_init(&ex.maps[i], warps);
            bar_init(&ex.starts[i], 1);
        }
        sets_begin(ex.bytes, 2);
    }
    __syncthreads();
    cluster_arrive();
}
// a warp's map of a round, and the state in front of its steps
__device__ __forceinline__ void publish(Scan& ex, unsigned round, const Map& own) {
    const int set = round & 1;
    Affine a;
    a.from(own);
    put(ex.warp[set][threadIdx.y], a);
    __syncwarp();
    if (threadIdx.x == 0) bar_arrive(smem_of(&ex.maps[set]));
}
__device__ __forceinline__ void collect(Scan& ex, unsigned round, float (&start)[V], bool& broken) {
    const int set = round & 1;
    wait_set(smem_of(&ex.starts[set]), (round >> 1) & 1, broken);
    lds(start, &ex.start[set][threadIdx.y][threadIdx.x * V]);
    if (broken) {
#pragma unroll
        for (int v = 0; v < V; ++v) start[v] = __int_as_float(0x7fffffff);
    }
}
// The warp between them: `carry` is the state in front of the first round, and then the one behind the last
__device__ __forceinline__ void scan(Scan& ex, unsigned base, unsigned stride, unsigned end, float (&carry)[V], int warps, int blocks, int rank) {
    bool broken = false;
    for (unsigned round = 0; base < end; base += stride, ++round) {
        const int set = round & 1;
        const unsigned parity = (round >> 1) & 1;
        Affine a;
        wait_set(smem_of(&ex.maps[set]), parity, broken);
        float state[V];
        Map all;
#pragma unroll 4
        for (int w = 0; w < warps; ++w) {
            fetch(a, ex.warp[set][w]);
            a.follow(all);
        }
        a.from(all);
        const unsigned at = smem_of(&ex.block[set][rank][0][threadIdx.x * V]), bar = smem_of(&ex.bytes[set]);
        if (threadIdx.x == 0) set_expects(bar, blocks * 3 * 32 * V * 4);
        for (int to = 0; to < blocks; ++to) {
            const unsigned there = peer_of(at, to), count = peer_of(bar, to);
            send(there, a.m[0], a.m[1], count);
            send(there + 32 * V * 4, a.k[0], a.k[1], count);
            send(there + 64 * V * 4, a.u[0], a.u[1], count);
        }
        wait_set(bar, parity, broken);
#pragma unroll 4
        for (int r = 0; r < blocks; ++r) {
            if (r == rank) {
#pragma unroll
                for (int v = 0; v < V; ++v) state[v] = carry[v];
            }
            fetch(a, ex.block[set][r]);
            a.apply(carry);
        }
        if (broken) {
#pragma unroll
            for (int v = 0; v < V; ++v) state[v] = carry[v] = __int_as_float(0x7fffffff);
        }
#pragma unroll 4
        for (int w = 0; w < warps; ++w) {
            sts(&ex.start[set][w][threadIdx.x * V], state);
            fetch(a, ex.warp[set][w]);
            a.apply(state);
        }
        __syncwarp();
        if (threadIdx.x == 0) bar_arrive(smem_of(&ex.starts[set]));
    }
}

// How rows are read and written
enum Access : int {
    STAGED = 0,     // rows of multiples of 16 bytes from aligned pointers: bulk tensor copies to shared memory, neighbouring channels a lane
    PAIRS = 1,      // even widths and strides, pointers aligned to two elements: neighbouring channels a lane, one access
    SINGLES = 2,    // anything: channels 32 apart a lane, an access each
    PIPED = 3       // STAGED, in clusters: a round's maps are on their way while those of the one before are waited for
};
__host__ __device__ constexpr bool staged_rows(int access) { return access == STAGED || access == PIPED; }
__host__ __device__ constexpr int most_warps(int access) { return access == PIPED ? kPipedWarps : kMaxWarps; }
// Which channels and steps a thread works on.  Channels behind the last one are the last one again (the last pair), and the same values go to the same
// places: a condition at each store costs more than the rest of the second run (1320 cycles a round of 16 steps instead of 520).
struct Place { int seq, tile, lane, col[2], len, rank; unsigned slot; };      // tile: the first channel of the warp
template <int ACCESS> __device__ __forceinline__ Place place(const RecArgs& p, int blocks, int warps) {
    const int tiles = (p.width + 63) / 64, tile = blockIdx.x / blocks;
    Place q;
    q.rank = blockIdx.x - tile * blocks;
    q.seq = tile / tiles;
    q.tile = (tile - q.seq * tiles) * 64;
    if (ACCESS == SINGLES) {
        q.lane = threadIdx.x;
        q.col[0] = min(q.tile + (int)threadIdx.x, p.width - 1);
        q.col[1] = min(q.tile + (int)threadIdx.x + 32, p.width - 1);
    } else {
        q.lane = min((int)threadIdx.x, (p.width - q.tile) / 2 - 1);
        q.col[0] = q.tile + 2 * q.lane;
        q.col[1] = q.col[0] + 1;
    }
    q.len = p.n_steps;
    if (p.lengths != nullptr) q.len = min(max(p.lengths[q.seq], 0), p.n_steps);
    q.slot = q.rank * warps + threadIdx.y;
    return q;
}
// a lane's two channels of the row at base + off; apart: bytes from one to the other (SINGLES)
template <typename T, int ACCESS> __device__ __forceinline__ typename Word<T>::type load_pair(const char* base, unsigned off, unsigned apart) {
    using word = typename Word<T>::type;
    if constexpr (ACCESS != SINGLES) return *(const word*)(base + off);
    else if constexpr (sizeof(T) == 4) return make_float2(*(const float*)(base + off), *(const float*)(base + off + apart));
    else return (uint32_t)*(const uint16_t*)(base + off) | (uint32_t)*(const uint16_t*)(base + off + apart) << 16;
}
template <typename T, int ACCESS> __device__ __forceinline__ void store_pair(char* base, unsigned off, unsigned apart, typename Word<T>::type w) {
    using word = typename Word<T>::type;
    if constexpr (ACCESS != SINGLES) *(word*)(base + off) = w;
    else if constexpr (sizeof(T) == 4) {
        *(float*)(base + off) = w.x;
        *(float*)(base + off + apart) = w.y;
    } else {
        *(uint16_t*)(base + off) = (uint16_t)w;
        *(uint16_t*)(base + off + apart) = (uint16_t)(w >> 16);
    }
}

// A round in which every step of every warp exists, one in which that has to be asked at each step, or it is not known which of the two
enum Round : int { GUARDED = 0, WHOLE = 1, EITHER = 2 };
template <int R> struct Kind { static constexpr int value = R; };
template <bool B> struct Flag { static constexpr bool value = B; };
template <typename K, typename F> __device__ __forceinline__ void of_kind(K, bool whole, F&& run) {
    if constexpr (K::value == WHOLE) run(Flag<true>());
    else if constexpr (K::value == GUARDED) run(Flag<false>());
    else if (whole) run(Flag<true>());
    else run(Flag<false>());
}
// The rounds from `base` to `end`: both halves of each in turn (whole ones in a loop of their own), or the first half of the next one in front of the second
// half of this one
template <bool PIPED_ROUNDS, typename Turn, typename Whole, typename First, typename Second>
__device__ __forceinline__ void rounds(unsigned base, unsigned stride, unsigned end, Whole&& whole, First& first, Second& second) {
    unsigned round = 0;
    if constexpr (!PIPED_ROUNDS) {
        const auto one = [&](auto kind) {
            Turn a;
            first(kind, a, base, round++);
            second(kind, a);
            base += stride;
        };
        while (base < end && !whole(base)) one(Kind<GUARDED>());
        while (base < end && whole(base)) one(Kind<WHOLE>());
        while (base < end) one(Kind<GUARDED>());
    } else {
        const Kind<EITHER> kind;
        if (base >= end) return;
        Turn a, b;
        first(kind, a, base, round++);
        while (true) {
            base += stride;
            if (base >= end) { second(kind, a); return; }
            first(kind, b, base, round++);
            second(kind, a);
            base += stride;
            if (base >= end) { second(kind, b); return; }
            first(kind, a, base, round++);
            second(kind, b);
        }
    }
}

// Asks for rows that a warp is going to read: N arrays of L rows, `bytes` bytes of each (64 channels at most) from at(array, row) on, null for one that is not
// there.  A request a cache line; one for each sector, to the nearest cache, costs more than it saves (37 x 1000 x 785 float16 backward 125 us instead of 115,
// without requests 127).
template <typename T, int L, int N, typename At> __device__ __forceinline__ void touch_rows(int bytes, At&& at) {
    constexpr int S = sizeof(T) == 4 ? 3 : 2;               // lines of 128 bytes that 64 channels reach into
#pragma unroll
    for (int j = 0; j < N * L * S; j += 32) {
        const int r = (j + threadIdx.x) / S, line = j + threadIdx.x - r * S;
        const char* const p = r < N * L ? at(r / L, r % L) : nullptr;
        if (p != nullptr) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + min(128 * line, bytes - 1)));
    }
}

// Where a warp finds its steps: a tile of N arrays, L steps of two channels a lane.
//   STAGED, PIPED: brought to shared memory two or three rounds ahead (each warp its own stages and barriers, so that no other warp has to be waited for), read from there
//           as often as needed.  (Asynchronous copies of 16 bytes a lane in their place took 320 cycles a round of 2200 for issuing them.)  A tile that reaches
//           behind its sequence's length, one a warp at most, comes as asynchronous copies of a lane's two channels, row by row.
//   else:   loaded into registers when the round starts, from the cache, for which the lanes have asked for its rows a round ahead.
template <typename T> constexpr int kRowBytes = 32 * V * (int)sizeof(T);
constexpr int kMaxStages = 3;
template <typename T, int L, int N> constexpr int kStageBytes = N * L * kRowBytes<T>;      // of a warp
template <typename T, int L, int N, int ACCESS, bool SHARED = staged_rows(ACCESS)> struct Tile {
    using word = typename Word<T>::type;
    word w[N][L];
    unsigned apart;
    // step i of array k lies at base + off + i * step bytes; steps lo .. hi - 1 exist (FULL: all)
    template <bool FULL> __device__ __forceinline__ void load(int k, const char* base, unsigned off, unsigned step, int lo, int hi) {
#pragma unroll
        for (int i = 0; i < L; ++i, off += step) {
            if (!FULL) w[k][i] = word{};
            if (FULL || (i >= lo && i < hi)) w[k][i] = load_pair<T, ACCESS>(base, off, apart);
        }
    }
    __device__ __forceinline__ word get(int, int k, int i) const { return w[k][i]; }
};
// (a call, because it is rare: in line it cost every round of the piped kernel 4 %; a tile that is read when its turn has come cost 37 x 1000 x 784 46 us instead of 41)
template <int BYTES> __device__ __noinline__ void copy_rows(unsigned to, unsigned pitch, const char* from, long long step, int count) {
    for (; count > 0; --count, to += pitch, from += step) asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}
template <typename T, int L, int N, int ACCESS> struct Tile<T, L, N, ACCESS, true> {
    using word = typename Word<T>::type;
    static constexpr int kRow = kRowBytes<T>, kArray = L * kRow;
    unsigned at, lane, bar, next = 0, parity = 0, count;
    __device__ __forceinline__ void bind(char* smem, unsigned long long* bars, int l, int stages) {
        count = stages;
        at = smem_of(smem) + threadIdx.y * stages * kStageBytes<T, L, N>;
        bar = smem_of(bars) + threadIdx.y * (kMaxStages * 8);
        lane = at + l * (unsigned)sizeof(word);
        if (threadIdx.x == 0) {
            sets_begin(bars + threadIdx.y * kMaxStages, stages);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncwarp();
    }
    // one lane: L steps of `arrays` arrays from step t0[k] on, upwards; what lies outside is filled with zeros
    __device__ __forceinline__ void request(int stage, const RecMaps& maps, unsigned mask, int tile, int seq, bool time_major, int t0, int t0_y) {
        set_expects(bar + 8 * stage, __popc(mask) * kArray);
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (mask >> k & 1) {
                const int t = k == 2 ? t0_y : t0;
                asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                             ::"r"(at + (stage * N + k) * kArray), "l"(reinterpret_cast<unsigned long long>(&maps.m[k])), "r"(bar + 8 * stage), "r"(tile),
                               "r"(time_major ? seq : t), "r"(time_major ? t : seq) : "memory");
            }
    }
    // all lanes: `count` rows of array k from row lo of the tile on, which lies at `from`; then, when all are under way, that there are no more
    __device__ __forceinline__ void request_rows(int stage, int k, int lo, int count, const char* from, long long step) const {
        copy_rows<sizeof(word)>(lane + (stage * N + k) * kArray + lo * kRow, kRow, from, step, count);
    }
    __device__ __forceinline__ void rows_requested(int stage) const {
        asm volatile("cp.async.mbarrier.arrive.shared.b64 [%0];" ::"r"(bar + 8 * stage) : "memory");      // (holds the phase open until this lane's are there)
        __syncwarp();
        if (threadIdx.x == 0) bar_arrive(bar + 8 * stage);
    }
    // the next round's stage, once it is there
    __device__ __forceinline__ int wait(bool& broken) {
        const int stage = next;
        wait_set(bar + 8 * stage, parity, broken);
        if (++next == count) { next = 0; parity ^= 1; }
        return stage;
    }
    __device__ __forceinline__ word get(int stage, int k, int i) const {
        const unsigned a = lane + (stage * N + k) * kArray + i * kRow;
        if constexpr (sizeof(word) == 8) {
            float2 f;
            asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(f.x), "=f"(f.y) : "r"(a));
            return *reinterpret_cast<word*>(&f);
        } else {
            uint32_t u;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(u) : "r"(a));
            return *reinterpret_cast<word*>(&u);
        }
    }
};

template <typename T, bool COUPLED, int L, int ACCESS>
__global__ void __launch_bounds__(32 * (ACCESS == PIPED ? kPipedWarps + 1 : kMaxWarps), ACCESS == PIPED ? 1 : 2) recurrence_forward_kernel(const RecArgs p, const __grid_constant__ RecMaps maps, const int blocks) {
    using W = Word<T>;
    constexpr int kArrays = 2;
    extern __shared__ __align__(128) char staged[];
    __shared__ unsigned long long arrived[staged_rows(ACCESS) ? most_warps(ACCESS) * kMaxStages : 1];
    constexpr bool kScan = ACCESS == PIPED;                 // the last warp scans
    const int warps = kScan ? (int)blockDim.y - 1 : (int)blockDim.y;
    const bool alone = !kScan && blocks == 1 && warps == 1;
    using Shared = std::conditional_t<kScan, Scan, Exchange>;
    Shared& ex = *reinterpret_cast<Shared*>(staged + warps * (staged_rows(ACCESS) ? p.stages : 0) * kStageBytes<T, L, kArrays>);
    const Place q = place<ACCESS>(p, blocks, warps);
    if (!alone) exchange_begin(ex, warps, blocks);
    const unsigned stride = blocks * warps * L, es = sizeof(T), apart = (q.col[1] - q.col[0]) * es;
    const unsigned in_step = (unsigned)p.in_step * es, out_step = (unsigned)p.out_step * es;
    const unsigned in_at = q.col[0] * es + q.slot * L * in_step, out_at = q.col[0] * es + q.slot * L * out_step;
    const char* x = (const char*)p.x + q.seq * p.in_seq * es;
    const char* g = (const char*)p.gate + q.seq * p.in_seq * es;
    char* out = (char*)p.out + q.seq * p.out_seq * es;
    const long long in_round = (long long)stride * in_step, out_round = (long long)stride * out_step;
    const long long states = (long long)q.seq * p.width;
    float carry[V];                                         // -y when coupled
    bool broken = false;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        carry[v] = p.y0 != nullptr ? p.y0[states + q.col[v]] : 0.f;
        if (COUPLED) carry[v] = -carry[v];
    }
    if constexpr (kScan)
    if ((int)threadIdx.y == warps) {
        cluster_wait();
        scan(ex, 0u, stride, (unsigned)q.len, carry, warps, blocks, q.rank);
        cluster_arrive();
        cluster_wait();                                     // every block has read the state that the one behind the last step may replace
        if (p.last != nullptr && q.rank == 0) {
#pragma unroll
            for (int v = 0; v < V; ++v) p.last[states + q.col[v]] = COUPLED ? -carry[v] : carry[v];
        }
        return;
    }
    Tile<T, L, kArrays, ACCESS> tile;
    // steps of this warp's tile that exist
    auto count = [&](unsigned base) {
        const unsigned t0 = base + q.slot * L;
        return t0 < (unsigned)q.len ? (int)min((unsigned)L, (unsigned)q.len - t0) : 0;
    };
    const unsigned copied = staged_rows(ACCESS) ? copied_below(q.slot * L, L, q.len, p.n_steps) : 0u;
    auto request = [&](unsigned base, int stage) {
        if constexpr (staged_rows(ACCESS))
            if (base < copied && elected()) tile.request(stage, maps, 3u, q.tile, q.seq, p.time_major != 0, (int)(base + q.slot * L), 0);
    };
    // the tile that is not copied: in the last round only
    auto request_rows = [&](unsigned base, int stage) {
        if constexpr (staged_rows(ACCESS))
            if (base >= copied && base < (unsigned)q.len) {
                const long long from = (long long)base * in_step + in_at;
                tile.request_rows(stage, 0, 0, count(base), g + from, in_step);
                tile.request_rows(stage, 1, 0, count(base), x + from, in_step);
                tile.rows_requested(stage);
            }
    };
    auto load = [&](auto full, unsigned base) {
        if constexpr (!staged_rows(ACCESS)) {
            const int n = count(base);
            tile.template load<full.value>(0, g, in_at, in_step, 0, n);
            tile.template load<full.value>(1, x, in_at, in_step, 0, n);
            if (alone) __syncwarp();                        // lanes behind the last channel have read before the others write results over these rows
            x += in_round; g += in_round;
            const int ahead = count(base + stride);
            const unsigned first = in_at - (q.col[0] - q.tile) * es;
            touch_rows<T, L, 2>(min(64, p.width - q.tile) * (int)es, [&](int k, int i) { return i < ahead ? (k == 0 ? g : x) + (unsigned)(first + i * in_step) : nullptr; });
        }
    };
    if constexpr (staged_rows(ACCESS)) {
        tile.bind(staged, arrived, q.lane, p.stages);
        for (int k = 0; k < p.stages; ++k) {
            request(k * stride, k);
            request_rows(k * stride, k);
        }
    } else tile.apart = apart;
    if (blocks > 1) cluster_wait();
    // A round's two halves: gates and the map of this warp's steps, published; then the steps again from the state in front of them
    struct Turn { float nb[L][V]; Affine before; unsigned base, round; int stage; };
    auto whole = [&](unsigned base) { return base + stride <= (unsigned)q.len; };
    auto first = [&](auto kind, Turn& r, unsigned base, unsigned round) {
        r.base = base;
        r.round = round;
        const int n = count(base);
        int stage = 0;
        if constexpr (staged_rows(ACCESS)) stage = tile.wait(broken);
        r.stage = stage;
        auto run = [&](auto full) {
            load(full, base);
#pragma unroll
            for (int i = 0; i < L; ++i) {
                float f[V], none[V];
                W::get(tile.get(stage, 0, i), f);
                negated_gate<T, false>(f, r.nb[i], none);
                if (!full.value && i >= n) {                // a step that does not exist keeps the state
#pragma unroll
                    for (int v = 0; v < V; ++v) r.nb[i][v] = kKeep;
                }
            }
            if (alone) return;
            Map own;
#pragma unroll
            for (int i = 0; i < L; ++i) {
                float xs[V];
                W::get(tile.get(stage, 1, i), xs);
                if (!full.value && i >= n) {
#pragma unroll
                    for (int v = 0; v < V; ++v) xs[v] = 0.f;
                }
                own.decay(r.nb[i]);
                step_forward<COUPLED>(own.u, r.nb[i], xs);
            }
            if constexpr (kScan) publish(ex, round, own);
            else publish(ex, round, own, r.before, blocks, q.rank);
        };
        of_kind(kind, whole(base), run);
    };
    auto second = [&](auto kind, const Turn& r) {
        float start[V];
        const int stage = r.stage, n = count(r.base);
        if constexpr (kScan) collect(ex, r.round, start, broken);
        else if (!alone) collect(ex, r.round, r.before, carry, start, blocks, q.rank, broken);
        else {
#pragma unroll
            for (int v = 0; v < V; ++v) start[v] = carry[v];
        }
        auto run = [&](auto full) {
            unsigned at = out_at;
#pragma unroll
            for (int i = 0; i < L; ++i, at += out_step) {
                float xs[V];
                W::get(tile.get(stage, 1, i), xs);
                if (!full.value && i >= n) {
#pragma unroll
                    for (int v = 0; v < V; ++v) xs[v] = 0.f;
                }
                step_forward<COUPLED>(start, r.nb[i], xs);
                if (full.value || i < n) store_pair<T, ACCESS>(out, at, apart, COUPLED ? W::negate(W::put(start)) : W::put(start));
            }
        };
        of_kind(kind, whole(r.base), run);
        out += out_round;
        if (alone) {
#pragma unroll
            for (int v = 0; v < V; ++v) carry[v] = staged_rows(ACCESS) && broken ? __int_as_float(0x7fffffff) : start[v];
        }
        if constexpr (staged_rows(ACCESS)) {
            __syncwarp();                                   // all lanes have read this stage
            request(r.base + p.stages * stride, stage);
            request_rows(r.base + p.stages * stride, stage);
        }
    };
    rounds<ACCESS == PIPED, Turn>(0u, stride, (unsigned)q.len, whole, first, second);
    if (p.zero_behind) {
        const long long n = blocks * warps, apace = n * out_step;
        long long i = (long long)q.len + q.slot;
        for (char* to = (char*)p.out + (q.seq * p.out_seq + i * p.out_step + q.col[0]) * es; i < p.n_steps; i += n, to += apace) store_pair<T, ACCESS>(to, 0, apart, typename W::type{});
    }
    if (blocks > 1) { cluster_arrive(); cluster_wait(); }   // nobody leaves while its shared memory may be written, and every block has read its y0
    else if (alone) __syncwarp();                           // every lane, or warp, has read its y0
    else __syncthreads();
    if (!kScan && p.last != nullptr && q.slot == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) p.last[states + q.col[v]] = COUPLED ? -carry[v] : carry[v];
    }
}

// A few steps of many sequences (serving token by token): a thread runs them for two channels; nothing to exchange and no shared memory, so that a call costs
// little more than its launch (100 sequences of 1024 channels, one step: 4 us less than the kernel above)
constexpr int kFewSteps = 4;
template <typename T, bool COUPLED, int ACCESS> __global__ void __launch_bounds__(128) recurrence_steps_kernel(const RecArgs p) {
    using W = Word<T>;
    const int pairs = (p.width + 1) / 2;
    const long long i = (long long)blockIdx.x * 128 + threadIdx.x;
    const int seq = (int)(i / pairs);
    if (seq >= p.n_seq) return;
    const int col = (int)(i - (long long)seq * pairs) * 2, col2 = min(col + 1, p.width - 1);
    const unsigned es = sizeof(T), apart = (col2 - col) * es;
    const int len = p.lengths != nullptr ? min(max(p.lengths[seq], 0), p.n_steps) : p.n_steps;
    const long long states = (long long)seq * p.width;
    float s[2] = {0.f, 0.f};
    if (p.y0 != nullptr) { s[0] = p.y0[states + col]; s[1] = p.y0[states + col2]; }
    if (COUPLED) { s[0] = -s[0]; s[1] = -s[1]; }
    const char *x = (const char*)p.x + (seq * p.in_seq + col) * es, *g = (const char*)p.gate + (seq * p.in_seq + col) * es;
    char* out = (char*)p.out + (seq * p.out_seq + col) * es;
    for (int t = 0; t < len; ++t) {
        float xs[2], f[2], nb[2], none[2];
        W::get(load_pair<T, ACCESS>(x + t * p.in_step * es, 0, apart), xs);
        W::get(load_pair<T, ACCESS>(g + t * p.in_step * es, 0, apart), f);
        negated_gate<T, false>(f, nb, none);
        step_forward<COUPLED>(s, nb, xs);
        store_pair<T, ACCESS>(out + t * p.out_step * es, 0, apart, COUPLED ? W::negate(W::put(s)) : W::put(s));
    }
    if (p.zero_behind)
        for (int t = len; t < p.n_steps; ++t) store_pair<T, ACCESS>(out + t * p.out_step * es, 0, apart, typename W::type{});
    if (p.last != nullptr) {
        p.last[states + col] = COUPLED ? -s[0] : s[0];
        p.last[states + col2] = COUPLED ? -s[1] : s[1];
    }
}

// Steps counted from the end: step i of a warp's tile is time n_steps - 1 - (base + slot * L + i).
// Arrays of the tile: gate, cotangent, state in front of the step, x (coupled only)
template <typename T, bool COUPLED, int L, int ACCESS>
__global__ void __launch_bounds__(32 * (ACCESS == PIPED ? kPipedWarps + 1 : kMaxWarps), ACCESS == PIPED ? 1 : 2) recurrence_backward_kernel(const RecArgs p, const __grid_constant__ RecMaps maps, const int blocks) {
    using W = Word<T>;
    constexpr int kArrays = COUPLED ? 4 : 3;
    using word = typename W::type;
    extern __shared__ __align__(128) char staged[];
    __shared__ unsigned long long arrived[staged_rows(ACCESS) ? most_warps(ACCESS) * kMaxStages : 1];
    constexpr bool kScan = ACCESS == PIPED;                 // the last warp scans
    const int warps = kScan ? (int)blockDim.y - 1 : (int)blockDim.y;
    const bool alone = !kScan && blocks == 1 && warps == 1;
    using Shared = std::conditional_t<kScan, Scan, Exchange>;
    Shared& ex = *reinterpret_cast<Shared*>(staged + warps * (staged_rows(ACCESS) ? p.stages : 0) * kStageBytes<T, L, kArrays>);
    const Place q = place<ACCESS>(p, blocks, warps);
    if (!alone) exchange_begin(ex, warps, blocks);
    const unsigned stride = blocks * warps * L, es = sizeof(T), apart = (q.col[1] - q.col[0]) * es;
    // offsets count down from the last time of the round
    const unsigned in_step = (unsigned)p.in_step * es, out_step = (unsigned)p.out_step * es, back = (stride - 1) - q.slot * L;
    const unsigned in_at = q.col[0] * es + back * in_step, out_at = q.col[0] * es + back * out_step;
    const unsigned skipped = p.n_steps - q.len;             // steps at the start of the count that do not exist
    unsigned base = skipped / stride * stride;              // rounds that lie behind the sequence are passed over
    const long long in_round = (long long)stride * in_step, out_round = (long long)stride * out_step;
    const long long first_in = q.seq * p.in_seq * es + ((long long)p.n_steps - stride - base) * in_step;
    const long long first_out = q.seq * p.out_seq * es + ((long long)p.n_steps - stride - base) * out_step;
    const char *x = (const char*)p.x + first_in, *g = (const char*)p.gate + first_in, *y = (const char*)p.y + first_out - out_step, *dy = (const char*)p.dy + first_out;
    char *dx = (char*)p.out + first_in, *dg = (char*)p.out2 + first_in;
    const long long states = (long long)q.seq * p.width;
    float carry[V];
    bool broken = false;
    Largest<T> largest;
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = p.dyT != nullptr ? p.dyT[states + q.col[v]] : 0.f;
    if constexpr (kScan)
    if ((int)threadIdx.y == warps) {
        cluster_wait();
        scan(ex, base, stride, (unsigned)p.n_steps, carry, warps, blocks, q.rank);
        cluster_arrive();
        cluster_wait();                                     // every block has read the state that the one behind the last step may replace
        if (p.last != nullptr && q.rank == 0) {
#pragma unroll
            for (int v = 0; v < V; ++v) p.last[states + q.col[v]] = carry[v];
        }
        return;
    }
    Tile<T, L, kArrays, ACCESS> tile;
    // the tile's steps lo .. hi - 1 exist
    auto range = [&](unsigned base, int& lo, int& hi) {
        const unsigned first = base + q.slot * L;
        lo = first < skipped ? (int)min((unsigned)L, skipped - first) : 0;
        hi = first < (unsigned)p.n_steps ? (int)min((unsigned)L, p.n_steps - first) : 0;
    };
    auto request = [&](unsigned base, int stage) {
        if constexpr (staged_rows(ACCESS))
            if (base < (unsigned)p.n_steps && elected()) {
                const int t0 = p.n_steps - (int)(base + q.slot * L) - L;                        // the tile's earliest time; its steps lie the other way round
                tile.request(stage, maps, (COUPLED ? 13u : 5u) | (p.dy != nullptr ? 2u : 0u), q.tile, q.seq, p.time_major != 0, t0, t0 - 1);
            }
    };
    auto load = [&](auto full, unsigned base) {
        if constexpr (!staged_rows(ACCESS)) {
            constexpr bool F = full.value;
            int lo, hi;
            range(base, lo, hi);
            const int before = base + q.slot * L + hi == (unsigned)p.n_steps ? hi - 1 : hi;     // time 0 has no stored state in front of it
            tile.template load<F>(0, g, in_at, 0u - in_step, lo, hi);
            if (p.dy != nullptr) tile.template load<F>(1, dy, out_at, 0u - out_step, lo, hi);
            tile.template load<F>(2, y, out_at, 0u - out_step, lo, before);
            if constexpr (COUPLED) tile.template load<F>(3, x, in_at, 0u - in_step, lo, hi);
            if (alone) __syncwarp();                        // as in the forward pass
            x -= in_round; g -= in_round; y -= out_round; dy -= out_round;
            range(base + stride, lo, hi);
            const unsigned to_tile = (q.col[0] - q.tile) * es;
            const int zero = (int)(p.n_steps - 1 - (base + stride + q.slot * L));
            touch_rows<T, L, kArrays>(min(64, p.width - q.tile) * (int)es, [&](int k, int i) {
                const char* const from = k == 0 ? g : k == 1 ? dy : k == 2 ? y : x;
                const bool there = i >= lo && i < hi && (k != 1 || p.dy != nullptr) && (k != 2 || i != zero);
                return there ? from + (unsigned)((k == 0 || k == 3 ? in_at - i * in_step : out_at - i * out_step) - to_tile) : nullptr;
            });
        }
    };
    if constexpr (staged_rows(ACCESS)) {
        tile.bind(staged, arrived, q.lane, p.stages);
        int lo, hi;
        range(base, lo, hi);
        if (copied_back(base + q.slot * L, skipped)) request(base, 0);
        else {                                              // (in the first round only)
            const long long t = (long long)p.n_steps - base - q.slot * L - hi;                      // the earliest step that exists
            const long long in = (q.seq * p.in_seq + q.col[0]) * es + t * in_step, outer = (q.seq * p.out_seq + q.col[0]) * es + t * out_step;
            const int before = t == 0 ? 1 : 0;                                                      // time 0 has no stored state in front of it
            tile.request_rows(0, 0, L - hi, hi - lo, (const char*)p.gate + in, in_step);
            if (p.dy != nullptr) tile.request_rows(0, 1, L - hi, hi - lo, (const char*)p.dy + outer, out_step);
            tile.request_rows(0, 2, L - hi + before, hi - lo - before, (const char*)p.y + outer + (before - 1ll) * out_step, out_step);
            if (COUPLED) tile.request_rows(0, 3, L - hi, hi - lo, (const char*)p.x + in, in_step);
            tile.rows_requested(0);
        }
        for (int k = 1; k < p.stages; ++k) request(base + k * stride, k);
    } else tile.apart = apart;
    auto get = [&](int stage, int k, int i) { return tile.get(stage, k, staged_rows(ACCESS) ? L - 1 - i : i); };
    if (blocks > 1) cluster_wait();
    const bool no_dy = p.dy == nullptr;
    struct Turn { float nb[L][V], slope[L][V]; Affine before; unsigned base, round; int stage; };
    // every step of the round exists, and none is time 0
    auto whole = [&](unsigned base) { return base >= skipped && base + stride < (unsigned)p.n_steps; };
    auto first = [&](auto kind, Turn& r, unsigned base, unsigned round) {
        r.base = base;
        r.round = round;
        int stage = 0, lo, hi;
        range(base, lo, hi);
        if constexpr (staged_rows(ACCESS)) stage = tile.wait(broken);
        r.stage = stage;
        auto run = [&](auto full) {
            if (staged_rows(ACCESS) && !full.value && lo > 0) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // (a tile of rows; a copy goes there next)
            load(full, base);
#pragma unroll
            for (int i = 0; i < L; ++i) {
                float f[V];
                W::get(get(stage, 0, i), f);
                negated_gate<T, true>(f, r.nb[i], r.slope[i]);
                if (!full.value && (i < lo || i >= hi)) {                                       // a step that does not exist keeps the adjoint
#pragma unroll
                    for (int v = 0; v < V; ++v) r.nb[i][v] = kKeep;
                }
            }
            if (alone) return;
            Map own;
#pragma unroll
            for (int i = 0; i < L; ++i) {
                float d[V], l[V];
                W::get(get(stage, 1, i), d);
                if (no_dy || (!full.value && (i < lo || i >= hi))) {
#pragma unroll
                    for (int v = 0; v < V; ++v) d[v] = 0.f;
                }
                own.decay(r.nb[i]);
                Ops::add(l, own.u, d);
                Ops::fma(own.u, r.nb[i], l, l);
            }
            if constexpr (kScan) publish(ex, round, own);
            else publish(ex, round, own, r.before, blocks, q.rank);
        };
        of_kind(kind, whole(base), run);
    };
    auto second = [&](auto kind, const Turn& r) {
        float start[V];
        const int stage = r.stage;
        int lo, hi;
        range(r.base, lo, hi);
        const int zero = (int)(p.n_steps - 1 - (r.base + q.slot * L));                          // index of time 0
        if constexpr (kScan) collect(ex, r.round, start, broken);
        else if (!alone) collect(ex, r.round, r.before, carry, start, blocks, q.rank, broken);
        else {
#pragma unroll
            for (int v = 0; v < V; ++v) start[v] = carry[v];
        }
        auto run = [&](auto full) {
            unsigned at = in_at;
#pragma unroll
            for (int i = 0; i < L; ++i, at -= in_step) {
                float ys[V], d[V], l[V], gx[V], gg[V];
                W::get(get(stage, 1, i), d);
                if (no_dy || (!full.value && (i < lo || i >= hi))) {
#pragma unroll
                    for (int v = 0; v < V; ++v) d[v] = 0.f;
                }
                W::get(get(stage, 2, i), ys);
                if (!full.value && i == zero) {
#pragma unroll
                    for (int v = 0; v < V; ++v) ys[v] = p.y0 != nullptr ? p.y0[states + q.col[v]] : 0.f;
                }
                Ops::add(l, start, d);
                Ops::fma(start, r.nb[i], l, l);
                Ops::mul(gg, r.slope[i], l);
                if constexpr (COUPLED) {
                    float xs[V], minus[V];
                    W::get(get(stage, 3, i), xs);
                    Ops::mul(gx, r.nb[i], l);
#pragma unroll
                    for (int v = 0; v < V; ++v) minus[v] = -1.f;
                    Ops::fma(ys, ys, minus, xs);
                }
                Ops::mul(gg, gg, ys);
                if (full.value || (i >= lo && i < hi)) {
                    const word wx = COUPLED ? W::negate(W::put(gx)) : W::put(l), wg = COUPLED ? W::put(gg) : W::negate(W::put(gg));
                    if (p.flag != nullptr) { see<T>(largest, wx); see<T>(largest, wg); }
                    store_pair<T, ACCESS>(dx, at, apart, wx);
                    store_pair<T, ACCESS>(dg, at, apart, wg);
                }
            }
        };
        of_kind(kind, whole(r.base), run);
        if (alone) {
#pragma unroll
            for (int v = 0; v < V; ++v) carry[v] = staged_rows(ACCESS) && broken ? __int_as_float(0x7fffffff) : start[v];
        }
        dx -= in_round; dg -= in_round;
        if constexpr (staged_rows(ACCESS)) {
            __syncwarp();
            request(r.base + p.stages * stride, stage);
        }
    };
    rounds<ACCESS == PIPED, Turn>(base, stride, (unsigned)p.n_steps, whole, first, second);
    if (p.zero_behind) {
        const long long n = blocks * warps, apace = n * in_step;
        long long i = (long long)q.len + q.slot, to = (q.seq * p.in_seq + i * p.in_step + q.col[0]) * es;
        for (; i < p.n_steps; i += n, to += apace) {
            store_pair<T, ACCESS>((char*)p.out + to, 0, apart, word{});
            store_pair<T, ACCESS>((char*)p.out2 + to, 0, apart, word{});
        }
    }
    warp_flag_or(p.flag, largest.nonfinite());
    if (blocks > 1) { cluster_arrive(); cluster_wait(); }   // as in the forward pass
    else if (alone) __syncwarp();
    else __syncthreads();
    if (!kScan && p.last != nullptr && q.slot == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) p.last[states + q.col[v]] = carry[v];
    }
}

// How a call is spread over the GPU: warps along the time axis of a block, then blocks of a cluster, until every SM has its warps or no steps are left
struct Shape { int warps, blocks; long long tiles; };
// a round's bytes have to stay within 32-bit offsets
bool round_fits(const RecArgs& a, long long steps, int es) {
    const long long step = a.in_step > a.out_step ? a.in_step : a.out_step;
    return step < (1ll << 32) && (steps * step + a.width) * es < (1ll << 32);
}
// Blocks of a cluster: of the sizes that the GPU holds as many of at once as there are tiles, the largest (65536 steps of 1024 channels, 16 tiles: 148 SMs hold 15
// clusters of 8 blocks and 22 of 6, with the last cluster of 8 behind the others 1.4 times the time).  `room` asks the runtime how many clusters of a size there is room for.
template <typename Room> Shape shape_of(const mpode_recurrence_desc& d, const RecArgs& a, int steps_of_warp, Room&& room) {
    Shape s;
    s.tiles = (long long)d.n_seq * ((d.width + 63) / 64);
    s.warps = s.blocks = 1;
    // (128 sequences of 128 steps, 4096 tiles: 57 us with 2 warps, 65 with 4, 74 with 8)
    while (s.warps < kMaxWarps && (long long)s.warps * steps_of_warp < d.n_steps && s.tiles * s.warps < 32 * sm_count()) s.warps *= 2;
    if (s.tiles * 2 <= sm_count())
        for (int c : {16, 8, 6, 4, 3, 2})
            if ((c - 1ll) * s.warps * steps_of_warp < d.n_steps && round_fits(a, (long long)c * s.warps * steps_of_warp, (int)low_size(d.low)) && s.tiles <= room(c)) {
                s.blocks = c;
                break;
            }
    while (s.warps > 1 && !round_fits(a, (long long)s.warps * steps_of_warp, (int)low_size(d.low))) s.warps /= 2;
    return s;
}

// most: the shared memory that any call of this kernel asks for.  The limit is set to that and not to this call's, which another host thread's call may be about
// to replace by its own.
cudaError_t launch(void (*kernel)(const RecArgs, const RecMaps, const int), const RecArgs& a, const RecMaps& maps, const Shape& s, bool scans, size_t smem, size_t most,
                   cudaStream_t st) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(s.tiles * s.blocks));
    cfg.blockDim = dim3(32, s.warps + (scans ? 1 : 0));
    cfg.stream = st;
    cfg.dynamicSmemBytes = smem;
    const cudaError_t set = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
    if (set != cudaSuccess) return set;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)s.blocks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = s.blocks > 1 ? 1 : 0;
    if (s.blocks > 8) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
    }
    return cudaLaunchKernelEx(&cfg, kernel, a, maps, s.blocks);
}

// steps of a warp in a round
template <typename T> constexpr int kForwardSteps = sizeof(T) == 4 ? 8 : 16;
template <typename T> constexpr int kBackwardSteps = sizeof(T) == 4 ? 4 : 8;

// two channels an access need even widths and strides and rows aligned to two elements
bool words_fit(const mpode_recurrence_desc& d, const RecArgs& a) {
    if (d.width & 1) return false;
    if ((a.in_step | a.in_seq | a.out_step | a.out_seq) & 1) return false;
    const void* const all[] = {a.x, a.gate, a.y, a.dy, a.out, a.out2};
    for (const void* q : all)
        if (misaligned(q, 2 * low_size(d.low))) return false;
    return true;
}
// rows of multiples of 16 bytes from aligned pointers everywhere
bool pieces_fit(const mpode_recurrence_desc& d, const RecArgs& a) {
    const long long es = (long long)low_size(d.low);
    if (((a.in_step | a.in_seq | a.out_step | a.out_seq | d.width) * es) & 15) return false;
    const void* const all[] = {a.x, a.gate, a.y, a.dy};
    for (const void* q : all)
        if (misaligned(q, 16)) return false;
    return true;
}
template <int A> struct Way { static constexpr int value = A; };
// maps of [n_seq][n_steps][width] with boxes of L steps; the dimension with the larger stride comes last
bool map_of(const void* p, const mpode_recurrence_desc& d, long long seq, long long step, int steps, bool time_major, CUtensorMap* out) {
    return time_major ? make_tensor_map(p, d.low, d.width, d.n_seq, d.n_steps, seq, step, 64, 1, steps, out)
                      : make_tensor_map(p, d.low, d.width, d.n_steps, d.n_seq, step, seq, 64, steps, 1, out);
}
// Shared memory of a block: the stages of its warps, and the exchange
template <typename T, int L, int N> constexpr size_t smem_bytes(int access, int warps, int stages, int blocks) {
    return (staged_rows(access) ? warps * stages * kStageBytes<T, L, N> : 0) + (access == PIPED ? sizeof(Scan) : blocks > 1 ? sizeof(Exchange) : kBlockExchange);
}
template <typename T, int L, int N> constexpr size_t most_bytes(int access) { return smem_bytes<T, L, N>(access, most_warps(access), kMaxStages, access == STAGED ? 1 : kMaxCluster); }
// How many clusters of a size the current device holds at once with one block an SM (asked once; the piped kernels are alike in what they need)
int cluster_room(int blocks) {
    static std::atomic<int> known[kMaxDevices][kMaxCluster + 1];
    std::atomic<int>& slot = known[current_device()][blocks];
    int n = slot.load(std::memory_order_relaxed);
    if (n > 0) return n - 1;
    using T = __nv_bfloat16;
    constexpr int L = kForwardSteps<T>;
    n = clusters_at_once((const void*)recurrence_forward_kernel<T, true, L, PIPED>, dim3(32, kPipedWarps + 1), most_bytes<T, L, 2>(PIPED), blocks);
    if (n < 0) return 0;                                    // (asked again by the next call)
    slot.store(n + 1, std::memory_order_relaxed);
    return n;
}
template <typename T, bool COUPLED, bool BACKWARD> cudaError_t run(const mpode_recurrence_desc& d, RecArgs a, cudaStream_t st) {
    constexpr int L = BACKWARD ? kBackwardSteps<T> : kForwardSteps<T>, N = BACKWARD ? (COUPLED ? 4 : 3) : 2;
    if (!BACKWARD && d.n_steps <= kFewSteps) {
        const unsigned grid = (unsigned)(((long long)d.n_seq * ((d.width + 1) / 2) + 127) / 128);
        return words_fit(d, a) ? launch_grid(recurrence_steps_kernel<T, COUPLED, PAIRS>, grid, 128, st, a)
                               : launch_grid(recurrence_steps_kernel<T, COUPLED, SINGLES>, grid, 128, st, a);
    }
    Shape s = shape_of(d, a, L, cluster_room);
    RecMaps maps;
    // Three rounds in shared memory, or two where two blocks of 8 warps share an SM (us with 2 / 3: backward of 8 x 4096 x 2048 bfloat16, 256 tiles, 143 / 152;
    // 8 x 2048 x 1024 float32, 128 tiles, 87 / 80; 128 x 128 x 2048, 2 warps a block, 96 / 82)
    const auto go = [&](auto access) {
        constexpr int A = access.value;
        a.stages = A == PIPED || s.warps < kMaxWarps || s.tiles <= sm_count() ? 3 : 2;
        const size_t smem = smem_bytes<T, L, N>(A, s.warps, a.stages, s.blocks), most = most_bytes<T, L, N>(A);
        if constexpr (BACKWARD) return launch(recurrence_backward_kernel<T, COUPLED, L, A>, a, maps, s, A == PIPED, smem, most, st);
        else return launch(recurrence_forward_kernel<T, COUPLED, L, A>, a, maps, s, A == PIPED, smem, most, st);
    };
    if (d.n_steps > 2 * s.warps * s.blocks * L && words_fit(d, a) && pieces_fit(d, a)) {
        a.time_major = d.n_seq > 1 && a.in_seq < a.in_step;
        const bool tm = a.time_major != 0;
        // (all arrays take their coordinates in one order: where inputs and outputs differ in theirs, registers)
        bool ok = tm == (d.n_seq > 1 && a.out_seq < a.out_step) && map_of(a.gate, d, a.in_seq, a.in_step, L, tm, &maps.m[0]);
        if (!BACKWARD) ok = ok && map_of(a.x, d, a.in_seq, a.in_step, L, tm, &maps.m[1]);
        else {
            if (a.dy != nullptr) ok = ok && map_of(a.dy, d, a.out_seq, a.out_step, L, tm, &maps.m[1]);
            ok = ok && map_of(a.y, d, a.out_seq, a.out_step, L, tm, &maps.m[2]);
            if (COUPLED) ok = ok && map_of(a.x, d, a.in_seq, a.in_step, L, tm, &maps.m[3]);
        }
        if (ok && s.blocks > 1) {
            // many rounds: more warps hide one another's phases (us with 8 / 11: 65536 steps of 1024 bfloat16 channels 123 / 109, backward of 32768 127 / 109;
            // few rounds: 4 x 2048 x 512, 16.4 / 18.5).  Twelve warps with the scanning one are three a scheduler, with 168 registers a thread; a thirteenth leaves 128 (117, 113)
            const long long steps = (long long)kPipedWarps * s.blocks * L;
            if (d.n_steps >= 8 * steps && round_fits(a, steps, (int)low_size(d.low))) s.warps = kPipedWarps;
            return go(Way<PIPED>());
        }
        if (ok) return go(Way<STAGED>());
    }
    return words_fit(d, a) ? go(Way<PAIRS>()) : go(Way<SINGLES>());
}
template <bool BACKWARD> cudaError_t run(const mpode_recurrence_desc& d, const RecArgs& a, cudaStream_t st) {
    return with_low(d.low, [&](auto t) {
        using T = decltype(t);
        return d.coupled ? run<T, true, BACKWARD>(d, a, st) : run<T, false, BACKWARD>(d, a, st);
    });
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
    const __int128 S = d->n_seq - 1, N = d->n_steps - 1;
    const auto overlap = [&](long long by_seq, long long by_step) { return by_seq <= N * by_step + lo - 1 && by_step <= S * by_seq + lo - 1; };
    if (S > 0 && N > 0 && (overlap(a.in_seq, a.in_step) || overlap(a.out_seq, a.out_step)))
        return operator_fail(MPODE_ERR_INVALID_ARG, "recurrence: the strides make rows overlap");
    a.n_seq = d->n_seq; a.n_steps = d->n_steps; a.width = d->width; a.zero_behind = d->zero_behind;
    if (d->n_steps <= 1) a.in_step = a.out_step = lo;
    if (!round_fits(a, 16, (int)low_size(d->low)))
        return operator_fail(MPODE_ERR_UNSUPPORTED, "recurrence: step strides %lld and %lld (16 steps have to lie within 4 GB)", a.in_step, a.out_step);
    return MPODE_OK;
}
mpode_status check_pointers(const mpode_recurrence_desc& d, const RecArgs& a) {
    // outputs over inputs of the other strides: y over x, dL_dx over dL_dy
    const bool alike = a.in_step == a.out_step && (d.n_seq <= 1 || a.in_seq == a.out_seq);
    if (d.n_steps > 0 && !alike && (a.y == nullptr ? a.out == a.x || a.out == a.gate : a.out == a.dy || a.out2 == a.dy))
        return operator_fail(MPODE_ERR_INVALID_ARG, "recurrence: an output lies on an input of other strides");
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
    return operator_launched(run<false>(*desc, a, (cudaStream_t)cuda_stream), "mpode_recurrence_forward");
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
    return operator_launched(run<true>(*desc, a, (cudaStream_t)cuda_stream), "mpode_recurrence_backward");
}

}  // extern "C"
