// Backward pass of the residual step: adjoint, cotangents and the weights' gradients of a row in one pass.
//
// With y, u the rows (less their means), r, s their reciprocal deviations, c = scale w_post, and drop() for the mask with the kept elements' factor:
//   e = r dz,  dw_pre += e y,  a = dy' + w_pre e - y r^2 mean(w_pre e y) - mean(w_pre e)
//   t = h s drop(a),  q = t u,  S += q sig,  dgate = c q sig',  du = c t sig - u s^2 mean(c q sig) - mean(c t sig)
// where the last means are taken only with MEANVAR; dw_post = scale S and dscale = w_post S come from one sum over the rows, formed behind the last one.
//
// A row goes through three phases with a sum over the row between them.  Its inputs lie in shared memory and are read again in the next phase: what a
// thread keeps of its eight columns are two gradients and two weights (32 registers) and one product, so that three blocks of 8 warps of 16-bit rows fit an SM
// (two of float32 rows, by their stages) and one's sums are hidden behind another's arithmetic.
#include "residual.cuh"

namespace mpode {
namespace {

template <typename T, bool VEC, bool CENTER, int WARPS, bool CLUSTER>
__global__ void __launch_bounds__(Lane<WARPS, CLUSTER>::kThreads, WARPS == 1 ? 2 : 768 / Lane<WARPS, CLUSTER>::kThreads)
residual_backward_kernel(const ResArgs p, const int blocks) {
    constexpr int N = CENTER ? 2 : 1;
    using Sum = RowSum<N, WARPS, CLUSTER>;
    using In = Rows<T, VEC, WARPS, CLUSTER, 2, 3>;          // y', dy', dz, u, gate
    extern __shared__ __align__(16) char staged[];
    __shared__ typename Sum::Shared shared;
    const Lane<WARPS, CLUSTER> q(p.width, blocks);
    Sum sum(shared, blocks);
    In in(staged, q);
    const uint64_t seed = p.drop.on ? p.drop.rng[0] : 0, step = p.drop.on ? p.drop.rng[1] : 0;
    const int groups_row = (p.width + 7) / 8;
    const float inv = 1.f / (float)p.width;
    const bool has_dz = p.dz != nullptr, has_dy = p.dy != nullptr, has_u = p.u != nullptr, has_gate = p.gate != nullptr;
    auto request = [&](long long r, int stage, bool ahead = false) {
        const int c = q.base;
        const void* const from[5] = {has_dz ? p.y + r * p.ld_y + c : nullptr, has_dy ? p.dy + r * p.ld_y + c : nullptr,
                                     has_dz ? (const T*)p.dz + r * p.ld_z + c : nullptr, has_u ? (const T*)p.u + r * p.ld_u + c : nullptr,
                                     has_gate ? (const T*)p.gate + r * p.ld_gate + c : nullptr};
        if (ahead) in.touch(from);
        else in.request(stage, from);
    };
    if (in.leader)
        for (int k = 0; k < in.kStages; ++k)
            if (q.first + (long long)k * q.step < p.rows) request(q.first + (long long)k * q.step, k);
    Oct S, gw_pre, w_pre = weights_of<VEC>(p.w_pre, q), c = weights_of<VEC>(p.scale, q);
    {
        const Oct w_post = weights_of<VEC>(p.w_post, q);
#pragma unroll
        for (int k = 0; k < 4; ++k) c.v[k] = __fmul2_rn(c.v[k], w_post.v[k]);
    }
    S.fill(0.f); gw_pre.fill(0.f);
    Largest<T> largest;
    float4 stats = make_float4(0.f, 1.f, 0.f, 1.f);
    int row = q.first;
    if (p.stats != nullptr && row < p.rows) stats = reinterpret_cast<const float4*>(p.stats)[row];
    // the row's means, negative; the first one times `factor`
    auto means = [&](float2 m0, float2 m1, int kind, float factor, float2& n0, float2& n1) {
        n0 = n1 = pair(0.f);
        if (kind == MPODE_NORM_NONE) return;
        float m[N];
        m[0] = m0.x + m0.y;
        if (CENTER) m[N - 1] = m1.x + m1.y;
        sum(m, q);
        n0 = pair(-m[0] * inv * factor);
        if (CENTER && kind == MPODE_NORM_MEANVAR) n1 = pair(-m[N - 1] * inv);
    };
    auto less = [&](Quad v, float2 mean) {
        if (CENTER) { v.v[0] = __fadd2_rn(v.v[0], mean); v.v[1] = __fadd2_rn(v.v[1], mean); }
        return v;
    };
    while (row < p.rows) {
        const int next = q.step < p.rows - row ? row + q.step : p.rows;
        const float4 st = stats;
        if (p.stats != nullptr && next < p.rows) stats = reinterpret_cast<const float4*>(p.stats)[next];
        if (!VEC) {
            if (row == q.first) request(row, 0, true);
            if (next < p.rows) request(next, 0, true);
            request(row, 0);
        }
        in.wait();
        const float s_u = st.y, r_y = in.broken ? __int_as_float(0x7fffffff) : st.w;
        float2 m0 = pair(0.f), m1 = pair(0.f), n0, n1;
        Oct kept;                                           // w_pre e, then c t sig
        kept.fill(in.broken ? __int_as_float(0x7fffffff) : 0.f);
        if (has_dz) {
            const float2 k = pair(p.cot_in * r_y);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Quad y = less(in.template get<0>(h), pair(-st.z)), dz = in.template get<2>(h);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int i = 2 * h + j;
                    const float2 e = __fmul2_rn(dz.v[j], k);
                    gw_pre.v[i] = __ffma2_rn(e, y.v[j], gw_pre.v[i]);
                    kept.v[i] = __fmul2_rn(e, w_pre.v[i]);
                    m0 = __ffma2_rn(kept.v[i], y.v[j], m0);
                    if (CENTER) m1 = __fadd2_rn(m1, kept.v[i]);
                }
            }
            means(m0, m1, p.pre, r_y * r_y, n0, n1);
        }
        KeptRow keep;
        if (p.drop.on) keep.draw(p.drop, (uint64_t)row * groups_row, q, seed, step);
        m0 = m1 = pair(0.f);
        const float2 hs = pair(p.h * p.drop.scale * s_u);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            Quad a;
            a.v[0] = kept.v[2 * h]; a.v[1] = kept.v[2 * h + 1];
            if (has_dy) {
                const Quad dy = in.template get<1>(h);
                a.v[0] = __fadd2_rn(a.v[0], dy.v[0]); a.v[1] = __fadd2_rn(a.v[1], dy.v[1]);
            }
            if (has_dz) {
                const Quad y = less(in.template get<0>(h), pair(-st.z));
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (CENTER) a.v[j] = __fadd2_rn(a.v[j], n1);
                    a.v[j] = __ffma2_rn(y.v[j], n0, a.v[j]);
                }
            }
            if (q.n(h) > 0) store4<float, VEC>(p.dy_out + row * p.ld_y + q.col(h), q.n(h), a);
            if (!has_u) continue;
            const Quad u = less(in.template get<3>(h), pair(-st.x));
            Quad g;
            if (has_gate) g = in.template get<4>(h);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int i = 2 * h + j;
                float2 t = __fmul2_rn(a.v[j], hs);
                if (p.drop.on) {
                    if (!keep[2 * i]) t.x = 0.f;
                    if (!keep[2 * i + 1]) t.y = 0.f;
                }
                if (CENTER) {                               // columns that do not exist, which the means would fill
                    if (2 * j >= q.n(h)) t.x = 0.f;
                    if (2 * j + 1 >= q.n(h)) t.y = 0.f;
                }
                float2 x = __fmul2_rn(t, u.v[j]);
                if (has_gate) {
                    float2 slope;
                    const float2 sig = gate_of<T, true>(g.v[j], slope);
                    g.v[j] = __fmul2_rn(__fmul2_rn(x, slope), __fmul2_rn(c.v[i], pair(p.cot_out)));
                    x = __fmul2_rn(x, sig);
                    t = __fmul2_rn(t, sig);
                }
                S.v[i] = __fadd2_rn(S.v[i], x);
                m0 = __ffma2_rn(x, c.v[i], m0);
                kept.v[i] = __fmul2_rn(t, c.v[i]);
                if (CENTER) m1 = __fadd2_rn(m1, kept.v[i]);
            }
            if (has_gate && q.n(h) > 0) {
                if (p.flag != nullptr) largest.see(g, q.n(h));
                store4<T, VEC>((T*)p.dgate + row * p.ld_gate + q.col(h), q.n(h), g);
            }
        }
        if (has_u) {
            means(m0, m1, p.post, s_u * s_u, n0, n1);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                Quad u = less(in.template get<3>(h), pair(-st.x));
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float2 t = kept.v[2 * h + j];
                    if (CENTER) t = __fadd2_rn(t, n1);
                    u.v[j] = __fmul2_rn(__ffma2_rn(u.v[j], n0, t), pair(p.cot_out));
                }
                if (q.n(h) > 0) {
                    if (p.flag != nullptr) largest.see(u, q.n(h));
                    store4<T, VEC>((T*)p.du + row * p.ld_u + q.col(h), q.n(h), u);
                }
            }
        }
        in.sync();                                          // everyone has read this stage
        if (in.leader && row + (long long)in.kStages * q.step < p.rows) request(row + (long long)in.kStages * q.step, in.slot());
        in.done();
        row = next;
    }
    warp_flag_or(p.flag, largest.nonfinite());
    if (p.partial != nullptr) {
        float* out = p.partial + (long long)q.first * 2 * p.width;
        store_row<float, VEC>(out, q, S);
        store_row<float, VEC>(out + p.width, q, gw_pre);
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
            constexpr size_t smem = Rows<T, true, W, C, 2, 3>::kBytes;
            if (!vec) return launch_rows(residual_backward_kernel<T, false, true, W, C>, a, s, 0, st);
            return center ? launch_rows(residual_backward_kernel<T, true, true, W, C>, a, s, smem, st)
                          : launch_rows(residual_backward_kernel<T, true, false, W, C>, a, s, smem, st);
        });
    });
}

int residual_backward_room(mpode_dtype dt, int blocks) {
    static std::atomic<int> known[kMaxDevices][2][kResBlocks + 1];
    return room_of(known, residual_backward_kernel<__nv_bfloat16, true, false, kResWarps, true>, residual_backward_kernel<float, true, false, kResWarps, true>,
                   Rows<__nv_bfloat16, true, kResWarps, true, 2, 3>::kBytes, Rows<float, true, kResWarps, true, 2, 3>::kBytes, dt, blocks);
}

}  // namespace mpode
