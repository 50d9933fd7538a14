// Forward pass of the residual step: z and y' of a row in one pass.  The row's inputs lie in shared memory, where the sum over u and the step read them; y' stays
// in registers while its sum meets.  Four blocks of 8 warps an SM hide one's sums behind another's arithmetic.
#include "residual.cuh"

namespace mpode {
namespace {

// CENTER: one of the norms takes the mean away
template <typename T, bool VEC, bool CENTER, int WARPS, bool CLUSTER>
__global__ void __launch_bounds__(Lane<WARPS, CLUSTER>::kThreads, 1024 / Lane<WARPS, CLUSTER>::kThreads) residual_forward_kernel(const ResArgs p, const int blocks) {
    using Sum = RowSum<1, WARPS, CLUSTER>;
    using In = Rows<T, VEC, WARPS, CLUSTER, 1, 2>;          // y, u, gate
    extern __shared__ __align__(16) char staged[];
    __shared__ typename Sum::Shared shared;
    const Lane<WARPS, CLUSTER> q(p.width, blocks);
    Sum sum(shared, blocks);
    In in(staged, q);
    const uint64_t seed = p.drop.on ? p.drop.rng[0] : 0, step = p.drop.on ? p.drop.rng[1] : 0;
    const int groups_row = (p.width + 7) / 8;
    const float inv = 1.f / (float)p.width;
    const bool has_u = p.u != nullptr, has_gate = p.gate != nullptr;
    auto request = [&](long long r, int stage, bool ahead = false) {
        const void* const from[3] = {p.y + r * p.ld_y + q.base, has_u ? (const T*)p.u + r * p.ld_u + q.base : nullptr,
                                     has_gate ? (const T*)p.gate + r * p.ld_gate + q.base : nullptr};
        if (ahead) in.touch(from);
        else in.request(stage, from);
    };
    if (in.leader)
        for (int k = 0; k < in.kStages; ++k)
            if (q.first + (long long)k * q.step < p.rows) request(q.first + (long long)k * q.step, k);
    Oct w_pre = weights_of<VEC>(p.w_pre, q), c = weights_of<VEC>(p.scale, q);        // c = scale w_post
    {
        const Oct w_post = weights_of<VEC>(p.w_post, q);
#pragma unroll
        for (int k = 0; k < 4; ++k) c.v[k] = __fmul2_rn(c.v[k], w_post.v[k]);
    }
    // less the mean, zero where no columns exist
    auto less = [&](float2 v, float mean, int i) {
        v = __fadd2_rn(v, pair(-mean));
        if (2 * (i & 1) >= q.n(i >> 1)) v.x = 0.f;
        if (2 * (i & 1) + 1 >= q.n(i >> 1)) v.y = 0.f;
        return v;
    };
    auto total = [&](float2 f) {
        float v[1] = {f.x + f.y};
        sum(v, q);
        return v[0] * inv;
    };
    int row = q.first;
    while (row < p.rows) {
        const int next = q.step < p.rows - row ? row + q.step : p.rows;
        float mean_u = 0.f, rstd_u = 1.f, mean_y = 0.f, rstd_y = 1.f;
        if (!VEC) {
            if (row == q.first) request(row, 0, true);
            if (next < p.rows) request(next, 0, true);
            request(row, 0);
        }
        in.wait();
        Oct y;
        if (has_u) {
            if (CENTER && p.post == MPODE_NORM_MEANVAR) {
                float2 s = pair(0.f);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const Quad u = in.template get<1>(h);
                    s = __fadd2_rn(s, __fadd2_rn(u.v[0], u.v[1]));
                }
                mean_u = total(s);
            }
            if (p.post != MPODE_NORM_NONE) {
                float2 s = pair(0.f);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    Quad u = in.template get<1>(h);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (CENTER) u.v[j] = less(u.v[j], mean_u, 2 * h + j);
                        s = __ffma2_rn(u.v[j], u.v[j], s);
                    }
                }
                rstd_u = rsqrtf(total(s) + p.eps);
            }
            KeptRow keep;
            if (p.drop.on) keep.draw(p.drop, (uint64_t)row * groups_row, q, seed, step);
            const float2 k = pair(p.h * p.drop.scale * rstd_u);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Quad u = in.template get<1>(h), yh = in.template get<0>(h);
                Quad g;
                if (has_gate) g = in.template get<2>(h);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int i = 2 * h + j;
                    float2 v = u.v[j], slope;
                    if (CENTER) v = less(v, mean_u, i);
                    v = __fmul2_rn(__fmul2_rn(v, k), c.v[i]);
                    if (has_gate) v = __fmul2_rn(v, gate_of<T, false>(g.v[j], slope));
                    if (p.drop.on) {
                        if (!keep[2 * i]) v.x = 0.f;
                        if (!keep[2 * i + 1]) v.y = 0.f;
                    }
                    y.v[i] = __fadd2_rn(yh.v[j], v);
                }
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Quad yh = in.template get<0>(h);
                y.v[2 * h] = yh.v[0];
                y.v[2 * h + 1] = yh.v[1];
            }
        }
        if (in.broken) y.fill(__int_as_float(0x7fffffff));
        in.sync();                                          // everyone has read this stage
        if (in.leader && row + (long long)in.kStages * q.step < p.rows) request(row + (long long)in.kStages * q.step, in.slot());
        in.done();
        if (p.y_out != nullptr) store_row<float, VEC>(p.y_out + row * p.ld_y, q, y);
        if (p.z != nullptr) {
            if (CENTER && p.pre == MPODE_NORM_MEANVAR) mean_y = total(__fadd2_rn(__fadd2_rn(y.v[0], y.v[1]), __fadd2_rn(y.v[2], y.v[3])));
            if (p.pre != MPODE_NORM_NONE) {
                float2 s = pair(0.f);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (CENTER) y.v[i] = less(y.v[i], mean_y, i);
                    s = __ffma2_rn(y.v[i], y.v[i], s);
                }
                rstd_y = rsqrtf(total(s) + p.eps);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) y.v[i] = __fmul2_rn(__fmul2_rn(y.v[i], pair(rstd_y)), w_pre.v[i]);
            store_row<T, VEC>((T*)p.z + row * p.ld_z, q, y);
        }
        if (p.stats != nullptr && q.col(0) == 0) reinterpret_cast<float4*>(p.stats)[row] = make_float4(mean_u, rstd_u, mean_y, rstd_y);
        row = next;
    }
    sum.end();
}

}  // namespace

cudaError_t launch_residual_forward(mpode_dtype dt, const ResArgs& a, const ResShape& s, bool vec, bool center, cudaStream_t st) {
    return with_low(dt, [&](auto t) {
        using T = decltype(t);
        return with_shape(s, [&](auto warps, auto cluster) {
            constexpr int W = warps.value;
            constexpr bool C = cluster.value;
            constexpr size_t smem = Rows<T, true, W, C, 1, 2>::kBytes;
            if (!vec) return launch_rows(residual_forward_kernel<T, false, true, W, C>, a, s, 0, st);
            return center ? launch_rows(residual_forward_kernel<T, true, true, W, C>, a, s, smem, st)
                          : launch_rows(residual_forward_kernel<T, true, false, W, C>, a, s, smem, st);
        });
    });
}

int residual_forward_room(mpode_dtype dt, int blocks) {
    static std::atomic<int> known[kMaxDevices][2][kResBlocks + 1];
    return room_of(known, residual_forward_kernel<__nv_bfloat16, true, false, kResWarps, true>, residual_forward_kernel<float, true, false, kResWarps, true>,
                   Rows<__nv_bfloat16, true, kResWarps, true, 1, 2>::kBytes, Rows<float, true, kResWarps, true, 1, 2>::kBytes, dt, blocks);
}

}  // namespace mpode
