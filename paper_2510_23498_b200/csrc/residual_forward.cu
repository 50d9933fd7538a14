// Forward pass of the residual step: z and y' of a row in one pass, the row in registers while its sums meet.
#include "residual.cuh"

namespace mpode {
namespace {

// CENTER: one of the norms takes the mean away
template <typename T, bool VEC, bool CENTER, int WARPS, bool CLUSTER>
__global__ void __launch_bounds__(Lane<WARPS, CLUSTER>::kThreads, 768 / Lane<WARPS, CLUSTER>::kThreads) residual_forward_kernel(const ResArgs p, const int blocks) {
    using Sum = RowSum<1, WARPS, CLUSTER>;
    __shared__ typename Sum::Shared shared;
    const Lane<WARPS, CLUSTER> q(p.width, blocks);
    Sum sum(shared, blocks);
    const uint64_t seed = p.drop.on ? p.drop.rng[0] : 0, step = p.drop.on ? p.drop.rng[1] : 0;
    const int groups_row = (p.width + 7) / 8;
    const float inv = 1.f / (float)p.width;
    // mean and 1 / deviation of the row (zero where no elements exist)
    auto stats_of = [&](const Oct& f, int kind, float& mean, float& rstd) {
        mean = 0.f;
        rstd = 1.f;
        if (kind == MPODE_NORM_NONE) return;
        if (CENTER && kind == MPODE_NORM_MEANVAR) {
            float v[1] = {f.sum()};
            sum(v, q);
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
        sum(v, q);
        rstd = rsqrtf(fmaf(v[0], inv, p.eps));
    };
    int row = q.first;
    // the next row is on its way while this one's sums meet
    Raw8<float> yr;
    Raw8<T> ur, gr;
    auto request = [&](int r) {
        load_raw<float, VEC>(p.y + r * p.ld_y + q.col, q.n, yr);
        if (p.u != nullptr) load_raw<T, VEC>((const T*)p.u + r * p.ld_u + q.col, q.n, ur);
        if (p.gate != nullptr) load_raw<T, VEC>((const T*)p.gate + r * p.ld_gate + q.col, q.n, gr);
    };
    if (row < p.rows) request(row);
    while (row < p.rows) {
        const int next = q.step < p.rows - row ? row + q.step : p.rows;
        float mean_u = 0.f, rstd_u = 1.f, mean_y = 0.f, rstd_y = 1.f;
        Oct y, u, g;
        unpack<float>(yr, y);
        if (p.u != nullptr) unpack<T>(ur, u);
        if (p.gate != nullptr) unpack<T>(gr, g);
        if (next < p.rows) request(next);
        if (p.u != nullptr) {
            Oct w, c;
            Kept keep;
            if (p.drop.on) keep = Kept(p.drop, (uint64_t)row * groups_row + q.col / 8, seed, step);
            stats_of(u, p.post, mean_u, rstd_u);
            load_weights<VEC>(p.w_post, q.col, q.n, w);
            load_weights<VEC>(p.scale, q.col, q.n, c);
            const float2 less = pair(-mean_u), r = pair(rstd_u), h = pair(p.h * p.drop.scale);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float2 v = u.v[j], slope;
                if (CENTER) v = __fadd2_rn(v, less);
                v = __fmul2_rn(__fmul2_rn(v, r), w.v[j]);
                if (p.gate != nullptr) v = __fmul2_rn(v, gate_of<T, false>(g.v[j], slope));
                v = __fmul2_rn(v, __fmul2_rn(h, c.v[j]));
                if (p.drop.on) {
                    if (!keep[2 * j]) v.x = 0.f;
                    if (!keep[2 * j + 1]) v.y = 0.f;
                }
                if (2 * j >= q.n) v.x = 0.f;                 // columns that do not exist stay zero in the sums below
                if (2 * j + 1 >= q.n) v.y = 0.f;
                y.v[j] = __fadd2_rn(y.v[j], v);
            }
        }
        if (p.y_out != nullptr) store8<float, VEC>(p.y_out + row * p.ld_y + q.col, q.n, y);
        if (p.z != nullptr) {
            Oct w;
            stats_of(y, p.pre, mean_y, rstd_y);
            load_weights<VEC>(p.w_pre, q.col, q.n, w);
            const float2 less = pair(-mean_y), r = pair(rstd_y);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (CENTER) y.v[j] = __fadd2_rn(y.v[j], less);
                y.v[j] = __fmul2_rn(__fmul2_rn(y.v[j], r), w.v[j]);
            }
            store8<T, VEC>((T*)p.z + row * p.ld_z + q.col, q.n, y);
        }
        if (p.stats != nullptr && q.col == 0) reinterpret_cast<float4*>(p.stats)[row] = make_float4(mean_u, rstd_u, mean_y, rstd_y);
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
            if (!vec) {
                if constexpr (W == 2 || W == 4) return cudaErrorInvalidValue;
                else return launch_rows(residual_forward_kernel<T, false, true, W, C>, a, s, 0, st);
            }
            return center ? launch_rows(residual_forward_kernel<T, true, true, W, C>, a, s, 0, st) : launch_rows(residual_forward_kernel<T, true, false, W, C>, a, s, 0, st);
        });
    });
}

}  // namespace mpode
