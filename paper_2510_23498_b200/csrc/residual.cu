// One forward Euler step of the float32 state around a block that the caller evaluates, with the norms on both sides of the block:
//     n = N_post(u),  y' = y + h scale * drop(sigmoid(gate) * w_post n),  z = Q16(w_pre N_pre(y')),
// u the block's output and z the next block's input, and the step's backward pass.  N: none, v / sqrt(mean(v^2) + eps), or the same of v - mean(v).
//
// This file: argument checks, how rows are spread over the GPU, and the weights' gradients' last sums; the passes are in residual_forward.cu and
// residual_backward.cu.  Bound by the bytes of its rows (16-bit formats: 14 an element forward, 22 backward): a row is read once from memory and
// written once.  Eight columns a thread, in two fours (neighbouring lanes share the generator's counters); a row takes one warp up to 256 columns, a block of
// up to 8 warps up to 2048, and a cluster of up to 8 blocks beyond that, whose partial sums meet in distributed shared memory.  All sums, statistics,
// gates and gradients are float32; what is stored in the low format is rounded once, when it is written.
#include "residual.cuh"

namespace mpode {
namespace {

// The weights' gradients from the partial rows [rows][2][width], summed in a fixed order: 8 columns (a 32-byte sector of each row) and 64 slices of the rows a
// block.  dw_post = scale S, dscale = w_post S, dw_pre.
struct FinishArgs { const float *partial, *w_post, *scale; float *dw_post, *dscale, *dw_pre; int rows, width, accumulate; };
__global__ void __launch_bounds__(512) residual_finish_kernel(const FinishArgs p) {
    __shared__ float part[64][9];
    chain_begin();
    const int c = threadIdx.x & 7, slice = threadIdx.x >> 3;
    const int i = blockIdx.x * 8 + c;                       // column of the two sums side by side
    float s = 0.f;
    if (i < 2 * p.width) {
#pragma unroll 4
        for (int r = slice; r < p.rows; r += 64) s += p.partial[(long long)r * 2 * p.width + i];
    }
    part[slice][c] = s;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    // 4 lanes a column, 16 slices each, then the four
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += part[(threadIdx.x >> 3) * 16 + k][c];
    s += __shfl_xor_sync(0xffffffffu, s, 8);
    s += __shfl_xor_sync(0xffffffffu, s, 16);
    if (threadIdx.x >= 8 || i >= 2 * p.width) return;
    auto put = [&](float* out, float v) {
        if (out != nullptr) *out = (p.accumulate ? *out : 0.f) + v;
    };
    if (i >= p.width) put(p.dw_pre == nullptr ? nullptr : p.dw_pre + (i - p.width), s);
    else {
        put(p.dw_post == nullptr ? nullptr : p.dw_post + i, p.scale == nullptr ? s : s * p.scale[i]);
        put(p.dscale == nullptr ? nullptr : p.dscale + i, p.w_post == nullptr ? s : s * p.w_post[i]);
    }
}

// at_once: clusters (of one warp row each) that the GPU is to hold
ResShape shape_of(int rows, int width, int at_once) {
    ResShape s;
    s.blocks = (width + kResWarps * 256 - 1) / (kResWarps * 256);
    s.warps = 1;
    while (s.warps * 256 < width && s.warps < kResWarps) s.warps *= 2;
    s.groups = s.warps == 1 ? kResGroups : 1;
    const int need = rows / s.groups + (rows % s.groups != 0);
    int most = at_once * (s.warps >= 8 || s.warps == 1 ? 1 : 8 / s.warps);
    most = most / s.blocks > 0 ? most / s.blocks : 1;
    s.clusters = need < most ? need : most;
    return s;
}
// Blocks of 8 warps: what an SM holds of 16-bit rows.  (Not everywhere: backward it holds two of float32 rows above 1024 columns, whose stages take 80 KB, and two of
// eight rows of one warp, with 122 to 126 registers a thread; the third then runs behind them.)
constexpr int kForwardBlocks = 148 * 4, kBackwardBlocks = 148 * 3;

mpode_status check(const mpode_residual_desc* d, int rows, const char* who) {
    if (d == nullptr) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: null descriptor", who);
    if (!known_dtype(d->low)) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: unknown format %d", who, (int)d->low);
    for (int k : {(int)d->post_norm, (int)d->pre_norm})
        if (k < MPODE_NORM_NONE || k > MPODE_NORM_MEANVAR) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: unknown norm %d", who, k);
    if (d->width < 1 || rows < 0) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: %d rows of width %d", who, rows, d->width);
    if (d->width > kResMaxWidth) return operator_fail(MPODE_ERR_UNSUPPORTED, "%s: width %d is above %d", who, d->width, kResMaxWidth);
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

// no more clusters than run at once (4096 x 8192 bfloat16 backward: 111 of 4 blocks fill the SMs' registers, 104 fit the GPU's groups of SMs)
ResShape within(ResShape s, int room) {
    if (s.blocks > 1 && room > 0 && s.clusters > room) s.clusters = room;
    return s;
}

// Rows of partial sums a backward pass leaves at most
size_t partial_rows(int rows, int width) {
    const ResShape s = shape_of(rows, width, kBackwardBlocks);
    return (size_t)s.clusters * s.groups;
}

}  // namespace
}  // namespace mpode

using namespace mpode;

extern "C" {

size_t mpode_residual_workspace_bytes(const mpode_residual_desc* desc, int rows) {
    if (check(desc, rows, "mpode_residual_workspace_bytes") != MPODE_OK || rows == 0) return 0;
    return partial_rows(rows, desc->width) * 2 * desc->width * sizeof(float);
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
    ResShape s = shape_of(rows, desc->width, kForwardBlocks);
    if (s.blocks > 1) s = within(s, residual_forward_room(desc->low, s.blocks));
    return operator_launched(launch_residual_forward(desc->low, a, s, vec, center(*desc), (cudaStream_t)cuda_stream),
                             "mpode_residual_forward");
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
    const auto meet = [&](const float* p, const float* q) { return p && q && p < q + desc->width && q < p + desc->width; };
    const bool shared = meet(dL_dw_post_dev, dL_dscale_dev) || meet(dL_dw_post_dev, dL_dw_pre_dev) || meet(dL_dscale_dev, dL_dw_pre_dev);
    if (shared && !accumulate) return operator_fail(MPODE_ERR_INVALID_ARG, "%s: weight gradients in one another's place (they can be added there: accumulate)", who);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    int partials = 0;
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
        ResShape s = shape_of(rows, desc->width, kBackwardBlocks);
        if (s.blocks > 1) s = within(s, residual_backward_room(desc->low, s.blocks));
        partials = s.clusters * s.groups;
        const mpode_status ran = operator_launched(launch_residual_backward(desc->low, a, s, vec, center(*desc), st), who);
        if (ran != MPODE_OK || !weights) return ran;
    }
    if (!weights) return MPODE_OK;
    FinishArgs f{a.partial, w_post_dev, scale_dev, dL_dw_post_dev, dL_dscale_dev, dL_dw_pre_dev, partials, desc->width, accumulate};
    const auto finish = [&] { return operator_launched(launch_chain(residual_finish_kernel, dim3((2 * desc->width + 7) / 8), dim3(512), 0, st, f), who); };
    if (!shared) return finish();
    // one sum after another into the buffer that they share
    for (int k = 0; k < 3; ++k) {
        f.dw_post = k == 0 ? dL_dw_post_dev : nullptr;
        f.dscale = k == 1 ? dL_dscale_dev : nullptr;
        f.dw_pre = k == 2 ? dL_dw_pre_dev : nullptr;
        const mpode_status s = f.dw_post || f.dscale || f.dw_pre ? finish() : MPODE_OK;
        if (s != MPODE_OK) return s;
    }
    return MPODE_OK;
}

}  // extern "C"
