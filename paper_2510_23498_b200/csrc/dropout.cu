// Dropout whose mask is never stored: the call that is given the cotangent with the same {seed, step}, site and shape is its backward pass,
// and a recompute of the stages (Alg. 2) finds the forward pass's mask again.
#include "operators.h"
#include "philox.cuh"
#include "rows.cuh"

namespace mpode {
namespace {

struct DropArgs {
    const void* x; void* out;
    long long ld_x, ld_out, groups;      // groups of eight columns in all rows
    int width, groups_row;
    Dropout d;
    unsigned* flag;
};

// One thread, one group of eight columns at a time: 16-byte accesses where the layout allows.  FLAT: rows of whole groups one behind the other, where a
// group's place needs no division.  Bound by the generator's wide products beside the bytes: 8192 x 8192 bfloat16 take 57 us (41 for the bytes alone), with one, two or
// four groups in flight alike.  Eight blocks an SM in 32 registers where that needs no memory for them (six: 60 us).
template <typename T, bool VEC, bool FLAT> __global__ void __launch_bounds__(256, VEC && sizeof(T) == 2 ? 8 : 6) dropout_kernel(const DropArgs p) {
    const uint64_t seed = p.d.rng[0], step = p.d.rng[1];
    Largest<T> largest;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < p.groups; i += (long long)gridDim.x * 256) {
        long long from = i * 8, to = i * 8;
        int n = 8;
        if (!FLAT) {
            const long long row = i / p.groups_row;
            const int col = (int)(i - row * p.groups_row) * 8;
            n = min(8, p.width - col);
            from = row * p.ld_x + col;
            to = row * p.ld_out + col;
        }
        Oct o;
        load8<T, VEC>((const T*)p.x + from, n, o);
        const Kept keep(p.d, (uint64_t)i, seed, step);
        const float2 s = make_float2(p.d.scale, p.d.scale);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            o.v[j] = __fmul2_rn(o.v[j], s);
            if (p.d.on && !keep[2 * j]) o.v[j].x = 0.f;
            if (p.d.on && !keep[2 * j + 1]) o.v[j].y = 0.f;
        }
        Raw8<T> r;
        pack<T>(o, r);
        store_raw<T, VEC>((T*)p.out + to, n, r);
        if (p.flag != nullptr) largest.see(r, n);
    }
    warp_flag_or(p.flag, largest.nonfinite());
}

}  // namespace
}  // namespace mpode

using namespace mpode;

extern "C" mpode_status mpode_dropout(mpode_dtype low, void* cuda_stream, long long rows, int width, const void* x_dev, long long ld_x, void* out_dev,
                                      long long ld_out, float p, const void* rng_dev, unsigned site, unsigned* flag_dev) {
    if (!known_dtype(low)) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_dropout: unknown format %d", (int)low);
    if (rows < 0 || width < 1) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_dropout: %lld rows of width %d", rows, width);
    if (!(p >= 0.f && p <= 1.f)) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_dropout: p = %g is not a probability", (double)p);
    if (ld_x == 0) ld_x = width;
    if (ld_out == 0) ld_out = width;
    if (ld_x < width || ld_out < width) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_dropout: rows overlap");
    if (rows == 0) return MPODE_OK;
    if (rows > (1ll << 40)) return operator_fail(MPODE_ERR_UNSUPPORTED, "mpode_dropout: %lld rows", rows);
    if (!x_dev || !out_dev || !rng_dev) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_dropout: null pointer argument");
    if (x_dev == out_dev && ld_x != ld_out && rows > 1) return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_dropout: out over x with other strides");
    const size_t es = low_size(low);
    if (misaligned(x_dev, es) || misaligned(out_dev, es) || misaligned(rng_dev, 8) || misaligned(flag_dev, 4))
        return operator_fail(MPODE_ERR_INVALID_ARG, "mpode_dropout: a pointer is not aligned to its elements");
    DropArgs a{x_dev, out_dev, ld_x, ld_out, 0, width, width / 8 + (width % 8 != 0), make_dropout(p, rng_dev, site), flag_dev};
    a.groups = rows * a.groups_row;
    const bool vec = width % 8 == 0 && !misaligned(x_dev, 16) && !misaligned(out_dev, 16) && (ld_x * es) % 16 == 0 && (ld_out * es) % 16 == 0;
    const long long blocks = (a.groups + 255) / 256, most = 148 * 16;
    const unsigned grid = (unsigned)(blocks < most ? blocks : most);
    return operator_launched(with_low(low, [&](auto t) {
        using T = decltype(t);
        const cudaStream_t st = (cudaStream_t)cuda_stream;
        if (vec && ld_x == width && ld_out == width) return launch_grid(dropout_kernel<T, true, true>, grid, 256, st, a);
        if (vec) return launch_grid(dropout_kernel<T, true, false>, grid, 256, st, a);
        return launch_grid(dropout_kernel<T, false, false>, grid, 256, st, a);
    }), "mpode_dropout");
}
