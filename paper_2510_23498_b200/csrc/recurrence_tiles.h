// Which tiles of a sequence the recurrence's bulk copies bring to shared memory.
#pragma once

namespace mpode {

// A copy brings a tile of `steps` rows; the tensor clips it at row 0 and at n_steps, but knows nothing of a sequence's length.  Tiles that would reach behind
// a length are therefore not copied: the lanes read the rows that exist.
//
// Forward: the tiles of a warp lie at base + from, base = 0, stride, ...  Those with base below the result touch no row behind len.
__host__ __device__ inline unsigned copied_below(unsigned from, unsigned steps, unsigned len, unsigned n_steps) {
    if (len == n_steps) return len;
    return len >= from + steps ? len - from - steps + 1 : 0u;
}
// Backward: steps are counted from n_steps - 1 down, of which the first `skipped` do not exist; tile of the steps from `first` on in that count.
__host__ __device__ inline bool copied_back(unsigned first, unsigned skipped) { return first >= skipped; }

}  // namespace mpode
