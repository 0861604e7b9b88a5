// wide_range.h - the scale of probabilities whose sums or maximum leave float32.
#pragma once

#include "attn_tile.h"

namespace ditango {
namespace {

// Rows whose scores or values are so large that sums of unnormalised
// probabilities, or a maximum rounded after its scaling, leave float32: their
// probabilities are taken as 2^low exp2(scale (s - mx)) against the maximum mx of
// the scores as they are, with low such that sums over n keys, and over eight
// waves' partial sums, stay below the largest value they weigh; and the maximum
// that such a state is against (base 2, scaled).
__device__ __forceinline__ float wide_low(int n) { return (float)(__builtin_clz(n | 1) - 35); }
__device__ __forceinline__ float wide_max(float mx, float sl2, float low) {
  return mx == -INFINITY ? mx : fminf(fmaxf(mx * sl2, -0x1.fffffep127f), 0x1.fffffep127f) - low;
}

}  // namespace
}  // namespace ditango
