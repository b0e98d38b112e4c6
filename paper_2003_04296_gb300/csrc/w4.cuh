// w4.cuh -- products with 4-bit weights, for other translation units.
#pragma once

#include "common.cuh"

namespace minw {
namespace w4 {

// The checks of minw_w4_matvec.
minw_status check(const void *x, int x_type, int64_t ldx, int64_t T, const uint8_t *codes, const uint16_t *scales, int O, int K,
                  int group, const float *scale, const float *shift, int act, const void *y, int y_type, int64_t ldy);

// minw_w4_matvec of checked arguments, T > 0.  add (nullable): fp32 [T][O], added to the products before scale and shift; the
// kernel before it in the stream wrote it, and let this one start only once all before itself was done, so that
// the products begin while it runs.
minw_status matvec(const void *x, int x_type, int64_t ldx, int T, const uint8_t *codes, const uint16_t *scales, int O, int K,
                   int group, const float *scale, const float *shift, int act, void *y, int y_type, int64_t ldy,
                   const float *add, cudaStream_t s);

}  // namespace w4
}  // namespace minw
