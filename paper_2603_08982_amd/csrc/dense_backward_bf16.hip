// The gradients of dense attention with masks in bf16.
#include "dense_tile.h"

namespace svgear {
int launch_dense_backward_bf16(const DenseArgs& a, int d, int what, hipStream_t s) {
  return what == kDenseDq ? launch_dense<bf16_t, kDenseDq>(a, d, s) : launch_dense<bf16_t, kDenseDkv>(a, d, s);
}
}  // namespace svgear
