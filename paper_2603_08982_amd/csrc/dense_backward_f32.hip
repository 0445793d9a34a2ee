// The gradients of dense attention with masks in fp32.
#include "dense_tile.h"

namespace svgear {
int launch_dense_backward_f32(const DenseArgs& a, int d, int what, hipStream_t s) {
  return what == kDenseDq ? launch_dense<float, kDenseDq>(a, d, s) : launch_dense<float, kDenseDkv>(a, d, s);
}
}  // namespace svgear
