// Dense attention with masks and its gradients in fp32.
#include "dense_tile.h"

namespace svgear {
int launch_dense_f32(const DenseArgs& a, int d, int what, hipStream_t s) { return launch_dense<float>(a, d, what, s); }
}  // namespace svgear
