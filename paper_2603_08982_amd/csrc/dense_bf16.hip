// Dense attention with masks and its gradients in bf16.
#include "dense_tile.h"

namespace svgear {
int launch_dense_bf16(const DenseArgs& a, int d, int what, hipStream_t s) { return launch_dense<bf16_t>(a, d, what, s); }
}  // namespace svgear
