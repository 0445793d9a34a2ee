// Dense attention with masks in fp32.
#include "dense_tile.h"

namespace svgear {
int launch_dense_f32(const DenseArgs& a, int d, hipStream_t s) { return launch_dense<float, kDenseForward>(a, d, s); }
}  // namespace svgear
