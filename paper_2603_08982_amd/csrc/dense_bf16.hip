// Dense attention with masks in bf16.
#include "dense_tile.h"

namespace svgear {
int launch_dense_bf16(const DenseArgs& a, int d, hipStream_t s) { return launch_dense<bf16_t, kDenseForward>(a, d, s); }
}  // namespace svgear
