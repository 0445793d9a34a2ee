// The matrix products of svgear_linear and its backward pass in fp32.
#include "linear_tile.h"

namespace svgear {

int launch_linear_f32(const LinearArgs& a, int form, hipStream_t s) { return launch_linear<float>(a, form, s); }

}  // namespace svgear
