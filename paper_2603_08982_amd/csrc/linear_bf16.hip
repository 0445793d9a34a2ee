// The matrix products of svgear_linear and its backward pass in bf16.
#include "linear_tile.h"

namespace svgear {

int launch_linear_bf16(const LinearArgs& a, int form, hipStream_t s) { return launch_linear<bf16_t>(a, form, s); }

}  // namespace svgear
