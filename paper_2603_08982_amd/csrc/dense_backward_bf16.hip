// The gradients of dense attention with masks in bf16: without a cap, and with caps up to kFarCap.
#include "dense_backward_bf16.h"

namespace svgear {
namespace {

template <int D>
int launch(const DenseArgs& a, int what, hipStream_t s) {
  return by_scores(a, [&](auto cap, auto slopes) -> int { return launch_gradients<D, decltype(cap)::value, decltype(slopes)::value>(a, what, s); });
}

}  // namespace

int launch_dense_backward_bf16(const DenseArgs& a, int d, int what, hipStream_t s) {
  if (a.cap > kFarCap) return launch_dense_backward_far_cap(a, d, what, s);
  return d == 64 ? launch<64>(a, what, s) : launch<128>(a, what, s);
}
}  // namespace svgear
