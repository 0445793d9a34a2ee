// The gradients of dense attention with masks in bf16 with caps over kFarCap.
#include "dense_backward_bf16.h"

namespace svgear {
namespace {

template <int D>
int launch(const DenseArgs& a, int what, hipStream_t s) {
  return a.slopes ? launch_gradients<D, kCapFar, true>(a, what, s) : launch_gradients<D, kCapFar, false>(a, what, s);
}

}  // namespace

int launch_dense_backward_far_cap(const DenseArgs& a, int d, int what, hipStream_t s) { return d == 64 ? launch<64>(a, what, s) : launch<128>(a, what, s); }
}  // namespace svgear
