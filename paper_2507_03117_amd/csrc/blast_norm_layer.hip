// Gradient of the layer norms with gate and residual.
#include "norm_backward.h"

int blast::norm_backward_layer(const blast_dev::NormArgs& a, bool vec, hipStream_t stream) {
  return dispatch_backward<true>(a, vec, stream);
}
