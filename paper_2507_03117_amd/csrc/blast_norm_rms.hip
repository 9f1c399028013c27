// Gradient of the RMS norms with gate and residual.
#include "norm_backward.h"

int blast::norm_backward_rms(const blast_dev::NormArgs& a, bool vec, hipStream_t stream) {
  return dispatch_backward<false>(a, vec, stream);
}
