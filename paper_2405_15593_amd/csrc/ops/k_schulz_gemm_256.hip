// The Newton-Schulz products in tiles of 256 x 256.
#include "schulz_gemm_kernel.h"

namespace microadam {

hipError_t launch_schulz_gemm_256(const GemmArgs& a, SchulzPhase phase, hipStream_t s) {
  if (a.split) return hipErrorInvalidValue;  // its results would not fit the registers
  return launch_products<256, false>(a, phase, s);
}

}  // namespace microadam
