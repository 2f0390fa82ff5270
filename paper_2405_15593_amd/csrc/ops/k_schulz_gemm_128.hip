// The Newton-Schulz products in tiles of 128 x 128.
#include "schulz_gemm_kernel.h"

namespace microadam {

hipError_t launch_schulz_gemm_128(const GemmArgs& a, SchulzPhase phase, hipStream_t s) {
  return a.split ? launch_products<128, true>(a, phase, s) : launch_products<128, false>(a, phase, s);
}

}  // namespace microadam
