// The Newton-Schulz products in tiles of 192 x 192.
#include "schulz_gemm_kernel.h"

namespace microadam {

hipError_t launch_schulz_gemm_192(const GemmArgs& a, SchulzPhase phase, hipStream_t s) {
  return a.split ? launch_products<192, true>(a, phase, s) : launch_products<192, false>(a, phase, s);
}

}  // namespace microadam
