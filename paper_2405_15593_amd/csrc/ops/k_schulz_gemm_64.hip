// The Newton-Schulz products in tiles of 64 x 64.
#include "schulz_gemm_kernel.h"

namespace microadam {

hipError_t launch_schulz_gemm_64(const GemmArgs& a, SchulzPhase phase, hipStream_t s) {
  return a.split ? launch_products<64, true>(a, phase, s) : launch_products<64, false>(a, phase, s);
}

}  // namespace microadam
