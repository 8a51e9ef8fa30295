// A warp's ring of copies: which ones are under way.  Without CUDA, so that it can be tested alone.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define PSKV_HD __host__ __device__ __forceinline__
#else
#define PSKV_HD inline
#endif

namespace pskv {

// Waits for every copy that is still under way, the one of the present stage first: `in_flight` copies that have not been
// used, in the order in which they were issued.  wait(stage, parity of its barrier's phase).
template <uint32_t STAGES, class Wait>
PSKV_HD void drain_ring(uint32_t stage, uint32_t phase, uint32_t in_flight, Wait wait) {
  for (; in_flight; --in_flight) {
    wait(stage, phase);
    if (++stage == STAGES) {
      stage = 0;
      phase ^= 1u;
    }
  }
}

}  // namespace pskv
