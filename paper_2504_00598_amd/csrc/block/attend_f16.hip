// Attention over a paged cache: float16.
#include "attend.h"

namespace cfp {

hipError_t attend_f16(const AttendArgs &A, bool bytes, hipStream_t st) {
  return bytes ? attend_dim<f16_t, true>(A, st) : attend_dim<f16_t, false>(A, st);
}

}  // namespace cfp
