// Attention over a paged cache: bfloat16.
#include "attend.h"

namespace cfp {

hipError_t attend_bf16(const AttendArgs &A, bool bytes, hipStream_t st) {
  return bytes ? attend_dim<bf16_t, true>(A, st) : attend_dim<bf16_t, false>(A, st);
}

}  // namespace cfp
