// Attention with changed scores and masks over pages of bf16 and 8 bits.
#include "kv_attend.h"

namespace skd {

void kv_attend_scored(hipStream_t s, const KvAttend &a, const AttendPlan &p) {
  if (a.kv.fp8) attend_elem<EL_FP8, true>(s, a, p);
  else attend_elem<EL_BF16, true>(s, a, p);
}

}  // namespace skd
