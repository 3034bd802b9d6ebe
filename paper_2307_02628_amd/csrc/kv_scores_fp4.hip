// Attention with changed scores and masks over pages of 4 bits.
#include "kv_scores.h"

namespace skd {
void kv_attend_scored_fp4(hipStream_t s, const KvAttend &a, const AttendPlan &p) { attend_scored<EL_FP4>(s, a, p); }
}  // namespace skd
