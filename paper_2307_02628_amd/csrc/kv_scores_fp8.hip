// Attention with changed scores and masks over pages of 8 bits.
#include "kv_scores.h"

namespace skd {
void kv_attend_scored_fp8(hipStream_t s, const KvAttend &a, const AttendPlan &p) { attend_scored<EL_FP8>(s, a, p); }
}  // namespace skd
