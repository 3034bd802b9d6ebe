// Attention with changed scores and masks over pages of bf16.
#include "kv_scores.h"

namespace skd {
void kv_attend_scored_bf16(hipStream_t s, const KvAttend &a, const AttendPlan &p) { attend_scored<EL_BF16>(s, a, p); }
}  // namespace skd
