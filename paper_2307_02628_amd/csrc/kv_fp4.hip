// Pages of 4 bits: filed, read back and attended to.
#include "kv_attend.h"
#include "kv_file.h"

namespace skd {

void kv_append_fp4(hipStream_t s, const KvView &kv, const KvTokens &tk, const KvRows &k, const KvRows &v) { append_elem<EL_FP4>(s, kv, tk, k, v); }
void kv_read_fp4(hipStream_t s, const KvView &kv, const KvTokens &tk, bool bf16, const KvRows &k, const KvRows &v) { read_elem<EL_FP4>(s, kv, tk, bf16, k, v); }
void kv_attend_fp4(hipStream_t s, const KvAttend &a, const AttendPlan &p) { attend_elem<EL_FP4, 0>(s, a, p); }

}  // namespace skd
