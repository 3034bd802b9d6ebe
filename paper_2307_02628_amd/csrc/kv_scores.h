// The kernels that a call with changed scores or masks takes, for one kind of page: one for each set of changes, since what a
// kernel does not need costs it registers and time.
#pragma once
#include "kv_attend.h"

namespace skd {

namespace {

template <int EL>
void attend_scored(hipStream_t s, const KvAttend &a, const AttendPlan &p) {
  if (a.sc.capped && a.sc.slopes) attend_elem<EL, SC_MASK | SC_CAP | SC_SLOPES>(s, a, p);
  else if (a.sc.capped) attend_elem<EL, SC_MASK | SC_CAP>(s, a, p);
  else if (a.sc.slopes) attend_elem<EL, SC_MASK | SC_SLOPES>(s, a, p);
  else attend_elem<EL, SC_MASK>(s, a, p);
}

}  // namespace

}  // namespace skd
