// Host-only stand-ins for the launchers of the attention over the cache and of the
// eviction by accumulated weight: each records its call and the workspace's
// layout instead of enqueueing a kernel.
#include "attention_stubs.hpp"

#include <string.h>

namespace stub {
int attention_calls[kNumAttention];
jacap::AttnLaunch attention;
jacap::AttendSpace attend;
jacap::WeightsSpace lse, sum;
void reset_attention() { memset(attention_calls, 0, sizeof(attention_calls)); }
}  // namespace stub

namespace jacap {

static hipError_t note(int which) {
  ++stub::attention_calls[which];
  return hipSuccess;
}

hipError_t launch_attend(const AttnLaunch& A, const AttendSpace& w, const void*, const void*, const void*,
                         const void*, const void*, void*, float*, const float*) {
  stub::attention = A;
  stub::attend = w;
  return note(stub::kAttend);
}
bool attend_joins(const AttnLaunch&, const AttendSpace& w) { return w.rw == 0 || w.splits > 1; }
hipError_t launch_attend_join(const AttnLaunch&, const AttendSpace&, void*, float*, float*, float*) {
  return note(stub::kJoin);
}
hipError_t launch_attn_lse(const AttnLaunch& A, const WeightsSpace& w, const void*, const void*, const float*,
                           float*) {
  stub::attention = A;
  stub::lse = w;
  return note(stub::kLse);
}
hipError_t launch_attn_sum(const AttnLaunch& A, const WeightsSpace& w, const void*, const void*, const float*,
                           float*, uint32_t*) {
  stub::attention = A;
  stub::sum = w;
  return note(stub::kSum);
}
hipError_t launch_draft_sum(const AttnLaunch&, const void*, const void*, const float*, float*) {
  return note(stub::kDraftSum);
}
hipError_t launch_compact_weighted(const Launch&, const int32_t*, const void*, const void*, void*, void*,
                                   const float*, float*, int64_t, int64_t, int64_t) {
  return note(stub::kCompactWeighted);
}
hipError_t launch_select_empty(const Launch&, float*, int32_t*, int) { return note(stub::kSelectEmpty); }

}  // namespace jacap
