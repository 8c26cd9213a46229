// Call records of the attention launchers' stand-ins (attention_stubs.cpp).
#pragma once
#include "attention.hpp"

namespace stub {
enum { kAttend, kJoin, kLse, kSum, kDraftSum, kCompactWeighted, kSelectEmpty, kNumAttention };
extern int attention_calls[kNumAttention];
extern jacap::AttnLaunch attention;   // of the last launch
extern jacap::AttendSpace attend;
extern jacap::WeightsSpace lse, sum;
void reset_attention();
}  // namespace stub
