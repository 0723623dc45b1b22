// Attention by a rule over caches in MXFP4.
#include "paged_attention_scores.h"

namespace torq {

void go_scored_mxfp4(const AttentionPlan &plan, const AttentionArgs &a, bool once, hipStream_t stream) { go_scored<FMT_MXFP4>(plan, a, once, stream); }

}  // namespace torq
