// Attention by a rule over caches in MXFP8.
#include "paged_attention_scores.h"

namespace torq {

void go_scored_mxfp8(const AttentionPlan &plan, const AttentionArgs &a, bool once, hipStream_t stream) { go_scored<FMT_MXFP8>(plan, a, once, stream); }

}  // namespace torq
