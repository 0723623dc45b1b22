// Attention by a rule over caches in BF16.
#include "paged_attention_scores.h"

namespace torq {

void go_scored_bf16(const AttentionPlan &plan, const AttentionArgs &a, bool once, hipStream_t stream) { go_scored<FMT_BF16>(plan, a, once, stream); }

}  // namespace torq
