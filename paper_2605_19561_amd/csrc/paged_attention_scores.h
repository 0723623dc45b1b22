// The attention kernels whose scores and new tokens go by a rule, of one format (each compiled apart, which takes its time).
#pragma once

#include "paged_attention_body.h"

namespace torq {

template <int DP, int FMT, bool ONCE, int WAYS, int RT, bool SOLO>
__global__ void __launch_bounds__(256) scored_attention_kernel(AttentionArgs a) {
  attention_body<DP, FMT, ONCE, WAYS, RT, SOLO, true>(a);
}

template <int FMT>
void go_scored(const AttentionPlan &plan, const AttentionArgs &a, bool once, hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(plan.groups), dim3(256), 0, stream, a); };
  auto of_hint = [&](auto dp, auto hint) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool ONCE = decltype(hint)::value;
    auto of_launch = [&](auto solo) {
      constexpr bool SOLO = decltype(solo)::value;
      if constexpr (DP <= 128)
        if (plan.rows > ATT_ROWS) {
          if (plan.ways == 1) return go(scored_attention_kernel<DP, FMT, false, 1, 2, SOLO>);
          return go(scored_attention_kernel<DP, FMT, ONCE, ATT_WAVES, 2, SOLO>);
        }
      plan.ways > 1 ? go(scored_attention_kernel<DP, FMT, ONCE, ATT_WAVES, 1, SOLO>) : go(scored_attention_kernel<DP, FMT, ONCE, 1, 1, SOLO>);
    };
    plan.solo ? of_launch(std::true_type{}) : of_launch(std::false_type{});
  };
  auto of_dim = [&](auto dp) {
    // (rows of less than whole lines never go past the cache)
    constexpr int BITS = FMT == FMT_BF16 ? 16 : FMT == FMT_MXFP8 ? 8 : 4;
    if constexpr (decltype(dp)::value * BITS >= 1024)
      if (once) return of_hint(dp, std::true_type{});
    of_hint(dp, std::false_type{});
  };
  if (a.dim <= 64) of_dim(std::integral_constant<int, 64>{});
  else if (a.dim <= 128) of_dim(std::integral_constant<int, 128>{});
  else of_dim(std::integral_constant<int, 256>{});
}

}  // namespace torq
