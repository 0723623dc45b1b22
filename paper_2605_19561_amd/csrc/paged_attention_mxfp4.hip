// torq_paged_attention over caches in MXFP4: the kernels of paged_attention_body.h that widen E2M1 codes with their scale, two of them in an
// instruction.
#include "paged_attention_body.h"

namespace torq {

template <int DP, bool ONCE, int WAYS, int RT, bool SOLO>
__global__ void __launch_bounds__(256) paged_attention4_kernel(AttentionArgs a) {
  attention_body<DP, FMT_MXFP4, ONCE, WAYS, RT, SOLO, false>(a);
}

void go_attention4(const AttentionPlan &plan, const AttentionArgs &a, bool once, hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(plan.groups), dim3(256), 0, stream, a); };
  auto of_hint = [&](auto dp, auto hint) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool ONCE = decltype(hint)::value;
    auto of_launch = [&](auto solo) {
      constexpr bool SOLO = decltype(solo)::value;
      if constexpr (DP <= 128)
        if (plan.rows > ATT_ROWS) {
          if (plan.ways == 1) return go(paged_attention4_kernel<DP, false, 1, 2, SOLO>);
          return go(paged_attention4_kernel<DP, ONCE, ATT_WAVES, 2, SOLO>);
        }
      plan.ways > 1 ? go(paged_attention4_kernel<DP, ONCE, ATT_WAVES, 1, SOLO>) : go(paged_attention4_kernel<DP, ONCE, 1, 1, SOLO>);
    };
    plan.solo ? of_launch(std::true_type{}) : of_launch(std::false_type{});
  };
  if (a.dim <= 64) of_hint(std::integral_constant<int, 64>{}, std::false_type{});
  else if (a.dim <= 128) of_hint(std::integral_constant<int, 128>{}, std::false_type{});
  else if (once) of_hint(std::integral_constant<int, 256>{}, std::true_type{});
  else of_hint(std::integral_constant<int, 256>{}, std::false_type{});
}

}  // namespace torq
