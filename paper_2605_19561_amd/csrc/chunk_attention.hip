// torq_chunk_attention: who runs which kernel of chunk_attention_body.h, and the join of their parts.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "chunk_attention_body.h"

namespace torq {

// The parts of a row tile's rows put together in the order of the keys: a thread takes four values of a row.
__global__ void __launch_bounds__(256) chunk_join_kernel(ChunkArgs a) {
  const int kv_head = blockIdx.x % a.kv_heads, slot = blockIdx.x / a.kv_heads;
  RowTile it;
  if (!row_tile_of(a, slot, it)) return;
  const int row_tile = it.tile, rows = min(it.rows_there, a.rule.most) * a.rule.heads_each, quads = a.dim / 4;
  const int64_t part0 = ((int64_t)slot * a.kv_heads + kv_head) * a.splits * a.tile_rows;
  for (int x = blockIdx.y * 256 + threadIdx.x; x < a.tile_rows * quads; x += gridDim.y * 256) {
    const int r = x / quads, c = x - r * quads;
    if (row_tile * a.tile_rows + r >= rows) break;
    float top = -INFINITY;
    for (int i = 0; i < a.splits; ++i) top = fmaxf(top, a.part_ml[2 * (part0 + (int64_t)i * a.tile_rows + r)]);
    const float base = top == -INFINITY ? 0.0f : top;
    float l = 0.0f;
    f32x4 v = {0, 0, 0, 0};
#pragma unroll 4
    for (int i = 0; i < a.splits; ++i) {
      const int64_t part = part0 + (int64_t)i * a.tile_rows + r;
      const float f = __builtin_amdgcn_exp2f(a.part_ml[2 * part] - base);
      l += f * a.part_ml[2 * part + 1];
      v += f * *reinterpret_cast<const f32x4 *>(a.part + part * a.dim + 4 * c);
    }
    v *= l != 0.0f ? 1.0f / l : 0.0f;
    uint16_t *const out = a.out + ruled_row(a, it.q_at, kv_head, row_tile * a.tile_rows + r) * a.dim;
    *reinterpret_cast<bf16x4 *>(out + 4 * c) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
  }
}

namespace {
// So few rows of a request that they are columns of the single token's kernels
bool few_rows(const torq_kv_cache_t &cache, int heads, int most) { return (int64_t)(heads / cache.heads) * most <= 32; }
// A cap whose tangent may be taken in the short form, off by 2^-23 of the cap: below 2^-15 of a weight.
bool short_cap(const torq_scores_t *scores) { return scores->cap <= 177.0f; }
// What the kernel does to scores ahead of the weights: such a cap, or slopes; any other rule, and a scale of 0 or nearly (0 times minus infinity is
// none: times it ahead of the maximum) by the kernel that looks.
int bend_of(float scale, const torq_scores_t *scores) {
  const bool cap = scores && scores->cap > 0.0f, slopes = scores && scores->slopes;
  if (cap) return slopes || !short_cap(scores) ? BEND_ANY : BEND_CAP;
  return slopes ? BEND_SLOPES : std::fabs(scale) < 2.0f * FLT_MIN ? BEND_ANY : BEND_NONE;
}
struct ChunkPlan {
  int64_t slots, items;
  int splits, rows;
};
// Rows of a workgroup: 64 where a request has no more, whose four waves then share the keys out.
int rows_of(const torq_kv_cache_t &cache, int heads, int most) {
  return cache.head_dim <= 128 && (int64_t)most * (heads / cache.heads) <= 64 ? 64 : 128;
}
ChunkPlan chunk_plan(const torq_kv_cache_t &cache, int heads, int64_t tokens, int most, int64_t B, int width) {
  ChunkPlan p;
  const int64_t each = heads / cache.heads;
  p.rows = rows_of(cache, heads, most);
  p.slots = std::min(tokens * each / p.rows + std::min(B, tokens), B * ((most * each + p.rows - 1) / p.rows));
  p.items = p.slots * cache.heads;
  const int64_t steps = ((int64_t)width * cache.page_size + CHUNK_STEP - 1) / CHUNK_STEP, full = cache.head_dim <= 128 && p.rows == 128 ? 512 : 256;
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({(full + p.items - 1) / std::max<int64_t>(p.items, 1), steps / 8, 64}));
  return p;
}
}  // namespace

size_t chunk_attention_workspace_bytes(const torq_kv_cache_t &cache, int heads, int64_t tokens, int most, int64_t B, int width) {
  if (few_rows(cache, heads, most)) return paged_attention_workspace_bytes(cache, heads * most, B, width);
  const ChunkPlan p = chunk_plan(cache, heads, tokens, most, B, width);
  return p.splits == 1 ? 0 : (size_t)p.items * p.splits * p.rows * (cache.head_dim + 2) * sizeof(float);
}

hipError_t launch_chunk_attention(const torq_kv_cache_t &cache, const void *q, int64_t q_stride, int64_t q_head_stride, int heads, int64_t tokens,
                                  const int32_t *starts, int most, const int32_t *block_tables, int64_t table_stride, int width,
                                  const int32_t *lengths, int64_t B, float scale, const torq_scores_t *scores, void *out, void *workspace,
                                  hipStream_t stream) {
  if (few_rows(cache, heads, most))
    return launch_paged_attention(cache, q, q_stride, q_head_stride, heads, block_tables, table_stride, width, lengths, B, scale, out, workspace,
                                  scores, starts, most, tokens, stream);
  const int bend = bend_of(scale, scores);
  const ChunkPlan plan = chunk_plan(cache, heads, tokens, most, B, width);
  ChunkArgs a;
  static_cast<AttentionArgs &>(a) = attention_args(cache, q, q_stride, q_head_stride, heads, block_tables, table_stride, width, lengths, B, scale,
                                                   out, scores, starts, most, tokens);
  a.part = (float *)workspace, a.part_ml = a.part + plan.items * plan.splits * plan.rows * cache.head_dim;
  a.c = std::fabs(a.scale_log2), a.flip = a.scale_log2 < 0.0f;
  a.any_cap = 0;
  if (a.rule.cap_out > 0.0f) {
    a.any_cap = short_cap(scores) ? CAP_SHORT : CAP_LONG, a.scale_log2 = a.rule.cap_out;
    if (a.any_cap == CAP_SHORT)
      a.scale_log2 = 2.0f * a.rule.cap_out, a.rule.cap_in = std::max(-FLT_MAX, std::min(FLT_MAX, 2.88539008177792681472f * a.rule.cap_in));
    a.c = a.scale_log2;
  }
  if (bend >= BEND_SLOPES) a.c = 1.0f;
  a.slots = (int)plan.slots, a.splits = plan.splits, a.tile_rows = plan.rows;
  const unsigned groups = (unsigned)(plan.items * plan.splits);
  (cache.head_dim <= 64    ? go_chunk_64
   : cache.head_dim <= 96  ? go_chunk_96
   : cache.head_dim <= 128 ? go_chunk_128
   : cache.head_dim <= 192 ? go_chunk_192
                           : go_chunk_256)(a, cache.format, bend, groups, stream);
  if (plan.splits > 1)
    hipLaunchKernelGGL(chunk_join_kernel, dim3((unsigned)plan.items, 8), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace torq
