// torq_paged_attention: one new token of each request over its pages, out = softmax(scale q K^T) V for each head.
//
// The query heads of a key head are the columns of one matrix product, up to 16 at a time, so K and V are read once for all of
// them: HBM-bound, 2 (bf16) or 1 1/32 (MXFP8) bytes for 2 heads / kv_heads flops.  Split over the length: a workgroup takes a range of the tokens of one
// (request, key head); its four waves take turns at the range's tiles of 32 tokens, each with a softmax of its own in one pass (running
// maximum m, sum l, unnormalised O), put together in LDS at the end.  A second kernel joins the ranges.
//
// A tile goes through the matrix cores transposed, and nothing of it passes between lanes but the column maxima:
//   S^T [token][head] = K [token][i] Q^T [i][head]           v_mfma_f32_16x16x32_bf16, two groups of 16 tokens
//   lane (n = l % 16, g = l / 16) then holds head n's S for tokens 4g + r of both groups, r < 4
//   O^T [i][head] += V^T [i][token] P^T [token][head]        the k index of this product runs over the 32 tokens in the order in
//                                                            which the lanes hold them, so P^T is already its B operand
// Its A operand wants 8 tokens of one i in a lane.  The lane loads, for its 8 tokens, E consecutive values of V (coalesced
// rows), and pairs of them are put together by v_perm_b32: slot j holds V[its tokens][E * (l % 16) + j].
// In MXFP8 the elements are widened to bf16 with their scale in one instruction (exact: 4 bits of significand).
#include "torq_device.h"
#include "torq_internal.h"

namespace torq {

constexpr int ATT_TILE = 32;          // tokens of a wave's step
constexpr int ATT_WAVES = 4;
constexpr int ATT_ROWS = 16;          // query heads of a workgroup

struct AttentionArgs {
  const char *k, *v;
  const uint8_t *k_scales, *v_scales;
  int64_t pages, page_stride, head_stride, token_stride;
  const uint16_t *q;
  int64_t q_stride, q_head_stride;
  const int *tables, *lengths;
  int64_t table_stride;
  int width, page_size, kv_heads, group, row_groups, dim, splits, chunk;
  float scale_log2;                   // scale * log2(e): the softmax is taken to base 2
  uint16_t *out;
  float *part;                        // [(request, key head, rows of 16)][split][16][dim + 2]: O, then m and l
};

__device__ __forceinline__ bf16x8 as_bf16(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }
// four E4M3 bytes -> two words of two bf16, times scale
__device__ __forceinline__ void widen4(uint32_t v, float scale, uint32_t &a, uint32_t &b) {
  a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, false));
  b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, true));
}

// DP: head_dim rounded up to what the operands hold.
template <int DP, bool F8>
__global__ void __launch_bounds__(256) paged_attention_kernel(AttentionArgs a) {
  constexpr int KS = DP / 32;                       // k-steps of S
  constexpr int E = DP < 128 ? DP / 16 : 8;         // consecutive values of V in a lane
  constexpr int NH = DP / (16 * E);                 // such pieces of a row
  constexpr int BYTES = F8 ? 1 : 2;
  __shared__ float o_all[ATT_WAVES][ATT_ROWS][16 * E + 4];      // a piece of O at a time
  __shared__ float m_all[ATT_WAVES][ATT_ROWS], l_all[ATT_WAVES][ATT_ROWS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int64_t item = blockIdx.x;                  // (request, key head, rows)
  const int split = blockIdx.y;
  const int rows_at = (int)(item % a.row_groups), kv_head = (int)(item / a.row_groups % a.kv_heads);
  const int64_t b = item / a.row_groups / a.kv_heads;
  int64_t len64 = a.lengths[b];
  const int64_t most = (int64_t)a.width * a.page_size;
  len64 = len64 < 0 ? 0 : len64 > most ? most : len64;
  const int len = (int)len64;
  const int begin = split * a.chunk, end = min(len, begin + a.chunk);      // (width * page_size is at most 2^30)
  const int *const table = a.tables + b * a.table_stride;
  const int row = rows_at * ATT_ROWS + n;           // query head of this lane's column within the group
  const bool real = row < a.group;

  // Q^T as the B operand: column n, the i of this lane's K values
  bf16x8 q[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int i = F8 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
    u32x4 v = {0, 0, 0, 0};
    if (real && i < a.dim)
      v = *reinterpret_cast<const u32x4 *>(a.q + b * a.q_stride + (int64_t)(kv_head * a.group + row) * a.q_head_stride + i);
    q[s] = as_bf16(v);
  }
  f32x4 o[NH * E];
#pragma unroll
  for (int i = 0; i < NH * E; ++i) o[i] = f32x4{0, 0, 0, 0};
  float m = -INFINITY, l = 0.0f;

  for (int t0 = begin + wave * ATT_TILE; t0 < end; t0 += ATT_WAVES * ATT_TILE) {
    // the two groups of 16 tokens lie in one page each
    int64_t at[2];
    bool there[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int t = min(t0 + 16 * u, end - 1), entry = t / a.page_size;
      const int page = table[entry];
      there[u] = page >= 0 && page < a.pages;
      at[u] = (there[u] ? (int64_t)page : 0) * a.page_stride + kv_head * a.head_stride +
              (int64_t)((t0 + 16 * u < end ? t0 + 16 * u : t) / 16 * 16 - entry * a.page_size) * a.token_stride;
    }
    f32x4 st[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      // tokens past the end: the last one's address again, their S is masked
      const int first = t0 + 16 * u, token = max(0, min(n, end - 1 - first));
      const int64_t k_at = at[u] + token * a.token_stride;
      st[u] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < KS; s += F8 ? 2 : 1) {
        const int i = F8 ? 32 * s + 16 * g : 32 * s + 8 * g;
        u32x4 v = {0, 0, 0, 0};
        if (i < a.dim) v = *reinterpret_cast<const u32x4 *>(a.k + (k_at + i) * BYTES);
        if constexpr (F8) {
          const float scale = i < a.dim ? e8m0_to_f32(a.k_scales[(k_at + i) >> 5]) : 1.0f;
          u32x4 lo, hi;
          uint32_t w[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) widen4(v[e], scale, w[2 * e], w[2 * e + 1]);
          lo = u32x4{w[0], w[1], w[2], w[3]};
          hi = u32x4{w[4], w[5], w[6], w[7]};
          st[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(lo), q[s], st[u], 0, 0, 0);
          st[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(hi), q[s + 1], st[u], 0, 0, 0);
        } else {
          st[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(v), q[s], st[u], 0, 0, 0);
        }
      }
    }
    float m_new = m, p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int t = t0 + 16 * (e / 4) + 4 * g + e % 4;
      p[e] = t < end && there[e / 4] ? st[e / 4][e % 4] * a.scale_log2 : -INFINITY;
      m_new = fmaxf(m_new, p[e]);
    }
    m_new = fmaxf(m_new, __shfl_xor(m_new, 16));
    m_new = fmaxf(m_new, __shfl_xor(m_new, 32));
    // (nothing but masked tokens so far: everything below is 0)
    const float base = m_new == -INFINITY ? 0.0f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m - base);
    m = m_new;
    l *= alpha;
    // p as two bf16 parts, the first cut off and the second rounded: p to 2^-16, so the output's own rounding is the only one to
    // bf16 that shows.  Both are positive: an infinite v stays infinite (masked tokens have a v of 0 below).
    u32x4 pt, pt_rest;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[e] = __builtin_amdgcn_exp2f(p[e] - base);
      l += p[e];
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t lo = __float_as_uint(p[2 * c]), hi = __float_as_uint(p[2 * c + 1]);
      pt[c] = __builtin_amdgcn_perm(hi, lo, 0x07060302);
      const bf16x2 rest = {(__bf16)fmaxf(p[2 * c] - __uint_as_float(lo & 0xFFFF0000u), 0x1p-126f),
                           (__bf16)fmaxf(p[2 * c + 1] - __uint_as_float(hi & 0xFFFF0000u), 0x1p-126f)};
      pt_rest[c] = __builtin_bit_cast(uint32_t, rest);
    }
#pragma unroll
    for (int i = 0; i < NH * E; ++i) o[i] *= alpha;
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      const int i = h * 16 * E + E * n;
      uint32_t w[8][E / 2];                         // 8 tokens, E values each
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int u = e / 4, first = t0 + 16 * u, token = 4 * g + e % 4;
#pragma unroll
        for (int c = 0; c < E / 2; ++c) w[e][c] = 0;
        if (first + token < end && there[u] && i < a.dim) {      // a weight of 0 would not hide a NaN
          const int64_t v_at = at[u] + token * a.token_stride + i;
          if constexpr (F8) {
            const float scale = e8m0_to_f32(a.v_scales[v_at >> 5]);
            const uint32_t *src = reinterpret_cast<const uint32_t *>(a.v + v_at);
#pragma unroll
            for (int c = 0; c < E / 4; ++c) widen4(src[c], scale, w[e][2 * c], w[e][2 * c + 1]);
          } else {
            const uint32_t *src = reinterpret_cast<const uint32_t *>(a.v + v_at * 2);
#pragma unroll
            for (int c = 0; c < E / 2; ++c) w[e][c] = src[c];
          }
        }
      }
#pragma unroll
      for (int j = 0; j < E; ++j) {
        u32x4 vt;
#pragma unroll
        for (int c = 0; c < 4; ++c)
          vt[c] = __builtin_amdgcn_perm(w[2 * c + 1][j / 2], w[2 * c][j / 2], j % 2 ? 0x07060302 : 0x05040100);
        o[h * E + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(vt), as_bf16(pt), o[h * E + j], 0, 0, 0);
        o[h * E + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(vt), as_bf16(pt_rest), o[h * E + j], 0, 0, 0);
      }
    }
  }
  // the lanes of a column hold the sums of their own tokens
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (g == 0) m_all[wave][n] = m, l_all[wave][n] = l;
  const int rows = min(ATT_ROWS, a.group - rows_at * ATT_ROWS);
#pragma unroll
  for (int h = 0; h < NH; ++h) {
    // lane (n, g), o[h E + j][r] = O[head n][16 E h + E (4 g + r) + j]
#pragma unroll
    for (int j = 0; j < E; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) o_all[wave][n][E * (4 * g + r) + j] = o[h * E + j][r];
    __syncthreads();
    const int first = 16 * E * h, count = min(16 * E, a.dim - first);
    for (int x = threadIdx.x; x < rows * count; x += 256) {
      const int r = x / count, i = x - r * count;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < ATT_WAVES; ++w) top = fmaxf(top, m_all[w][r]);
      const float base = top == -INFINITY ? 0.0f : top;
      float sum = 0.0f, value = 0.0f;
#pragma unroll
      for (int w = 0; w < ATT_WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f(m_all[w][r] - base);
        sum += f * l_all[w][r];
        value += f * o_all[w][r][i];
      }
      if (a.splits == 1) {
        const int head = kv_head * a.group + rows_at * ATT_ROWS + r;
        const __bf16 y = (__bf16)(sum != 0.0f ? value / sum : 0.0f);
        a.out[(b * a.kv_heads * a.group + head) * a.dim + first + i] = __builtin_bit_cast(uint16_t, y);
      } else {
        float *to = a.part + ((item * a.splits + split) * ATT_ROWS + r) * (a.dim + 2);
        to[first + i] = value;
        if (first + i == 0) to[a.dim] = top, to[a.dim + 1] = sum;
      }
    }
    __syncthreads();
  }
}

__global__ void __launch_bounds__(256) paged_attention_join_kernel(AttentionArgs a) {
  const int64_t item = blockIdx.x;
  const int rows_at = (int)(item % a.row_groups);
  const int64_t b_head = item / a.row_groups;       // (request, key head)
  const int rows = min(ATT_ROWS, a.group - rows_at * ATT_ROWS);
  for (int x = threadIdx.x; x < rows * a.dim; x += 256) {
    const int r = x / a.dim, i = x % a.dim;
    const float *from = a.part + (item * a.splits * ATT_ROWS + r) * (a.dim + 2);
    const int64_t step = (int64_t)ATT_ROWS * (a.dim + 2);
    float top = -INFINITY, sum = 0.0f, value = 0.0f;
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, from[s * step + a.dim]);
    const float base = top == -INFINITY ? 0.0f : top;
    for (int s = 0; s < a.splits; ++s) {
      const float f = __builtin_amdgcn_exp2f(from[s * step + a.dim] - base);
      sum += f * from[s * step + a.dim + 1];
      value += f * from[s * step + i];
    }
    const __bf16 y = (__bf16)(sum != 0.0f ? value / sum : 0.0f);
    a.out[(b_head * a.group + rows_at * ATT_ROWS + r) * a.dim + i] = __builtin_bit_cast(uint16_t, y);
  }
}

namespace {
// Ranges of the length: enough workgroups for two on each of the 256 CUs, none under 256 tokens
int attention_splits(int64_t items, int64_t most) {
  int64_t s = (512 + items - 1) / items;
  const int64_t cap = (most + 255) / 256;
  s = s < cap ? s : cap;
  return (int)(s < 1 ? 1 : s);
}
}  // namespace

size_t paged_attention_workspace_bytes(const torq_kv_cache_t &cache, int heads, int64_t B, int width) {
  const int group = heads / cache.heads;
  const int64_t items = B * cache.heads * ((group + ATT_ROWS - 1) / ATT_ROWS);
  const int splits = attention_splits(items, (int64_t)width * cache.page_size);
  return splits > 1 ? (size_t)items * splits * ATT_ROWS * (cache.head_dim + 2) * sizeof(float) : 0;
}

hipError_t launch_paged_attention(const torq_kv_cache_t &cache, const void *q, int64_t q_stride, int64_t q_head_stride, int heads,
                                  const int32_t *block_tables, int64_t table_stride, int width, const int32_t *lengths,
                                  int64_t B, float scale, void *out, void *workspace, hipStream_t stream) {
  const int group = heads / cache.heads, row_groups = (group + ATT_ROWS - 1) / ATT_ROWS;
  if (cache.pages == 0) width = 0;                  // no token has a page: nothing of the cache is touched
  const int64_t items = B * cache.heads * row_groups, most = (int64_t)width * cache.page_size;
  const int splits = attention_splits(items, most);
  int64_t chunk = (most + splits - 1) / splits;
  chunk = (chunk + ATT_TILE - 1) / ATT_TILE * ATT_TILE;
  AttentionArgs a{(const char *)cache.k, (const char *)cache.v, cache.k_scales, cache.v_scales, cache.pages, cache.page_stride,
                  cache.head_stride, cache.token_stride, (const uint16_t *)q, q_stride, q_head_stride, block_tables, lengths,
                  table_stride, width, cache.page_size, cache.heads, group, row_groups, cache.head_dim, splits, (int)chunk,
                  scale * 1.44269504088896340736f, (uint16_t *)out, (float *)workspace};
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)items, splits), dim3(256), 0, stream, a);
  };
  const bool f8 = cache.format == FMT_MXFP8;
  if (cache.head_dim <= 64) go(f8 ? paged_attention_kernel<64, true> : paged_attention_kernel<64, false>);
  else if (cache.head_dim <= 128) go(f8 ? paged_attention_kernel<128, true> : paged_attention_kernel<128, false>);
  else go(f8 ? paged_attention_kernel<256, true> : paged_attention_kernel<256, false>);
  if (splits > 1) hipLaunchKernelGGL(paged_attention_join_kernel, dim3((unsigned)items), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace torq
