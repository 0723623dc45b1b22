// torq_block_tables and torq_cache_append: what a step does to a paged key-value cache ahead of its attention.
#include "torq_device.h"
#include "torq_internal.h"

namespace torq {

// ---- pages and slots ---------------------------------------------------------------------------
// Two running sums over the requests, pages wanted and new tokens, and a search in them for every entry that is written.  A few KB
// in, 8 bytes a token out: bound by the launch and by what hangs on one another, lengths -> sums -> search -> page -> slot.
//
// Every workgroup makes the sums of all requests itself (no second launch, nothing handed over), 1024 requests at a time in
// LDS, and writes its own part of the entries.
constexpr int TAB_CHUNK = 1024;

__global__ void __launch_bounds__(256) block_tables_kernel(const int *__restrict__ held, const int *__restrict__ lengths, int64_t B,
                                                           const int *__restrict__ free_pages, int64_t free_count,
                                                           const int *cursor, int *cursor_out, int *block_tables,
                                                           int64_t table_stride, int width, int page_size, int64_t *slots,
                                                           int64_t tokens, bool cursor_only) {
  __shared__ int64_t page_end[TAB_CHUNK], token_end[TAB_CHUNK];       // inclusive sums over the chunk, from 0
  __shared__ int held_at[TAB_CHUNK], had_at[TAB_CHUNK];
  __shared__ int64_t wave_pages[4], wave_tokens[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t first = *cursor;
  const int64_t gid = (int64_t)blockIdx.x * 256 + tid, stride = (int64_t)gridDim.x * 256;
  int64_t pages_before = 0, tokens_before = 0;
  for (int64_t b0 = 0; b0 < B; b0 += TAB_CHUNK) {
    int64_t pages[4], news[4], psum = 0, tsum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t b = b0 + 4 * tid + i;
      int h = 0, n = 0;
      if (b < B) h = max(held[b], 0), n = max(lengths[b], 0);
      // ceil as (n - 1) / P + 1 for n > 0: no sum that passes 32 bits
      const int had = min(h ? (h - 1) / page_size + 1 : 0, width), have = min(n ? (n - 1) / page_size + 1 : 0, width);
      held_at[4 * tid + i] = h;
      had_at[4 * tid + i] = had;
      pages[i] = psum += max(have - had, 0);
      news[i] = tsum += max(n - h, 0);
    }
    int64_t p = psum, t = tsum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t pu = __shfl_up(p, o), tu = __shfl_up(t, o);
      if (lane >= o) p += pu, t += tu;
    }
    if (lane == 63) wave_pages[wave] = p, wave_tokens[wave] = t;
    __syncthreads();
    int64_t pall = 0, tall = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w < wave) p += wave_pages[w], t += wave_tokens[w];
      pall += wave_pages[w], tall += wave_tokens[w];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      page_end[4 * tid + i] = p - psum + pages[i];
      token_end[4 * tid + i] = t - tsum + news[i];
    }
    __syncthreads();
    if (!cursor_only) {
      // the first request whose running sum passes v
      auto owner = [&](const int64_t *ends, int64_t v) {
        int lo = 0;
#pragma unroll
        for (int step = TAB_CHUNK / 2; step; step >>= 1)
          if (ends[lo + step - 1] <= v) lo += step;
        return lo;
      };
      auto from_list = [&](int64_t i) { return i >= 0 && i < free_count ? free_pages[i] : -1; };
      for (int64_t v = gid; v < pall; v += stride) {
        const int r = owner(page_end, v);
        const int64_t j = v - (r ? page_end[r - 1] : 0);
        block_tables[(b0 + r) * table_stride + had_at[r] + j] = from_list(first + pages_before + v);
      }
      for (int64_t v = gid; v < tall && tokens_before + v < tokens; v += stride) {
        const int r = owner(token_end, v);
        const int position = held_at[r] + (int)(v - (r ? token_end[r - 1] : 0));
        const int entry = position / page_size;
        int page = -1;
        if (entry < had_at[r]) page = block_tables[(b0 + r) * table_stride + entry];
        else if (entry < width) page = from_list(first + pages_before + (r ? page_end[r - 1] : 0) + entry - had_at[r]);
        slots[tokens_before + v] = page < 0 ? -1 : (int64_t)page * page_size + position % page_size;
      }
    }
    pages_before += pall;
    tokens_before += tall;
    __syncthreads();
  }
  if (!cursor_only)
    for (int64_t v = tokens_before + gid; v < tokens; v += stride) slots[v] = -1;
  if (cursor_out && gid == 0) *cursor_out = (int)(first + pages_before);
}

hipError_t launch_block_tables(const int32_t *held, const int32_t *lengths, int64_t B, const int32_t *free_pages,
                               int64_t free_count, const int32_t *cursor, int32_t *cursor_out, int32_t *block_tables,
                               int64_t table_stride, int width, int page_size, int64_t *slots, int64_t tokens,
                               hipStream_t stream) {
  int64_t groups = (tokens + 1023) / 1024;
  groups = groups < 1 ? 1 : groups > 256 ? 256 : groups;
  // workgroups of one launch may still be reading the cursor when another is done: in place it takes a launch of its own
  const bool later = cursor_out == cursor && groups > 1;
  hipLaunchKernelGGL(block_tables_kernel, dim3((unsigned)groups), dim3(256), 0, stream, held, lengths, B, free_pages, free_count,
                     cursor, later ? nullptr : cursor_out, block_tables, table_stride, width, page_size, slots, tokens, false);
  if (later)
    hipLaunchKernelGGL(block_tables_kernel, dim3(1), dim3(256), 0, stream, held, lengths, B, free_pages, free_count, cursor,
                       cursor_out, block_tables, table_stride, width, page_size, slots, tokens, true);
  return hipGetLastError();
}

// ---- new keys and values -----------------------------------------------------------------------
// A copy with a place to look up, and to MXFP8 a rounding: HBM-bound, 4 bytes a value to bf16, 3 1/32 to MXFP8.  A lane moves 8
// consecutive values of a token's head, four lanes a block of MXFP8.
struct AppendArgs {
  torq_kv_cache_t cache;
  const uint16_t *key, *value;
  int64_t key_token, key_head, value_token, value_head;      // strides in elements
  const int64_t *slots;
  int64_t tokens, total;                                     // total: 8-element pieces of keys and values
  int per_head, per_token;                                   // pieces of a head, and of a token's keys and values
};

template <int FMT>
__global__ void __launch_bounds__(256) cache_append_kernel(AppendArgs a) {
  const int64_t slots = a.cache.pages * a.cache.page_size, stride = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.total; i += stride) {
    const int64_t token = i / a.per_token;
    int piece = (int)(i - token * a.per_token);
    const int64_t slot = a.slots[token];
    if (slot < 0 || slot >= slots) continue;                 // (all four lanes of a block together)
    const bool is_value = piece >= a.per_token / 2;
    if (is_value) piece -= a.per_token / 2;
    const int head = piece / a.per_head, at = 8 * (piece - head * a.per_head);
    const uint16_t *src = is_value ? a.value + token * a.value_token + head * a.value_head
                                   : a.key + token * a.key_token + head * a.key_head;
    const u32x4 v = *reinterpret_cast<const u32x4 *>(src + at);
    const int64_t page = slot / a.cache.page_size;
    const int64_t dst = page * a.cache.page_stride + head * a.cache.head_stride +
                        (slot - page * a.cache.page_size) * a.cache.token_stride + at;
    void *const to = is_value ? a.cache.v : a.cache.k;
    if constexpr (FMT == FMT_BF16) {
      *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(to) + dst) = v;
    } else {
      float f[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[2 * e] = bf16_bits_to_f32(v[e] & 0xFFFFu);
        f[2 * e + 1] = __uint_as_float(v[e] & 0xFFFF0000u);
      }
      const uint32_t byte = mxfp8_scale_from_amax(quad_amax_nan(amax8_nan(f)));
      *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(to) + dst) = pack8_e4m3(f, byte);
      if ((threadIdx.x & 3) == 0) (is_value ? a.cache.v_scales : a.cache.k_scales)[dst >> 5] = (uint8_t)byte;
    }
  }
}

hipError_t launch_cache_append(const torq_kv_cache_t &cache, const void *key, int64_t key_token_stride, int64_t key_head_stride,
                               const void *value, int64_t value_token_stride, int64_t value_head_stride,
                               const int64_t *slots, int64_t tokens, hipStream_t stream) {
  AppendArgs a{cache, (const uint16_t *)key, (const uint16_t *)value, key_token_stride, key_head_stride, value_token_stride,
               value_head_stride, slots, tokens, 0, cache.head_dim / 8, 2 * cache.heads * (cache.head_dim / 8)};
  a.total = tokens * a.per_token;
  int64_t groups = (a.total + 255) / 256;
  if (groups > 256 * 16) groups = 256 * 16;
  auto kernel = cache.format == FMT_BF16 ? cache_append_kernel<FMT_BF16> : cache_append_kernel<FMT_MXFP8>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace torq
