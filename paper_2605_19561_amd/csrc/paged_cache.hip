// torq_block_tables and torq_cache_append: what a step does to a paged key-value cache ahead of its attention.
#include "torq_device.h"
#include "torq_internal.h"

namespace torq {

// ---- pages and slots ---------------------------------------------------------------------------
// Two running sums over the requests, pages wanted and new tokens, and what they say written out.  A few KB in, 8 bytes a token
// out: bound by the launch and by what hangs on one another, lengths -> sums -> page -> slot.
//
// Every workgroup makes the sums of all requests itself (no second launch, nothing handed over), 1024 requests at a time.  The few entries
// of a request that goes on by a token or some (a decode step) its own lane writes; where one of the 1024 has more, all entries of those are
// looked for in the sums in LDS, by lanes that take four consecutive tokens or one page each, over all workgroups.
constexpr int TAB_CHUNK = 1024;
constexpr int TAB_FEW = 2;            // entries of a request that its lane writes

// T: what holds the sums of a chunk.
template <class T>
__global__ void __launch_bounds__(256) block_tables_kernel(const int *__restrict__ held, const int *__restrict__ lengths, int64_t B,
                                                           const int *__restrict__ free_pages, int64_t free_count,
                                                           const int *cursor, int *cursor_out, int *block_tables,
                                                           int64_t table_stride, int width, int page_size, int64_t *slots,
                                                           int64_t tokens, bool cursor_only) {
  __shared__ T page_end[TAB_CHUNK], token_end[TAB_CHUNK];             // inclusive sums over the chunk, from 0
  __shared__ int held_at[TAB_CHUNK], had_at[TAB_CHUNK];
  __shared__ T wave_pages[4], wave_tokens[4];
  __shared__ int wave_many[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t first = *cursor;
  const int64_t gid = (int64_t)blockIdx.x * 256 + tid, stride = (int64_t)gridDim.x * 256;
  auto from_list = [&](int64_t i) { return i >= 0 && i < free_count ? free_pages[i] : -1; };
  int64_t pages_before = 0, tokens_before = 0;
  for (int64_t b0 = 0; b0 < B; b0 += TAB_CHUNK) {
    // a lane's requests: as many as spread them over all lanes
    const int per = B - b0 >= TAB_CHUNK ? 4 : (int)((B - b0 + 255) / 256);
    int had[4], page_count[4], at[4];
    T token_count[4], psum = 0, tsum = 0;
    bool many = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      at[i] = per * tid + i;
      const bool there = i < per && b0 + at[i] < B;
      const int h = there ? max(held[b0 + at[i]], 0) : 0, n = there ? max(lengths[b0 + at[i]], 0) : 0;
      // ceil as (n - 1) / P + 1 for n > 0: no sum that passes 32 bits
      had[i] = min(h ? (h - 1) / page_size + 1 : 0, width);
      page_count[i] = max(min(n ? (n - 1) / page_size + 1 : 0, width) - had[i], 0);
      // (past the last slot it does not matter how far, and the sums of 1024 stay in 32 bits)
      const int64_t fresh = max(n - h, 0);
      token_count[i] = (T)(sizeof(T) == 4 && fresh > tokens ? tokens + 1 : fresh);
      many |= page_count[i] > TAB_FEW || token_count[i] > TAB_FEW;
      psum += page_count[i];
      tsum += token_count[i];
    }
    T p = wave_sum(psum), t = wave_sum(tsum);
    if (lane == 63) wave_pages[wave] = p, wave_tokens[wave] = t;
    const bool many_here = __any(many);
    if (lane == 0) wave_many[wave] = many_here;
    __syncthreads();
    T pall = 0, tall = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w < wave) p += wave_pages[w], t += wave_tokens[w];
      pall += wave_pages[w], tall += wave_tokens[w];
    }
    p -= psum, t -= tsum;                                             // ahead of this lane's
    const bool search = wave_many[0] | wave_many[1] | wave_many[2] | wave_many[3];
    if (!search && !cursor_only && (b0 / TAB_CHUNK) % gridDim.x == blockIdx.x) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        int *const row = block_tables + (b0 + at[i]) * table_stride;
        if (i < per && b0 + at[i] < B) {
          const int64_t list = first + pages_before + p;
          for (int j = 0; j < page_count[i]; ++j) row[had[i] + j] = from_list(list + j);
          int position = token_count[i] ? max(held[b0 + at[i]], 0) : 0;
          for (int j = 0; j < (int)token_count[i] && tokens_before + t + j < tokens; ++j, ++position) {
            const int entry = position / page_size;
            const int page = entry < had[i] ? row[entry] : entry < width ? from_list(list + entry - had[i]) : -1;
            slots[tokens_before + t + j] = page < 0 ? -1 : (int64_t)page * page_size + (position - entry * page_size);
          }
        }
        p += page_count[i];
        t += token_count[i];
      }
    }
    if (search && !cursor_only) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < per) {
          p += page_count[i], t += token_count[i];
          page_end[at[i]] = p, token_end[at[i]] = t;
          held_at[at[i]] = b0 + at[i] < B ? max(held[b0 + at[i]], 0) : 0, had_at[at[i]] = had[i];
        }
      __syncthreads();
      const int count = per * 256;
      // the first request whose running sum passes v
      auto owner = [&](const T *ends, int64_t v) {
        int lo = 0;
        for (int step = TAB_CHUNK / 2; step; step >>= 1)
          if (lo + step <= count && ends[lo + step - 1] <= v) lo += step;
        return lo;
      };
      for (int64_t v = gid; v < pall; v += stride) {
        const int r = owner(page_end, v);
        const int64_t j = v - (r ? page_end[r - 1] : 0);
        block_tables[(b0 + r) * table_stride + had_at[r] + j] = from_list(first + pages_before + v);
      }
      const int64_t here = min((int64_t)tall, tokens - tokens_before);
      for (int64_t v = 4 * gid; v < here; v += 4 * stride) {
        int r = owner(token_end, v), place[4];
        int64_t begin = r ? token_end[r - 1] : 0, end = token_end[r], list = r ? page_end[r - 1] : 0;
        const int *from[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          from[i] = nullptr;
          if (v + i >= here) continue;
          while (v + i >= end) begin = end, list = page_end[r], end = token_end[++r];      // (v + i < tall: some request has it)
          const int position = held_at[r] + (int)(v + i - begin), entry = position / page_size;
          const int64_t at = first + pages_before + list + entry - had_at[r];
          place[i] = position - entry * page_size;
          if (entry < had_at[r]) from[i] = block_tables + (b0 + r) * table_stride + entry;
          else if (entry < width && at >= 0 && at < free_count) from[i] = free_pages + at;
        }
        int page[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) page[i] = from[i] ? *from[i] : -1;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (v + i < here) slots[tokens_before + v + i] = page[i] < 0 ? -1 : (int64_t)page[i] * page_size + place[i];
      }
    }
    pages_before += pall;
    tokens_before += tall;
    __syncthreads();
  }
  if (!cursor_only)
    for (int64_t v = tokens_before + gid; v < tokens; v += stride) slots[v] = -1;
  if (cursor_out && gid == 0) *cursor_out = (int)min(first + pages_before, (int64_t)0x7FFFFFFF);
}

hipError_t launch_block_tables(const int32_t *held, const int32_t *lengths, int64_t B, const int32_t *free_pages,
                               int64_t free_count, const int32_t *cursor, int32_t *cursor_out, int32_t *block_tables,
                               int64_t table_stride, int width, int page_size, int64_t *slots, int64_t tokens,
                               hipStream_t stream) {
  int64_t groups = (tokens + 1023) / 1024;
  groups = groups < 1 ? 1 : groups > 256 ? 256 : groups;
  // workgroups of one launch may still be reading the cursor when another is done: in place it takes a launch of its own
  const bool later = cursor_out == cursor && groups > 1;
  // 1024 requests' sums in 32 bits: up to 2^20 pages and (counted no further) slots each
  auto kernel = tokens < (1 << 20) && width <= (1 << 20) ? block_tables_kernel<int> : block_tables_kernel<int64_t>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, stream, held, lengths, B, free_pages, free_count,
                     cursor, later ? nullptr : cursor_out, block_tables, table_stride, width, page_size, slots, tokens, false);
  if (later)
    hipLaunchKernelGGL(kernel, dim3(1), dim3(256), 0, stream, held, lengths, B, free_pages, free_count, cursor,
                       cursor_out, block_tables, table_stride, width, page_size, slots, tokens, true);
  return hipGetLastError();
}

// ---- new keys and values -----------------------------------------------------------------------
// A copy with a place to look up, and to MXFP8 a rounding: HBM-bound, 4 bytes a value to bf16, 3 1/32 to MXFP8.  A lane moves 16
// consecutive values of a token's head (8 to bf16), so it stores 16 bytes and two lanes have a block of MXFP8; the values and slots of
// APPEND_PASSES tokens are on their way together.  (A block's elements and scale are three stores in no order with other workgroups', so a
// slot named twice is left to no one's values.)  Measured: [8192 tokens, 8, 128] to MXFP8 10.8 us (4.7 TB/s), to bf16 11.7 (5.7).
struct AppendArgs {
  torq_kv_cache_t cache;
  const uint16_t *key, *value;
  int64_t key_token, key_head, value_token, value_head;      // strides in elements
  const int64_t *slots;
  int64_t tokens;
  int per_head, per_side, abreast;                           // pieces of a head, of a token's keys; tokens that a workgroup takes at a time
};

constexpr int APPEND_PASSES = 2;      // [8192 tokens, 8, 128] to MXFP8 with 1, 2, 4, 8: 11.2, 10.8, 10.9, 12.8 us; 256 tokens to bf16 2.7, 3.0, 3.4, 4.3

template <int FMT>
__global__ void __launch_bounds__(256) cache_append_kernel(AppendArgs a) {
  constexpr int N = FMT == FMT_BF16 ? 8 : 16;                // values of a lane
  const int64_t places = a.cache.pages * a.cache.page_size;
  const int per_token = 2 * a.per_side;
  // lane -> token of the workgroup's and piece; the pieces of a token beyond 256 by rounds
  const int token_at = a.abreast > 1 ? threadIdx.x / per_token : 0;
  if (token_at >= a.abreast) return;
  for (int piece = threadIdx.x - token_at * per_token; piece < per_token; piece += 256) {
    const bool is_value = piece >= a.per_side;
    const int p = is_value ? piece - a.per_side : piece, head = p / a.per_head, at = N * (p - head * a.per_head);
    const uint16_t *const src = is_value ? a.value + head * a.value_head + at : a.key + head * a.key_head + at;
    const int64_t src_token = is_value ? a.value_token : a.key_token;
    const int64_t dst = head * a.cache.head_stride + at;
    void *const to = is_value ? a.cache.v : a.cache.k;
    for (int64_t t0 = (int64_t)blockIdx.x * a.abreast * APPEND_PASSES + token_at; t0 < a.tokens;
         t0 += (int64_t)gridDim.x * a.abreast * APPEND_PASSES) {
      u32x4 v[APPEND_PASSES][N / 8];
      int64_t slot[APPEND_PASSES];
#pragma unroll
      for (int i = 0; i < APPEND_PASSES; ++i) {
        const int64_t t = t0 + i * a.abreast;
        slot[i] = -1;
        if (t < a.tokens) {
          slot[i] = a.slots[t];
#pragma unroll
          for (int c = 0; c < N / 8; ++c) v[i][c] = *reinterpret_cast<const u32x4 *>(src + t * src_token + 8 * c);
        }
      }
#pragma unroll
      for (int i = 0; i < APPEND_PASSES; ++i) {
        if (slot[i] < 0 || slot[i] >= places) continue;      // (the two lanes of a block together)
        // (a division of 64 bits is 40 times one of 32)
        const int64_t page = slot[i] >> 32 ? slot[i] / a.cache.page_size : (int64_t)((uint32_t)slot[i] / (uint32_t)a.cache.page_size);
        const int64_t where = page * a.cache.page_stride + (slot[i] - page * a.cache.page_size) * a.cache.token_stride + dst;
        if constexpr (FMT == FMT_BF16) {
          *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(to) + where) = v[i][0];
        } else {
          float f[2][8];
          uint32_t amax = 0;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              f[c][2 * e] = bf16_bits_to_f32(v[i][c][e] & 0xFFFFu);
              f[c][2 * e + 1] = __uint_as_float(v[i][c][e] & 0xFFFF0000u);
            }
            amax = max(amax, __float_as_uint(amax8_nan(f[c])));
          }
          amax = max(amax, (uint32_t)__builtin_amdgcn_mov_dpp((int)amax, 0xB1, 0xF, 0xF, true));
          const uint32_t byte = mxfp8_scale_from_amax(__uint_as_float(amax));
          const uint2 lo = pack8_e4m3(f[0], byte), hi = pack8_e4m3(f[1], byte);
          *reinterpret_cast<u32x4 *>(static_cast<uint8_t *>(to) + where) = u32x4{lo.x, lo.y, hi.x, hi.y};
          if ((piece & 1) == 0) (is_value ? a.cache.v_scales : a.cache.k_scales)[where >> 5] = (uint8_t)byte;
        }
      }
    }
  }
}

hipError_t launch_cache_append(const torq_kv_cache_t &cache, const void *key, int64_t key_token_stride, int64_t key_head_stride,
                               const void *value, int64_t value_token_stride, int64_t value_head_stride,
                               const int64_t *slots, int64_t tokens, hipStream_t stream) {
  const int per_head = cache.head_dim / (cache.format == FMT_BF16 ? 8 : 16), per_side = cache.heads * per_head;
  const int abreast = 2 * per_side >= 256 ? 1 : 256 / (2 * per_side);
  AppendArgs a{cache, (const uint16_t *)key, (const uint16_t *)value, key_token_stride, key_head_stride, value_token_stride,
               value_head_stride, slots, tokens, per_head, per_side, abreast};
  const int64_t at_a_time = (int64_t)abreast * APPEND_PASSES;
  int64_t groups = (tokens + at_a_time - 1) / at_a_time;
  if (groups > 256 * 64) groups = 256 * 64;
  auto kernel = cache.format == FMT_BF16 ? cache_append_kernel<FMT_BF16> : cache_append_kernel<FMT_MXFP8>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace torq
