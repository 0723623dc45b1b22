// torq_chunk_attention: several new tokens of each request over its pages, out = softmax(scores) V for each (token, head).
//
// 4 head_dim flops for each (row, key) that sees the other: bound by the matrix cores, whose two products take 32 cycles of a SIMD for 32 rows x
// 32 keys x 16 values, and beside them by the vector instructions of the softmax (a fused multiply-add, an exponential, a maximum and halves of a
// conversion and a sum for each score, 3 of the 8 cycles that a score's products take at head_dim 128, and 4 for the exponential).
//
// Work: the (token, head) pairs of a request under one key head are rows, 128 of them a workgroup's, 32 a wave's; its keys come in tiles of 64.  A wave
// brings 16 of a tile's keys (they lie in one page) into registers while the tile before is worked on, widens them to bf16 and puts them into LDS,
// two tiles of it, for all four waves.  Few rows over many keys: the tiles of a row tile are cut into equal parts, one for each workgroup, whose O, m
// and l a second kernel joins in the order of the keys.
//
// A tile goes through the matrix cores transposed, and nothing of it passes between lanes but maxima between two halves of a wave:
//   S^T [key][row] = K [key][i] Q^T [i][row]            v_mfma_f32_32x32x16_bf16
//   lane (n = l % 32, h = l / 32) then holds row n's S for the keys 8 (r / 4) + 4 h + r % 4, r < 16
//   O^T [i][row] += V^T [i][key] P^T [key][row]          the k index runs over the keys in that order, so P^T is already its B operand, and
//                                                        ds_read_b64_tr_b16 reads four keys of one i from rows of V for the A operand
// The weights are rounded to bf16 (8 bits, to nearest), and the sum that the output is divided by is that of the rounded ones: what is left is
// the rounding's own scatter, 2^-9 / sqrt(3) of a weight, beside the output's rounding to bf16 of the same size; two parts as for single tokens would
// take half as many products again.  The maximum that weights are taken against is moved on only when a row's passes it by 2^8: until then they stay
// below 2^8, and O, most of a tile's vector work at the beginning, need not be scaled.
#pragma once

#include "paged_attention_body.h"

namespace torq {

constexpr int CHUNK_ROWS = 128, CHUNK_KEYS = 64, CHUNK_WAVE_ROWS = 32;

struct ChunkArgs : AttentionArgs {
  float c;                             // what scores are times in the exponent of 2
  int flip;                            // q's signs (a scale below 0)
  int slots, splits;                   // row tiles of a key head at most; parts of the keys of one
};

// 16-byte pieces of a row of LDS are permuted by the row, so that what lanes read at a time lies in different banks: K, a piece of 32 rows (DP / 8
// pieces each); V, eight pieces (128 bytes) of four rows
template <int DP>
__device__ __forceinline__ int k_place(int key, int piece) {
  const int by = DP == 64 ? key >> 1 & 7 : key & 15;
  return key * DP * 2 + (piece ^ by) * 16;
}
template <int DP>
__device__ __forceinline__ int v_place(int key, int piece) {
  const int by = DP == 64 ? (key >> 1 & 1) << 2 : (key & 3) << 2;
  return key * DP * 2 + (piece ^ by) * 16;
}

// The request and the tile of its rows that a slot is, the last tiles of a request first; the same in every lane.
__device__ __forceinline__ bool row_tile_of(const ChunkArgs &a, int slot, int &b, int &row_tile) {
  const int lane = threadIdx.x & 63;
  auto tiles_of = [&](int i) {
    if (i >= a.B) return 0;
    const int2 rows = rows_of_request(a, a.rule.starts[i], a.rule.starts[i + 1]);
    return (int)(((int64_t)min(rows.y - rows.x, a.rule.most) * a.rule.heads_each + CHUNK_ROWS - 1) / CHUNK_ROWS);
  };
  int before = 0, found = -1, at_it = 0, there = 0;
  for (int b0 = 0; b0 < a.B && found < 0; b0 += 512) {          // a lane adds up eight requests
    int count[8], mine = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) mine += count[i] = tiles_of(b0 + lane * 8 + i);
    const int sum = before + wave_sum(mine);
    const uint64_t behind = __ballot(slot < sum);
    if (behind) {
      const int owner = __builtin_ctzll(behind);
      int at = __builtin_amdgcn_readlane(sum - mine, owner);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int here = __builtin_amdgcn_readlane(count[i], owner);
        if (found < 0 && slot < at + here) found = b0 + owner * 8 + i, at_it = at, there = here;
        at += here;
      }
    }
    before = __builtin_amdgcn_readlane(sum, 63);
  }
  b = __builtin_amdgcn_readfirstlane(found), row_tile = __builtin_amdgcn_readfirstlane(there - 1 - (slot - at_it));
  return b >= 0;
}

template <int DP, int FMT, bool BENT>
__global__ void __launch_bounds__(256, DP <= 128 ? 2 : 1) chunk_attention_kernel(ChunkArgs a) {
  constexpr bool SCALED = FMT != FMT_BF16;
  constexpr int BITS = FMT == FMT_BF16 ? 16 : FMT == FMT_MXFP8 ? 8 : 4;
  constexpr int W = DP * BITS / 32 < 16 ? DP * BITS / 32 : 16;  // bytes of a lane's load
  constexpr int PER = DP * BITS / 8 / W;                        // lanes of a key
  constexpr int L = 16 * PER / 64;                              // loads of a lane for 16 keys
  constexpr int VALUES = W * 8 / BITS;                          // of a load
  constexpr int SCALE_OF = 4 * BITS, KS = DP / 16, IB = DP / 32;
  constexpr int SIDE = CHUNK_KEYS * DP * 2;                     // bytes of a tile's K
  __shared__ __attribute__((aligned(1024))) char lds[2][2][SIDE];
  // of the keys that a wave has brought: 1 a value of V that is not finite (looked for where not every row sees all keys), 2 they have no page
  __shared__ __attribute__((aligned(16))) int odd[2][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
  const uniform_ints lengths = (uniform_ints)(uintptr_t)a.lengths, starts = (uniform_ints)(uintptr_t)a.rule.starts;
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };

  // the workgroup's key head, part and row tile (all key heads of a part side by side: with 8 of them one for each XCD's L2; the last rows of a request,
  // which have the most keys, first)
  const int kv_head = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, split = rest % a.splits, slot = rest / a.splits;
  int b, row_tile;
  if (!row_tile_of(a, slot, b, row_tile)) return;
  const int2 rows_there = rows_of_request(a, starts[b], starts[b + 1]);
  const int q_at = uniform(rows_there.x), fresh = uniform(min(rows_there.y - rows_there.x, a.rule.most)), each = a.rule.heads_each;
  const int length = uniform(length_of(a, lengths[b])), first = uniform(lengths[b] - (rows_there.y - rows_there.x));
  const int prefix = uniform(a.rule.prefix ? min(max(((uniform_ints)(uintptr_t)a.rule.prefix)[b], 0), length) : 0);
  const int window = a.rule.window, rows = fresh * each, row0 = row_tile * CHUNK_ROWS;
  auto low_of = [&](int p) { return window && p >= window ? p - window + 1 : 0; };
  auto position_of = [&](int row) { return first + min(row, rows - 1) / each; };
  // tiles of keys: those of the prefix, then those from the first to the last that some row sees, `skip` of them left out between
  const int last_key = min(position_of(row0 + CHUNK_ROWS - 1) + 1, length);
  const int prefix_tiles = (prefix + CHUNK_KEYS - 1) / CHUNK_KEYS, all = max((last_key + CHUNK_KEYS - 1) / CHUNK_KEYS, prefix_tiles);
  const int skip = max(min(low_of(position_of(row0)) / CHUNK_KEYS, all) - prefix_tiles, 0), tiles = all - skip;
  const int begin = (int)((int64_t)tiles * split / a.splits), end = (int)((int64_t)tiles * (split + 1) / a.splits);
  auto key_of = [&](int tile) { return (tile < prefix_tiles ? tile : tile + skip) * CHUNK_KEYS; };

  // this wave's rows, this lane's
  const int wave_row = row0 + wave * CHUNK_WAVE_ROWS, row = wave_row + n, token = row / each, head = kv_head * each + row - token * each;
  const bool wave_in = wave_row < rows, in = row < rows;
  const int p_first = uniform(position_of(wave_row)), p_last = uniform(position_of(wave_row + CHUNK_WAVE_ROWS - 1));
  const int position = first + token, low = low_of(position);
  const float slope = BENT && a.rule.slopes && in ? 1.44269504088896340736f * a.rule.slopes[head] : 0.0f;
  bf16x8 q[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int i = 16 * s + 8 * h;
    u32x4 v = {0, 0, 0, 0};
    if (in && i < a.dim) v = *reinterpret_cast<const u32x4 *>(a.q + (int64_t)(q_at + token) * a.q_stride + (int64_t)head * a.q_head_stride + i);
    if (!BENT && a.flip) v ^= 0x80008000u;
    q[s] = as_bf16(v);
  }

  // a tile's 16 keys of this wave: on their way, and into LDS
  const int load_key = lane / PER, load_at = lane % PER;
  const uniform_ints table = (uniform_ints)(uintptr_t)(a.tables + b * a.table_stride);
  auto page_of = [&](int tile) {
    const int t16 = max(min(key_of(tile) / 16 + wave, (length - 1) / 16), 0), entry = (int)((uint64_t)(uint32_t)t16 * (uint64_t)a.page16_magic >> 38);
    return make_int2(length > 0 ? table[entry] : -1, 16 * (t16 - entry * (a.page_size / 16)));
  };
  uint32_t k[L][W / 4], v[L][W / 4];
  uint8_t k_scales[L], v_scales[L];
  bool absent = false;
  auto load = [&](int tile, int2 page) {
    absent = (uint32_t)page.x >= (uint32_t)a.pages;
    const int left = absent ? 0 : length - (key_of(tile) + 16 * wave), count = max(min(left, 16), 0);
    const int64_t at = (left > 0 ? page.x : 0) * a.page_bytes + (kv_head * a.head_bytes + (int64_t)(page.y * a.token_bytes));
    auto side = [&](const char *base, const uint8_t *base_scales, uint32_t (&x)[L][W / 4], uint8_t (&scales)[L]) {
      const __amdgpu_buffer_rsrc_t r = records(base, at, count ? (count - 1) * a.token_bytes + a.dim * BITS / 8 : 0);
      __amdgpu_buffer_rsrc_t rs;
      if constexpr (SCALED) rs = records(base_scales, at / SCALE_OF, count ? (count - 1) * (a.token_bytes / SCALE_OF) + a.dim / 32 : 0);
#pragma unroll
      for (int j = 0; j < L; ++j) {
        const int where = (load_key + 64 / PER * j) * a.token_bytes + load_at * W;
        const bool there = load_at * VALUES < a.dim;
        const auto y = buffer_load<W, false>(r, there ? where : ATT_FAR);
#pragma unroll
        for (int c = 0; c < W / 4; ++c) x[j][c] = y[c];
        if constexpr (SCALED) scales[j] = __builtin_amdgcn_raw_buffer_load_b8(rs, there ? where / SCALE_OF : ATT_FAR, 0, 0);
      }
    };
    side(a.k, a.k_scales, k, k_scales);
    side(a.v, a.v_scales, v, v_scales);
  };
  auto widened = [&](const uint32_t (&x)[L][W / 4], const uint8_t (&scales)[L], int j, int piece) {      // 8 values
    const float scale = SCALED ? __uint_as_float((uint32_t)scales[j] << 23) : 0.0f;
    if constexpr (FMT == FMT_BF16) return u32x4{x[j][0], x[j][1], x[j][2], x[j][3]};
    else if constexpr (FMT == FMT_MXFP4) return widen8(x[j][piece], scale);
    else {
      u32x4 y;
      uint32_t w[4];
      widen4(x[j][2 * piece], scale, w[0], w[1]);
      widen4(x[j][2 * piece + 1], scale, w[2], w[3]);
      y = u32x4{w[0], w[1], w[2], w[3]};
      return y;
    }
  };
  // whether every row of the workgroup sees all keys of a tile, or of this wave
  const int wg_first = uniform(position_of(row0)), wg_last = uniform(position_of(row0 + CHUNK_ROWS - 1));
  auto all_seen = [&](int key0, int from, int to) {
    return key0 + CHUNK_KEYS <= length && (key0 + CHUNK_KEYS <= prefix || (key0 + CHUNK_KEYS - 1 <= from && key0 >= low_of(to)));
  };
  auto put = [&](int buffer, int tile) {
    uint32_t bad = 0;
    const bool edge = !all_seen(key_of(tile), wg_first, wg_last);
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const int key = 16 * wave + load_key + 64 / PER * j;
#pragma unroll
      for (int piece = 0; piece < VALUES / 8; ++piece) {
        *reinterpret_cast<u32x4 *>(&lds[buffer][0][k_place<DP>(key, load_at * (VALUES / 8) + piece)]) = widened(k, k_scales, j, piece);
        const u32x4 x = widened(v, v_scales, j, piece);
        *reinterpret_cast<u32x4 *>(&lds[buffer][1][v_place<DP>(key, load_at * (VALUES / 8) + piece)]) = x;
        if (edge)
#pragma unroll
          for (int c = 0; c < 4; ++c) bad |= not_finite(x[c]);
      }
    }
    const bool any = __any(bad != 0);
    if (lane == 0) odd[buffer][wave] = any + 2 * absent;
  };

  f32x16 o[IB];
#pragma unroll
  for (int i = 0; i < IB; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[i][r] = 0.0f;
  float m = -INFINITY, l = 0.0f;
  const float c = BENT ? 1.0f : a.c;
  const int k_base = k_place<DP>(n, h);
  // where this lane's part of four keys' values lies, those of i = 0 ... 31 of the keys 4 h ... 4 h + 3
  const int v_key = 4 * h + (lane & 15) / 4, v_piece = 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
  int v_base[DP == 64 ? 2 : 4];
#pragma unroll
  for (int i = 0; i < (DP == 64 ? 2 : 4); ++i) v_base[i] = v_place<DP>(v_key, 4 * i + v_piece) + (lane & 1) * 8;
  typedef __attribute__((address_space(3))) i16x4 *lds_i16x4;

  auto work = [&](int buffer, int key0) {
    const i32x4 marks = *reinterpret_cast<const i32x4 *>(odd[buffer]);
    const int mark = uniform(marks[0] | marks[1] | marks[2] | marks[3]);
    const bool seen = mark < 2 && all_seen(key0, p_first, p_last);
    if (!wave_in || (!seen && key0 >= prefix && (key0 > p_last || key0 >= length || key0 + CHUNK_KEYS <= low_of(p_first)))) return;
    const char *const ks = lds[buffer][0], *const vs = lds[buffer][1];
    f32x16 st[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int r = 0; r < 16; ++r) st[u][r] = 0.0f;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(ks + (k_base ^ 32 * s) + u * 32 * DP * 2);
        st[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16(x), q[s], st[u], 0, 0, 0);
      }
    }
    auto key_at = [&](int u, int r) { return key0 + 32 * u + 8 * (r / 4) + 4 * h + r % 4; };
    if constexpr (BENT) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float x = st[u][r] * a.scale_log2;
          if (a.rule.cap_out > 0.0f) x = capped(st[u][r], a.rule.cap_in, a.rule.cap_out);
          if (a.rule.slopes) x -= slope * fabsf((float)(position - key_at(u, r)));
          st[u][r] = x;
        }
    }
    if (!seen) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int t = key_at(u, r);
          if (!(t < length && marks[2 * u + r / 8] < 2 && ((t <= position && t >= low) || t < prefix))) st[u][r] = -INFINITY;
        }
    }
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, st[u][r]);
    const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
    if (__any((top - m) * c > 8.0f)) {
      const float m_new = fmaxf(m, top), base = m_new == -INFINITY ? 0.0f : m_new, alpha = __builtin_amdgcn_exp2f((m - base) * c);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < IB; ++i) o[i] *= alpha;
    }
    const float base = m == -INFINITY ? 0.0f : m * c;
    u32x4 pt[4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const bf16x2 pair = {(__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(st[u][r], c, -base)),
                             (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(st[u][r + 1], c, -base))};
        l = __builtin_amdgcn_fdot2_f32_bf16(pair, bf16x2{(__bf16)1.0f, (__bf16)1.0f}, l, false);
        pt[2 * u + r / 8][r % 8 / 2] = __builtin_bit_cast(uint32_t, pair);
      }
    // four keys of 32 i for each of two: keys 16 s + 4 h + 0 ... 3 and + 8
    auto operand = [&](int s, int i) {
      const int at = v_base[i % (DP == 64 ? 2 : 4)] + i / 4 * 256 + s * 16 * DP * 2;
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(vs + at)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(vs + at + 8 * DP * 2));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    if (!seen && mark & 1) {
      // 0 times what is not finite is no 0: a row at a time, with nothing in the place of the keys that it does not see
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int i = 0; i < IB; ++i) {
          const auto there = operand(s, i);
#pragma nounroll
          for (int x = 0; x < CHUNK_WAVE_ROWS; ++x) {
            const int its_position = __builtin_amdgcn_readlane(position, x), its_low = __builtin_amdgcn_readlane(low, x);
            const u32x4 nothing = {0, 0, 0, 0}, p = n == x ? pt[s] : nothing;
            auto w = there;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int t = key0 + 16 * s + 8 * (e / 4) + 4 * h + e % 4;
              w[e] = t < length && ((t <= its_position && t >= its_low) || t < prefix) ? w[e] : (short)0;
            }
            f32x16 y;
#pragma unroll
            for (int r = 0; r < 16; ++r) y[r] = 0.0f;
            y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), as_bf16(p), y, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][r] += n == x ? y[r] : 0.0f;
          }
          __builtin_amdgcn_sched_barrier(0);
        }
    } else {
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int i = 0; i < IB; ++i)
          o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, operand(s, i)), as_bf16(pt[s]), o[i], 0, 0, 0);
    }
  };

  if (begin < end) {
    int2 page = page_of(begin);
    load(begin, page);
    page = page_of(begin + 1);
    put(0, begin);
    __syncthreads();
    int buffer = 0;
    for (int tile = begin; tile < end; ++tile, buffer ^= 1) {
      const bool more = tile + 1 < end;
      if (more) {
        load(tile + 1, page);
        page = page_of(tile + 2);
      }
      work(buffer, key_of(tile));
      if (more) put(buffer ^ 1, tile + 1);
      __syncthreads();
    }
  }
  if (!wave_in) return;
  const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(halves[0]) + __uint_as_float(halves[1]);
  if (!in) return;
  if (a.splits > 1) {
    const int64_t part = (((int64_t)slot * a.kv_heads + kv_head) * a.splits + split) * CHUNK_ROWS + wave * CHUNK_WAVE_ROWS + n;
    if (h == 0) a.part_ml[2 * part] = BENT || m == -INFINITY ? m : m * c, a.part_ml[2 * part + 1] = l;
#pragma unroll
    for (int i = 0; i < IB; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int at = 32 * i + 2 * r + 4 * h;
        if (at < a.dim) *reinterpret_cast<f32x4 *>(a.part + part * a.dim + at) = f32x4{o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]};
      }
    return;
  }
  const float inverse = l != 0.0f ? 1.0f / l : 0.0f;
  uint16_t *const out = a.out + ruled_row(a, q_at, kv_head, row) * a.dim;
#pragma unroll
  for (int i = 0; i < IB; ++i)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int at = 32 * i + 2 * r + 4 * h;
      if (at < a.dim)
        *reinterpret_cast<bf16x4 *>(out + at) = bf16x4{(__bf16)(o[i][r] * inverse), (__bf16)(o[i][r + 1] * inverse),
                                                       (__bf16)(o[i][r + 2] * inverse), (__bf16)(o[i][r + 3] * inverse)};
    }
}

template <int DP>
void go_chunk(const ChunkArgs &a, int format, bool bent, unsigned groups, hipStream_t stream) {
  auto of_format = [&](auto of) {
    constexpr int FMT = decltype(of)::value;
    if (bent) hipLaunchKernelGGL((chunk_attention_kernel<DP, FMT, true>), dim3(groups), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((chunk_attention_kernel<DP, FMT, false>), dim3(groups), dim3(256), 0, stream, a);
  };
  if (format == FMT_BF16) of_format(std::integral_constant<int, FMT_BF16>{});
  else if (format == FMT_MXFP8) of_format(std::integral_constant<int, FMT_MXFP8>{});
  else of_format(std::integral_constant<int, FMT_MXFP4>{});
}
void go_chunk_256(const ChunkArgs &a, int format, bool bent, unsigned groups, hipStream_t stream);      // chunk_attention_256.hip

}  // namespace torq
