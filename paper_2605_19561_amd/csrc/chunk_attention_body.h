// torq_chunk_attention: several new tokens of each request over its pages, out = softmax(scores) V for each (token, head).
//
// 4 head_dim flops for each (row, key) that sees the other: bound by the matrix cores, whose two products take 32 cycles of a SIMD for 32 rows x
// 32 keys x 16 values, and beside them by the vector instructions of the softmax (a fused multiply-add, an exponential, a maximum and halves of a
// conversion and a sum for each score, 3 of the 8 cycles that a score's products take at head_dim 128, and 4 for the exponential).
//
// Work: the (token, head) pairs of a request under one key head are rows, 128 or 64 of them a workgroup's, 32 a wave's; its keys come in steps of 32. 128 rows:
// four waves with the same keys, two workgroups on a CU where the registers allow it (up to 128 values). 64 rows: two waves for each half of the keys, put
// together in LDS at the end: few rows and many keys.
//
// A step's keys lie in a ring of four slots in LDS: bf16 comes straight from memory, three (K) and two (V) steps ahead; MXFP8 and MXFP4 through registers,
// loaded two steps before they are widened to bf16 into it.  Few workgroups over many keys: the steps of a row tile are cut into equal parts, one for each
// workgroup, whose O, m and l a second kernel joins in the order of the keys.
//
// A wave has three steps in hand at a time: the scores of step j + 1, the weights of j, the products with V of j - 1, none of which waits for another. With
// two waves on a SIMD the softmax comes first and then the products, and one wave's instructions fill the other's gaps; so it does in the one wave of
// head_dim over 128, which has no registers for more; a wave of 64 rows, alone on its SIMD too, has its softmax between its products piece by piece (IN_TURN, below).  Steps in which every row sees every key know no masks; the others, at the ends of windows,
// prefixes and lengths, do.  There 0 times a value that is not finite would be no 0: such values are left out, and at the end a second pass puts
// them back for the rows that see them, a case that costs a second look at the keys and is rare.
//
// Measured: one prompt of 8192 tokens, 32 / 8 heads of 128, bf16, 600 to 618 us from one card to another = 890 to 916 TFLOP/s (a large bf16 product reaches
// 1363); 512 tokens behind 60000 in MXFP4, 64 / 8 heads, 1067 to 1095 us = 922 to 946; 4 prompts of 4096 in MXFP8 687 to 709 us; 8 of 1024 by head_dim and format: see
// IN_TURN.  What bounds it is the issue of products and softmax together: LDS reads alone take 268 us of the
// 600, the products at their best 403.  The first version, tiles of 64 keys and no steps in hand: 799 and 1303.  Not taken: 64 rows a wave, whose
// O then fills the accumulators' half of the registers by name (less LDS traffic, one wave a SIMD): 624, 1076, 772.
// Short items (61 capped prompts of up to 1024 tokens, a window of 512, in MXFP8: 7960 of 10.0 steps on average, 433 us; without the cap 382; without the window, 11.3
// steps, 460): half of the time or more is what an item costs besides its steps, that is starts and lengths, table, first keys and first scores, each
// waiting for the one before, and the output's way through LDS.
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

constexpr int CHUNK_STEP = 32;         // keys of a step
constexpr int BEND_NONE = 0, BEND_CAP = 1, BEND_SLOPES = 2, BEND_ANY = 3;
constexpr int CAP_SHORT = 1, CAP_LONG = 2;

struct ChunkArgs : AttentionArgs {
  float c;                             // what (bent) scores are times in the exponent of 2
  int any_cap;                         // (BEND_ANY) which form of the tangent is taken ahead of scale_log2: -1 / (1 + exp2(cap_in s)), or that of every cap
  int flip;                            // q's signs (a scale below 0)
  int tile_rows;                       // rows of a workgroup
  int slots, splits;                   // row tiles of a key head at most; parts of the keys of one
};

// Where 16-byte pieces of keys lie in LDS, so that what lanes read at a time lies in different banks.  K, a piece of 16 rows: groups of 1024 bytes (what a
// wave's load brings) with room between them, the pieces within a group permuted by the row.  V, eight pieces (128 bytes) of four rows: permuted by the row.
template <int DP>
struct KLayout {
  static constexpr int GROUP_ROWS = 512 / DP, PERMUTED = DP == 256 ? 2 : 4, GROUP = 1024 + 16 * PERMUTED, BYTES = CHUNK_STEP / GROUP_ROWS * GROUP;
  static __device__ __forceinline__ int by(int key) { return DP == 64 ? key >> 1 & 3 : key & (PERMUTED - 1); }
  static __device__ __forceinline__ int at(int key, int piece) {
    return key / GROUP_ROWS * GROUP + key % GROUP_ROWS * DP * 2 + (piece ^ by(key)) * 16;
  }
};
template <int DP>
__device__ __forceinline__ int v_place(int key, int piece) {
  const int by = DP == 64 ? (key >> 1 & 1) << 2 : (key & 3) << 2;
  return key * DP * 2 + (piece ^ by) * 16;
}

// The request and the tile of its rows that a slot is, the last tiles of a request first, and what the kernel goes by of it: looked up by lanes, eight
// requests each, all in one go.  The same in every lane.
struct RowTile {
  int b, tile, q_at, rows_there, length, prefix;
};
__device__ __forceinline__ bool row_tile_of(const ChunkArgs &a, int slot, RowTile &found) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int b0 = 0; b0 < a.B; b0 += 512) {
    int start[8], there[8], length[8], prefix[8], mine = 0;
    const int per = min((a.B - b0 + 63) / 64, 8);
    auto tiles_of = [&](int rows) { return (int)(((int64_t)min(rows, a.rule.most) * a.rule.heads_each + a.tile_rows - 1) / a.tile_rows); };
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int b = b0 + lane * per + i;
      start[i] = there[i] = length[i] = prefix[i] = 0;
      if (i < per && b < a.B) {
        const int2 rows = rows_of_request(a, a.rule.starts[b], a.rule.starts[b + 1]);
        start[i] = rows.x, there[i] = rows.y - rows.x, length[i] = a.lengths[b];
        if (a.rule.prefix) prefix[i] = a.rule.prefix[b];
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) mine += tiles_of(there[i]);
    const int sum = before + wave_sum(mine);
    const uint64_t behind = __ballot(slot < sum);
    if (behind) {
      const int owner = __builtin_ctzll(behind);
      int at = __builtin_amdgcn_readlane(sum - mine, owner);
      bool done = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int rows = __builtin_amdgcn_readlane(there[i], owner), tiles = tiles_of(rows);
        if (!done && slot < at + tiles) {
          done = true;
          found = RowTile{b0 + owner * per + i, tiles - 1 - (slot - at), __builtin_amdgcn_readlane(start[i], owner), rows,
                          __builtin_amdgcn_readlane(length[i], owner), __builtin_amdgcn_readlane(prefix[i], owner)};
        }
        at += tiles;
      }
      return true;
    }
    before = __builtin_amdgcn_readlane(sum, 63);
  }
  return false;
}

// (256 values, plain, over MXFP8 and MXFP4: 8 and 20 bytes of scratch a lane beside all 512 registers.)
// DP: values of a row in LDS, of which the first DV are multiplied.  RW: waves that share keys, each with 32 rows of its own; the other
// 4 / RW - 1 such groups have the same rows and other keys.
// BEND: what is done to scores ahead of the weights; ANY looks what, and takes all steps one instruction after the other.
template <int DP, int DV, int FMT, int BEND, int RW>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DP * (4 / RW) > 128 ? 1 : 2, DP * (4 / RW) > 128 ? 1 : 2))) chunk_attention_kernel(ChunkArgs a) {
  constexpr bool SCALED = FMT != FMT_BF16;
  constexpr int BITS = FMT == FMT_BF16 ? 16 : FMT == FMT_MXFP8 ? 8 : 4;
  constexpr int KP = 4 / RW, WK = CHUNK_STEP / RW;              // groups of waves with keys of their own; keys that a wave brings
  constexpr bool DIRECT = FMT == FMT_BF16;                      // from memory straight into LDS
  constexpr int LANE = WK * DP * BITS / 512;                    // bytes of a lane's loads of them
  constexpr int WIDE = DP * BITS / 32 < 16 ? DP * BITS / 32 : 16, W = LANE < WIDE ? LANE : WIDE, L = LANE / W;   // (a load's keys lie in one page)
  constexpr int PER = DP * BITS / 8 / W;                        // lanes of a key
  constexpr int VALUES = W * 8 / BITS;                          // of a load
  constexpr int SCALE_OF = 4 * BITS, KS = DV / 16, IB = DV / 32, SIDE = CHUNK_STEP * DP * 2;
  typedef KLayout<DP> K;
  constexpr int SETS = 2;                                       // steps whose loads are on their way in registers
  static_assert(W >= 4 && 64 % PER == 0 && (64 / PER <= 16) && WK <= 16);
  constexpr int SLOTS = 4, ROWS = 32 * RW, PITCH = 9, RING = KP * SLOTS * (K::BYTES + SIDE), JOIN = KP * ROWS * (PITCH * 16 + 8);
  __shared__ __attribute__((aligned(1024))) char lds[RING > JOIN ? RING : JOIN];     // [keys' group][K, V][step by turns]; then what is put together
  __shared__ int strange;                                       // a value that is not finite has been left out
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
  const int rp = wave % RW, kp = wave / RW;
  char *const ring_k = lds + kp * SLOTS * (K::BYTES + SIDE), *const ring_v = ring_k + SLOTS * K::BYTES;
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };

  // the workgroup's key head, part and row tile (all key heads of a part side by side: with 8 of them one for each XCD's L2; the last rows of a request,
  // which have the most keys, first)
  const int kv_head = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, split = rest % a.splits, slot = rest / a.splits;
  RowTile it;
  if (!row_tile_of(a, slot, it)) return;
  const int b = uniform(it.b), row_tile = uniform(it.tile), q_at = uniform(it.q_at), each = a.rule.heads_each;
  const int fresh = uniform(min(it.rows_there, a.rule.most)), length = uniform(length_of(a, it.length)), first = uniform(it.length - it.rows_there);
  const int prefix = uniform(min(max(it.prefix, 0), length));
  const int window = a.rule.window, rows = fresh * each, row0 = row_tile * a.tile_rows;
  auto low_of = [&](int p) { return window && p >= window ? p - window + 1 : 0; };
  auto position_of = [&](int row) { return first + min(row, rows - 1) / each; };
  // steps over the keys: those of the prefix, then those from the first to the last that some row sees, `skip` of them left out between
  const int wg_first = uniform(position_of(row0)), wg_last = uniform(position_of(row0 + a.tile_rows - 1));
  const int prefix_steps = (prefix + CHUNK_STEP - 1) / CHUNK_STEP;
  const int all = max((max(min(wg_last + 1, length), 0) + CHUNK_STEP - 1) / CHUNK_STEP, prefix_steps);
  const int skip = max(min(low_of(wg_first) / CHUNK_STEP, all) - prefix_steps, 0), steps = all - skip;
  const int begin = (int)((int64_t)steps * split / a.splits), end = (int)((int64_t)steps * (split + 1) / a.splits);
  // this wave's: every KP-th, the same number for all of them
  const int count = (end - begin + KP - 1) / KP;
  auto key_of = [&](int j) {                        // the first key of the wave's step j; past the end: the length
    const int step = begin + j * KP + kp;
    return step >= end ? length : (step < prefix_steps ? step : step + skip) * CHUNK_STEP;
  };

  // this lane's row
  const bool wave_in = row0 + rp * 32 < rows;
  const int row = row0 + rp * 32 + n, token = row / each, head = kv_head * each + row - token * each;
  const bool in = row < rows;
  const int position = first + token, low = low_of(position), span = max(min(position + 1, length) - low, 0);     // it sees the window's `span` keys from low on
  const float slope = BEND >= BEND_SLOPES && a.rule.slopes && in ? slope_of(a, head) : 0.0f;
  bf16x8 q[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int i = 16 * s + 8 * h;
    u32x4 v = {0, 0, 0, 0};
    if (in && i < a.dim) v = *reinterpret_cast<const u32x4 *>(a.q + (int64_t)(q_at + token) * a.q_stride + (int64_t)head * a.q_head_stride + i);
    if (BEND == BEND_NONE && a.flip) v ^= 0x80008000u;
    q[s] = as_bf16(v);
  }

  // Where the keys lie.  A lane looks up one of the 64 groups of 16 keys of 32 steps from w on, two windows ahead of their use: its page, then its place in
  // bytes, and whether it has none.
  const int *const table = a.tables + b * a.table_stride;
  auto group_of = [&](int w) { return max(min(key_of(w + lane / 2) / 16 + (lane & 1), (length - 1) / 16), 0); };
  auto entry_of = [&](int group) { return (int)((uint64_t)(uint32_t)group * (uint64_t)a.page16_magic >> 38); };
  struct Window {
    int low, high;
    uint64_t lost;
  };
  auto window_of = [&](int w, int page) {
    const int group = group_of(w), entry = entry_of(group);
    const bool gone = (uint32_t)page >= (uint32_t)a.pages;
    const int64_t at = (gone ? 0 : page) * a.page_bytes + (kv_head * a.head_bytes + (int64_t)(16 * (group - entry * (a.page_size / 16)) * a.token_bytes));
    return Window{(int)at, (int)(at >> 32), __ballot(gone)};
  };
  // The wave's steps whose keys every row of the workgroup sees, if they have pages: those before sure_steps, and sure_count from sure_first on.
  int sure_steps = 0, sure_first = 0, sure_count = 0;
  {
    auto first_from = [&](int step) { return max((step - begin - kp + KP - 1) / KP, 0); };            // its first step that is `step` or later
    const int sure_from = low_of(wg_last), sure_to = min(wg_first, length - 1) - (CHUNK_STEP - 1);      // first keys of steps without a prefix
    sure_steps = first_from(min(prefix / CHUNK_STEP, end));
    if (sure_to >= sure_from) {
      const int from = max((sure_from + CHUNK_STEP - 1) / CHUNK_STEP, skip ? prefix_steps + skip : 0) - skip, to = sure_to / CHUNK_STEP - skip + 1;
      sure_first = first_from(from), sure_count = max(first_from(min(to, end)) - sure_first, 0);
    }
  }
  auto edge_at = [&](int j, int lost) { return lost || !(j < sure_steps || (uint32_t)(j - sure_first) < (uint32_t)sure_count); };
  auto base_of = [&](const void *base, int64_t at) {
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(reinterpret_cast<uint64_t>(base) + at), 0, 16 * a.token_bytes, 0x00020000);
  };
  // (loads of keys behind the length stay within their pages; their scores are masked, and what of their values is not finite is left out)
  const int load_at = lane % PER, load_key = lane / PER + rp * WK, where = (load_key & 15) * a.token_bytes + load_at * W;
  const bool load_in = load_at * VALUES < a.dim;
  uint32_t k[SETS][L][W / 4], v[SETS][L][W / 4];
  uint8_t k_scales[SETS][L], v_scales[SETS][L];
  auto load = [&](const char *base, const uint8_t *base_scales, int64_t at, uint32_t (&x)[L][W / 4], uint8_t (&scales)[L]) {
    const __amdgpu_buffer_rsrc_t r = base_of(base, at);
    __amdgpu_buffer_rsrc_t rs;
    if constexpr (SCALED) rs = base_of(base_scales, at / SCALE_OF);
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int from = where + 64 / PER * i * a.token_bytes;
      const auto y = buffer_load<W, false>(r, load_in ? from : ATT_FAR);
      if constexpr (W == 4) x[i][0] = y;
      else
#pragma unroll
        for (int c = 0; c < W / 4; ++c) x[i][c] = y[c];
      if constexpr (SCALED) scales[i] = __builtin_amdgcn_raw_buffer_load_b8(rs, load_in ? from / SCALE_OF : ATT_FAR, 0, 0);
    }
  };
  // straight into LDS: 64 pieces of 16 bytes in a row, so a lane brings the piece that lies at its place there
  constexpr int PIECES_IN = DP / 8, DL = WK / K::GROUP_ROWS > 0 ? WK / K::GROUP_ROWS : 1;
  int k_from[DL], v_from[DL];
  if constexpr (DIRECT)
#pragma unroll
    for (int i = 0; i < DL; ++i) {
      const int key = rp * WK + lane / PIECES_IN + K::GROUP_ROWS * i, at = (key & 15) * a.token_bytes;
      const int k_piece = lane % PIECES_IN ^ K::by(key), v_piece = (v_place<DP>(key, lane % PIECES_IN) - key * DP * 2) / 16;
      k_from[i] = 8 * k_piece < a.dim ? at + 16 * k_piece : ATT_FAR, v_from[i] = 8 * v_piece < a.dim ? at + 16 * v_piece : ATT_FAR;
    }
  auto bring = [&](const char *base, int64_t at, char *to, int pitch, const int (&from)[DL]) {
    const i32x4 r = raw_buffer(reinterpret_cast<const void *>(reinterpret_cast<uint64_t>(base) + at), 16 * a.token_bytes);
    const uint32_t to_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)to + rp * DL * pitch;
#pragma unroll
    for (int i = 0; i < DL; ++i) load_to_lds16<false>(r, to_lds + i * pitch, from[i], 0);
  };
  auto widened = [&](const uint32_t (&x)[L][W / 4], const uint8_t (&scales)[L], int i, int piece) {      // 8 values
    const float scale = SCALED ? __uint_as_float((uint32_t)scales[i] << 23) : 0.0f;
    if constexpr (FMT == FMT_BF16) return u32x4{x[i][0], x[i][1], x[i][2], x[i][3]};
    else if constexpr (FMT == FMT_MXFP4) return widen8(x[i][piece], scale);
    else {
      uint32_t w[4];
      widen4(x[i][2 * piece], scale, w[0], w[1]);
      widen4(x[i][2 * piece + 1], scale, w[2], w[3]);
      return u32x4{w[0], w[1], w[2], w[3]};
    }
  };
  auto put_k = [&](int turn, const uint32_t (&x)[L][W / 4], const uint8_t (&scales)[L]) {
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
      for (int piece = 0; piece < VALUES / 8; ++piece)
        *reinterpret_cast<u32x4 *>(ring_k + turn * K::BYTES + K::at(load_key + 64 / PER * i, load_at * (VALUES / 8) + piece)) = widened(x, scales, i, piece);
  };
  // eight values of which what is not finite is left out: where not every row sees the key, 0 times that is no 0
  auto finite = [&](u32x4 w) {
    bool left_out = false;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t lo = (w[c] & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u, hi = (w[c] & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u;
      left_out |= (lo | hi) != 0;
      w[c] &= ~(lo | hi);
    }
    if (left_out) strange = 1;
    return w;
  };
  auto put_v = [&](int turn, const uint32_t (&x)[L][W / 4], const uint8_t (&scales)[L], bool edge) {
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
      for (int piece = 0; piece < VALUES / 8; ++piece) {
        u32x4 w = widened(x, scales, i, piece);
        if (edge) w = finite(w);
        *reinterpret_cast<u32x4 *>(ring_v + turn * SIDE + v_place<DP>(load_key + 64 / PER * i, load_at * (VALUES / 8) + piece)) = w;
      }
  };

  f32x16 o[IB];                                     // O^T, 32 values each
#pragma unroll
  for (int i = 0; i < IB; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[i][r] = 0.0f;
  float m = -INFINITY, l = 0.0f;                    // m in the exponent of 2
  const float c = a.c;
  // this lane's pieces of its key
  int k_base[2] = {K::at(n, h), K::at(n, h + (DP < 256 ? 2 : 0))};
  // where this lane's part of four keys' values lies, those of i = 0 ... 31 of the keys 4 h ... 4 h + 3
  constexpr int VB = DP == 64 ? 2 : 4;
  const int v_key = 4 * h + (lane & 15) / 4, v_piece = 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
  int v_base[VB];
#pragma unroll
  for (int i = 0; i < VB; ++i) v_base[i] = v_place<DP>(v_key, 4 * i + v_piece) + (lane & 1) * 8;
  typedef __attribute__((address_space(3))) i16x4 *lds_i16x4;

  // What a step computes: KS products for the scores of the next one's keys, 2 IB with the weights of the last one's, and this one's weights, in pieces.
  auto k_operand = [&](int turn, int s) {
    return as_bf16(*reinterpret_cast<const u32x4 *>(ring_k + k_base[DP < 256 ? s % 2 : 0] + (turn * K::BYTES + (DP < 256 ? s / 2 * 64 : s * 32))));
  };
  auto v_operand = [&](int turn, int i) {           // of the products with 16 keys of 32 values
    const char *const at = ring_v + v_base[i % IB % VB] + (turn * SIDE + i % IB / VB * (VB * 64) + i / IB * 16 * DP * 2);
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(at + 8 * DP * 2));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto score = [&](f32x16 &st, bf16x8 operand, int s) {
    if (s == 0)
#pragma unroll
      for (int r = 0; r < 16; ++r) st[r] = 0.0f;
    st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand, q[s], st, 0, 0, 0);
  };
  auto product = [&](bf16x8 operand, const u32x4 (&pt)[2], auto number) {
    constexpr int I = decltype(number)::value;
    o[I % IB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand, as_bf16(pt[I / IB]), o[I % IB], 0, 0, 0);
  };
  // One after the other at every step where a workgroup's four waves share the keys: weights among the products take registers that two waves a SIMD (up to
  // 128 values) do not have, nor one of 256 values over 8 bits, and two waves fill one another's gaps without that.  Mixed / in turn, 8 prompts of 1024
  // tokens, 32 and 8 heads, us:
  //   values  bf16         MXFP8        MXFP4
  //   64      94.2 / 95.6  102 / 104    102 / 103
  //   96      114 / 115    126 / 126    124 / 125
  //   128     151 / 133    222 / 145    179 / 142     capped, MXFP8: 542 / 174, with slopes: 302 / 171
  //   192     279 / 286    309 / 319    313 / 318
  //   256     339 / 338    530 / 403    419 / 401
  // (64 and 192 lose up to 3 % by it.)  Not with 64 rows, one wave a SIMD whose registers hold both: 32 requests of 5 tokens in MXFP4 139 / 182.
  constexpr bool IN_TURN = BEND == BEND_ANY || RW == 4;
  constexpr int PIECES = 13;
  float top, base, alpha;
  bool moved = false;
  auto piece = [&](auto at_edge, int number, int key0, int lost, f32x16 &st, u32x4 (&weights)[2]) {
    constexpr bool EDGE = decltype(at_edge)::value;
    const int i = number, from = key0 + 4 * h;
    if (i < 4) {
      if constexpr (BEND == BEND_ANY) {
        // (four at a time: which way is the same for all)
        if (a.any_cap == CAP_SHORT) {
#pragma unroll
          for (int r = 4 * i; r < 4 * i + 4; ++r) st[r] = __builtin_amdgcn_rcpf(-1.0f - __builtin_amdgcn_exp2f(st[r] * a.rule.cap_in)) * a.scale_log2;
        } else if (a.any_cap == CAP_LONG) {
#pragma unroll
          for (int r = 4 * i; r < 4 * i + 4; ++r) st[r] = capped(st[r], a.rule.cap_in, 1.0f) * a.scale_log2;
        } else {
#pragma unroll
          for (int r = 4 * i; r < 4 * i + 4; ++r) st[r] *= a.scale_log2;
        }
      }
#pragma unroll
      for (int r = 4 * i; r < 4 * i + 4; ++r) {
        const int t = 8 * (r / 4) + r % 4;
        // (a row's scores are as good less a number of its own, so -1 / (1 + e^2y) does for tanh(y) / 2, to 2^-24)
        if constexpr (BEND == BEND_CAP) st[r] = __builtin_amdgcn_rcpf(-1.0f - __builtin_amdgcn_exp2f(st[r] * a.rule.cap_in));
        if constexpr (BEND == BEND_SLOPES) st[r] = __builtin_fmaf(st[r], a.scale_log2, -slope * fabsf((float)(position - from) - (float)t));
        if constexpr (BEND == BEND_ANY) st[r] -= slope * fabsf((float)(position - from) - (float)t);
        if constexpr (EDGE) {
          const bool seen = ((uint32_t)(from - low + t) < (uint32_t)span) | (from - prefix + t < 0);
          st[r] = (seen & !(lost >> (r / 8) & 1)) ? st[r] : -INFINITY;
        }
        top = r ? fmaxf(top, st[r]) : st[r];
      }
    } else if (i == 4) {
      const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      const float most = fmaxf(__uint_as_float(halves[0]), __uint_as_float(halves[1])) * c;
      moved = most - m > 8.0f;
      const float now = moved ? most : m;
      alpha = moved ? __builtin_amdgcn_exp2f(m - now) : 1.0f;
      m = now, base = now == -INFINITY ? 0.0f : now;
      l *= alpha;
    } else {
      const int r = 2 * (i - 5);
      const bf16x2 pair = {(__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(st[r], c, -base)),
                           (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(st[r + 1], c, -base))};
      l = __builtin_amdgcn_fdot2_f32_bf16(pair, bf16x2{(__bf16)1.0f, (__bf16)1.0f}, l, false);
      weights[r / 8][r % 8 / 2] = __builtin_bit_cast(uint32_t, pair);
    }
  };
  // Step j: the scores of step j + 1, the weights of j and the products of j - 1, none of which needs another.  Meanwhile what later steps need is on its
  // way into LDS, step x into slot x % SLOTS: straight from memory K of j + 3 and V of j + 2, or through registers K of j + 2 and V of j, with the loads for
  // SETS steps later.
  f32x16 st[2];
  u32x4 pt[2][2];
  if (tid == 0) strange = 0;
  if (count > 0) {
    constexpr int FAR = DIRECT ? 3 : 4;             // of the steps ahead, the one whose K sets out
    int w = 0;
    Window here = window_of(0, table[entry_of(group_of(0))]);
    int next = table[entry_of(group_of(32))], lost_ahead = 0;
    const int group = RW == 2 ? rp : rp / 2;        // of a step's two, the one that this wave brings keys of
    auto place = [&](int x) -> int64_t {            // of step x, which is a step later each time
      if (x == w + 32) {
        w = x;
        here = window_of(w, next);
        next = table[entry_of(group_of(w + 32))];
      }
      const int i = 2 * (x - w);
      lost_ahead = lost_ahead >> 2 | ((int)(here.lost >> i) & 3) << 2 * FAR;
      return (int64_t)__builtin_amdgcn_readlane(here.high, i + group) << 32 | (uint32_t)__builtin_amdgcn_readlane(here.low, i + group);
    };
    int64_t before[2];                              // places of the last two steps whose K has set out, the last first
    if constexpr (DIRECT) {
#pragma unroll
      for (int x = 0; x < 3; ++x) {
        before[0] = place(x);
        bring(a.k, before[0], ring_k + x * K::BYTES, K::GROUP, k_from);
        if (x < 2) bring(a.v, before[0], ring_v + x * SIDE, 1024, v_from);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    } else {
      const int64_t first_place = place(0), second_place = place(1);
      load(a.k, a.k_scales, first_place, k[0], k_scales[0]);
      load(a.k, a.k_scales, second_place, k[1], k_scales[1]);
      load(a.v, a.v_scales, first_place, v[0], v_scales[0]);
      load(a.v, a.v_scales, second_place, v[1], v_scales[1]);
      put_k(0, k[0], k_scales[0]);
      put_k(1, k[1], k_scales[1]);
      before[1] = place(2), before[0] = place(3);
      load(a.k, a.k_scales, before[1], k[0], k_scales[0]);
      load(a.k, a.k_scales, before[0], k[1], k_scales[1]);
    }
    __syncthreads();
    static_for<KS>([&](auto s) {
      if (s % 2 == 0) __builtin_amdgcn_sched_barrier(0);
      score(st[0], k_operand(0, s), s);
    });
    auto step = [&](auto with_products, auto parity, int j) {
      constexpr int P = decltype(parity)::value;
      const int64_t now = place(j + FAR);
      const int lost = lost_ahead & 3;
      const bool edge = edge_at(j, lost);
      const int key0 = key_of(j);
      if constexpr (DIRECT) {
        bring(a.k, now, ring_k + (j + 3) % SLOTS * K::BYTES, K::GROUP, k_from);
        bring(a.v, before[0], ring_v + (j + 2) % SLOTS * SIDE, 1024, v_from);
        before[0] = now;
        if (edge) {
#pragma unroll
          for (int i = 0; i < DL; ++i) {
            u32x4 *const at = reinterpret_cast<u32x4 *>(ring_v + j % SLOTS * SIDE + (rp * DL + i) * 1024) + lane;
            *at = finite(*at);
          }
        }
      } else {
        put_k((j + 2) % SLOTS, k[P], k_scales[P]);
        put_v(j % SLOTS, v[P], v_scales[P], edge);
        load(a.k, a.k_scales, now, k[P], k_scales[P]);
        load(a.v, a.v_scales, before[1], v[P], v_scales[P]);
        before[1] = before[0], before[0] = now;
      }
      if (wave_in) {
        constexpr int PRODUCTS = decltype(with_products)::value ? KS + 2 * IB : KS, AHEAD = 2;
        auto operand = [&](int i) { return i < KS ? k_operand(P ^ 1, i) : v_operand(P ^ 1, i - KS); };
        auto multiply = [&](bf16x8 x, auto number) {
          constexpr int I = decltype(number)::value;
          if constexpr (I < KS) score(st[P ^ 1], x, I);
          else product(x, pt[P ^ 1], std::integral_constant<int, I - KS>{});
        };
        bf16x8 x[PRODUCTS];
        if (IN_TURN || edge) {                      // one after the other (edges are few)
          if (!IN_TURN || edge) static_for<PIECES>([&](auto i) { piece(std::true_type{}, i, key0, lost, st[P], pt[P]); });
          else static_for<PIECES>([&](auto i) { piece(std::false_type{}, i, key0, lost, st[P], pt[P]); });
          static_for<PRODUCTS>([&](auto i) {
            if (i % 2 == 0) __builtin_amdgcn_sched_barrier(0);         // (two operands at a time, for the registers)
            multiply(operand(i), i);
          });
        } else {
          // a product, what a later one multiplies, a piece of the weights, and so on in this order
          static_for<AHEAD>([&](auto i) { x[i] = operand(i); });
          static_for<PRODUCTS>([&](auto i) {
            constexpr int I = decltype(i)::value;
            __builtin_amdgcn_sched_barrier(0);
            multiply(x[I], i);
            if constexpr (I + AHEAD < PRODUCTS) x[I + AHEAD] = operand(I + AHEAD);
            static_for<(I + 1) * PIECES / PRODUCTS - I * PIECES / PRODUCTS>(
                [&](auto k) { piece(std::false_type{}, I * PIECES / PRODUCTS + decltype(k)::value, key0, lost, st[P], pt[P]); });
          });
          __builtin_amdgcn_sched_barrier(0);
        }
        if (__any(moved)) {
#pragma unroll
          for (int i = 0; i < IB; ++i) o[i] *= alpha;
        }
      }
      // (the loads of this step stay on their way)
      if constexpr (DIRECT) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * DL) : "memory");
      __syncthreads();
    };
    // (two steps of K from slot 2 on, of V from slot 0 on; then the other way round)
    int k_move = 2 * K::BYTES, v_move = 2 * SIDE;
    auto turn = [&](int (&base)[2], int &move) { base[0] += move, base[1] += move, move = -move; };
    auto finish = [&](auto parity) {                // the products of the last step
      constexpr int P = decltype(parity)::value;
      static_for<2 * IB>([&](auto i) {
        if (i % 2 == 0) __builtin_amdgcn_sched_barrier(0);
        product(v_operand(P, i), pt[P], i);
      });
    };
    step(std::false_type{}, std::integral_constant<int, 0>{}, 0);
    turn(k_base, k_move);
    int j = 1;
    for (; j + 1 < count; j += 2) {
      step(std::true_type{}, std::integral_constant<int, 1>{}, j);
      step(std::true_type{}, std::integral_constant<int, 0>{}, j + 1);
      turn(k_base, k_move);
#pragma unroll
      for (int i = 0; i < VB; ++i) v_base[i] += v_move;
      v_move = -v_move;
    }
    if (j < count) {
      step(std::true_type{}, std::integral_constant<int, 1>{}, j);
      finish(std::integral_constant<int, 1>{});
    } else {
      finish(std::integral_constant<int, 0>{});
    }
  }
  // (what the last steps have set out for steps that are none arrives before LDS is another's, and before the workgroup gives it back)
  if constexpr (DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (strange) {
    // What has been left out: an infinity or NaN for every row that sees its key, whatever the weight.
#pragma nounroll
    for (int j = 0; j < count; ++j) {
      const int key0 = key_of(j);
      if (key0 >= length) continue;
      int page[2], in_page[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int group = min(key0 / 16 + u, (length - 1) / 16), entry = entry_of(group);
        page[u] = uniform(table[entry]), in_page[u] = 16 * (group - entry * (a.page_size / 16));
      }
      if (!edge_at(j, ((uint32_t)page[0] >= (uint32_t)a.pages) + 2 * ((uint32_t)page[1] >= (uint32_t)a.pages))) continue;
#pragma nounroll
      for (int x = 0; x < CHUNK_STEP; ++x) {
        const int key = key0 + x, its_page = x < 16 ? page[0] : page[1], place = (x < 16 ? in_page[0] : in_page[1]) + x % 16;
        if (key >= length || (uint32_t)its_page >= (uint32_t)a.pages) continue;
        const int64_t at = its_page * a.page_bytes + (kv_head * a.head_bytes + (int64_t)(place * a.token_bytes));
        static_for<IB * 4>([&](auto number) {
          constexpr int I = decltype(number)::value / 4, R = decltype(number)::value % 4 * 4;
          const int e = 32 * I + 2 * R + 4 * h;
          if (e >= a.dim) return;
          uint32_t y[2];
          if constexpr (FMT == FMT_BF16) {
            y[0] = reinterpret_cast<const uint32_t *>(a.v + at)[e / 2], y[1] = reinterpret_cast<const uint32_t *>(a.v + at)[e / 2 + 1];
          } else {
            const float scale = __uint_as_float((uint32_t)a.v_scales[at / SCALE_OF + e / 32] << 23);
            if constexpr (FMT == FMT_MXFP8) {
              widen4(*reinterpret_cast<const uint32_t *>(a.v + at + e), scale, y[0], y[1]);
            } else {
              const u32x4 wide = widen8(*reinterpret_cast<const uint16_t *>(a.v + at + e / 2), scale);
              y[0] = wide[0], y[1] = wide[1];
            }
          }
          const bool seen = (((uint32_t)(key - low) < (uint32_t)span) | (key < prefix)) & (m != -INFINITY);
          static_for<4>([&](auto z) {
            constexpr int Z = decltype(z)::value;
            const float value = bf16_bits_to_f32(y[Z / 2] >> 16 * (Z % 2) & 0xFFFFu);
            o[I][R + Z] += seen && !(fabsf(value) < INFINITY) ? value : 0.0f;
          });
        });
      }
    }
  }
  // (looked at anew from here on: what hangs on the row is not kept through the loop)
  int late = lane;
  asm volatile("" : "+v"(late));
  const int n_late = late & 31, h_late = late >> 5;
  const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(halves[0]) + __uint_as_float(halves[1]);
  const int64_t part = (((int64_t)slot * a.kv_heads + kv_head) * a.splits + split) * a.tile_rows;
  // four values of a row of the workgroup's
  auto store = [&](int row, int i, f32x4 x, float top, float sum) {
    if (row0 + row >= rows || i >= a.dim) return;
    if (a.splits > 1) {
      *reinterpret_cast<f32x4 *>(a.part + (part + row) * a.dim + i) = x;
      if (i == 0) a.part_ml[2 * (part + row)] = top, a.part_ml[2 * (part + row) + 1] = sum;
    } else {
      x *= sum != 0.0f ? 1.0f / sum : 0.0f;
      *reinterpret_cast<bf16x4 *>(a.out + ruled_row(a, q_at, kv_head, row0 + row) * a.dim + i) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
    }
  };
  // the groups' put together, 32 values of every row at a time
  f32x4 *const mine = reinterpret_cast<f32x4 *>(lds);
  float *const ml = reinterpret_cast<float *>(mine + KP * ROWS * PITCH);
  const int mine_at = kp * ROWS + rp * 32 + n_late;
  if (h_late == 0) ml[2 * mine_at] = m, ml[2 * mine_at + 1] = l;
  static_for<IB>([&](auto piece_number) {
    constexpr int i = decltype(piece_number)::value;
#pragma unroll
    for (int r = 0; r < 16; r += 4) mine[mine_at * PITCH + r / 2 + h_late] = f32x4{o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]};
    __syncthreads();
    for (int x = tid; x < ROWS * 8; x += 256) {
      const int row = x / 8, piece = x % 8;
      float top = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int w = 0; w < KP; ++w) top = fmaxf(top, ml[2 * (w * ROWS + row)]);
      const float base = top == -INFINITY ? 0.0f : top;
      f32x4 y = {0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < KP; ++w) {
        const float f = __builtin_amdgcn_exp2f(ml[2 * (w * ROWS + row)] - base);
        sum += f * ml[2 * (w * ROWS + row) + 1];
        y += f * mine[(w * ROWS + row) * PITCH + piece];
      }
      store(row, 32 * i + 4 * piece, y, top, sum);
    }
    if (i + 1 < IB) __syncthreads();
  });
}

// Kernels of one width, by the rows of a workgroup: 128 or 64.
template <int DP, int DV>
void go_chunk(const ChunkArgs &a, int format, int bend, unsigned groups, hipStream_t stream) {
  auto of_rows = [&](auto of, auto with, auto waves) {
    hipLaunchKernelGGL((chunk_attention_kernel<DP, DV, decltype(of)::value, decltype(with)::value, decltype(waves)::value>), dim3(groups), dim3(256), 0, stream, a);
  };
  auto of_scores = [&](auto of, auto with) {
    if constexpr (DP < 256)
      if (a.tile_rows == 64) return of_rows(of, with, std::integral_constant<int, 2>{});
    of_rows(of, with, std::integral_constant<int, 4>{});
  };
  auto of_format = [&](auto of) {
    if (bend == BEND_NONE) of_scores(of, std::integral_constant<int, BEND_NONE>{});
    else if (bend == BEND_CAP) of_scores(of, std::integral_constant<int, BEND_CAP>{});
    else if (bend == BEND_SLOPES) of_scores(of, std::integral_constant<int, BEND_SLOPES>{});
    else of_scores(of, std::integral_constant<int, BEND_ANY>{});
  };
  if (format == FMT_BF16) of_format(std::integral_constant<int, FMT_BF16>{});
  else if (format == FMT_MXFP8) of_format(std::integral_constant<int, FMT_MXFP8>{});
  else of_format(std::integral_constant<int, FMT_MXFP4>{});
}
void go_chunk_64(const ChunkArgs &a, int format, int bend, unsigned groups, hipStream_t stream);     // chunk_attention_64.hip, ...
void go_chunk_96(const ChunkArgs &a, int format, int bend, unsigned groups, hipStream_t stream);
void go_chunk_128(const ChunkArgs &a, int format, int bend, unsigned groups, hipStream_t stream);
void go_chunk_192(const ChunkArgs &a, int format, int bend, unsigned groups, hipStream_t stream);
void go_chunk_256(const ChunkArgs &a, int format, int bend, unsigned groups, hipStream_t stream);

}  // namespace torq
