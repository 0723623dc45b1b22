// The attention of one or a few new tokens of each request over its pages, out = softmax(scale q K^T) V for each head, as the kernels of
// paged_attention_mxfp4.hip and paged_attention_scores*.hip run it.  (paged_attention.hip has a kernel of its own for bf16 and MXFP8 without a rule, of the
// same mathematics and work but for the weights' base and the way to the pages: see there.  Arguments, products' operands and joins are these.)
//
// The query heads of a key head are the columns of one matrix product, up to 16, or of two side by side, up to 32, so K and V are
// read once for all of them: HBM-bound, 2 (bf16) or 1 1/32 (MXFP8) bytes for 2 heads / kv_heads flops.
//
// Work: the tokens of every (request, key head) in tiles of 32, all of them in one row of tiles (with room for what each one costs
// besides), cut into equal runs, one for each workgroup: lengths may be as ragged as they like, and the host need not know them, since every
// workgroup adds them up itself.  A run goes through one or several (request, key head)s.  The four waves of a workgroup take turns at
// the tiles of one, each with a softmax of its own in one pass (running maximum m, sum l, unnormalised O), put together in LDS at its end; or
// (few query heads for a key head and many of those, or more query heads than fit a column, whose waves then find the same lines in the cache)
// each has one for itself and they need not wait for one another.  What lies whole within a run is written as output; of the others
// O, m and l go to the workspace, two at most for a run (and wave), and a second kernel joins them in the order of the tokens.  Tables for
// at most 512 tokens (1024 if there are many): one launch, a workgroup for each (request, key head).
//
// A tile goes through the matrix cores transposed, and nothing of it passes between lanes but the column maxima:
//   S^T [token][head] = K [token][i] Q^T [i][head]           v_mfma_f32_16x16x32_bf16, two groups of 16 tokens
//   lane (n = l % 16, g = l / 16) then holds head n's S for tokens 4g + r of both groups, r < 4
//   O^T [i][head] += V^T [i][token] P^T [token][head]        the k index of this product runs over the 32 tokens in the order in
//                                                            which the lanes hold them, so P^T is already its B operand
// Its A operand wants 8 tokens of one i in a lane.  The lane loads, for its 8 tokens, E consecutive values of V (coalesced
// rows), and pairs of them are put together by v_perm_b32: slot j holds V[its tokens][E * (l % 16) + j].
// In MXFP8 the elements are widened to bf16 with their scale in one instruction, which takes of the scale its exponent field (so 0 is 2^-127 and
// 0xFF NaN).  4 bits of significand: exact from scale byte 3 on, whose least element is 2^-133 as bf16's, up to 2^128.
//
// K and V of a wave's next tile are on their way while it works on this one, K from the moment that S is there, V from the
// moment that O is.  The loads are buffer loads over the 16 tokens of a group (a group lies in one page) as far as they are tokens of
// the request: what is past the length, in no page or past the last tile has no records, costs no traffic and comes back as
// zeros, so the loop knows no other case (and a NaN behind the length is not read).
//
// MXFP4 is widened the same way, two codes in an instruction: exact, up to 2^128.
// RULED: scores go by a.rule (a cap, slopes, a window, a prefix), and the columns may be several new tokens of a request times their heads, token by token.
// The tiles between the prefix and the first window are left out of the row of tiles; masks are looked at only in tiles that some row does not see whole, and
// there values that are not finite take a row at a time.
//
// Here (not in paged_attention.hip) the weights are taken against a base that moves only when a score passes it by 2^8, so most tiles leave O alone, and
// where the groups of 16 tokens lie is worked out by the lanes for 32 tiles at a time: with a base that always moves and places by scalar instructions, 45 requests in MXFP4 (as below) took
// 304 us instead of 189, 77 with slopes 116 instead of 98: in MXFP4 a tile is 4.3 KB, and its 400 instructions were the bound, not its bytes.
//
// Measured (paged_attention.hip's, bf16 where not said; called in turn over three caches, 303 MB to 1.9 GB; 7.1 TB/s is what reading alone reaches): 16 requests of 1000 to 8192 tokens, 64 query
// and 8 key heads of 128, 55.2 us = 5.5 TB/s; one of 131072 87.6 us = 6.1; 45 of 8000 to 32768 in MXFP8 312 us = 6.2; 77 with 20 heads of 80 each, 85.9 us = 4.9.  The traffic
// is what has to be read (counters within 1 %); vector instructions take a third (bf16) to half (MXFP8) of the time.  What is left over HBM's time: 5 to 7 us until
// the first tiles are there, 5 for the join and its launch.  One request of 333 tokens 6.2 us, one launch: three rounds that
// hang on one another; compiled apart, since the runs' code in the same kernel cost it 0.45 in a graph and 0.85 in a call.
#pragma once

#include "torq_device.h"
#include "torq_internal.h"

namespace torq {

constexpr int ATT_TILE = 32;          // tokens of a wave's step
constexpr int ATT_WAVES = 4;
constexpr int ATT_ROWS = 16;          // query heads of a product's columns
constexpr int ATT_JOIN = 512;         // threads of a workgroup that joins, at most
// Columns from which each wave has one of its own, with up to 2 query heads for each or head_dim over 128.  77 x 20 heads 120 -> 91 us, 256 requests x 8 key heads
// with 2 query heads each 144.6 -> 139.7; with 4 146.7 -> 151.1, with 8 153 -> 162 (four times the parts to join).  head_dim 256, 4 query heads each, 128 x 8
// of 1000 to 1500 tokens 217 -> 213, MXFP8 of 1000 to 2500 174 -> 164.
constexpr int ATT_WAYS_ITEMS = 768;
// What a (request, key head) costs besides its tiles (its place, its query, putting it together), in tiles of the row of them that is cut
// into runs, by the waves that take turns.  64 requests of 1 to 600 tokens, 64 / 8 heads, with 0, 4, 8, 16: 35.4, 24.1, 23.9, 23.7 us;
// 16 of 1000 to 8192 58.6, 58.7, 59.1, 60.4; 77 x 20 heads, a wave each, with 0, 1, 2, 5: 89.6, 89.8, 92.8, 95.0.
constexpr int att_setup(int ways) { return ways > 1 ? 4 : 1; }
constexpr float ATT_SLACK = 8.0f;    // how far scores may pass the base of the weights, in the exponent of 2
constexpr int ATT_FAR = 0x7FFFFF00;   // an offset past every buffer

// What begins in a run and does not end there: a request, which of the columns that a workgroup works on at a time, the place of its first
// part (that of nothing: -1; the others are first in their runs), its last tile, and the runs' lengths.
struct alignas(16) Cut {
  int b, column, place, last_tile, each, more;
};

// How scores are given beyond scale q . k, and to how many new tokens of a request (RULED kernels).
struct ScoreArgs {
  float cap_in, cap_out;              // cap: cap_out tanh(cap_in q . k), cap_in = scale / cap, cap_out = cap * log2(e); 0: none
  const float *slopes;                // [heads], or null
  const int *prefix, *starts;         // [B] and [B + 1], or null: no prefix, one new token of each request
  int window, most, heads_each;       // tokens that a query sees (0: all); new tokens of a request at most; query heads for a key head
  int64_t tokens;                     // rows of q and out
};

struct AttentionArgs {
  const char *k, *v;
  const uint8_t *k_scales, *v_scales;
  int64_t page_bytes, head_bytes;     // from one to the next
  int pages, token_bytes;
  const uint16_t *q;
  int64_t q_stride, q_head_stride;
  const int *tables, *lengths;
  int64_t table_stride, page16_magic; // t / page_size = (t / 16) * page16_magic >> 38
  int64_t most;                       // width * page_size
  int B, page_size, kv_heads, group, rows, row_groups, dim;            // rows: query heads of a column at most
  float scale_log2;                   // scale * log2(e): the softmax is taken to base 2
  uint16_t *out;
  float *part, *part_ml;              // [run][2][columns at a time][rows][dim] and [2]: O, and m and l, of what is not whole in a run
  Cut *cuts;                          // [run], or [request][columns that a workgroup works on at a time]
  int by_item;
  ScoreArgs rule;                     // (group: rows of a request under a key head at most, `most` times heads_each, token by token)
};

// What a request's new tokens see, as tiles: those of its prefix, then those from the first that its first new token's window holds, `skip` of
// them left out between.  first: the position of its first new token.
struct Reach {
  int length, tiles, fresh, first, prefix, prefix_tiles, skip;
};
__device__ __forceinline__ int length_of(const AttentionArgs &a, int n) { return n < 0 ? 0 : n < a.most ? n : (int)a.most; }
__device__ __forceinline__ Reach reach_of(const AttentionArgs &a, int n, int fresh, int prefix) {
  Reach r;
  r.length = length_of(a, n);
  r.fresh = min(fresh, a.rule.most), r.first = n - fresh;
  r.prefix = min(max(prefix, 0), r.length), r.prefix_tiles = (r.prefix + ATT_TILE - 1) / ATT_TILE;
  const int all = (r.length + ATT_TILE - 1) / ATT_TILE, low = a.rule.window && r.first >= a.rule.window ? r.first - a.rule.window + 1 : 0;
  r.skip = max(min(low / ATT_TILE, all) - r.prefix_tiles, 0);
  r.tiles = r.fresh > 0 ? all - r.skip : 0;
  return r;
}
// rows of q and out that are request b's, [first, behind), whatever `starts` holds
__device__ __forceinline__ int2 rows_of_request(const AttentionArgs &a, int64_t start, int64_t end) {
  start = max((int64_t)0, min(start, a.rule.tokens));
  return make_int2((int)start, (int)max(start, min(end, a.rule.tokens)));
}

// The runs: `tiles` tiles (of a column, or of several side by side) over `runs` workgroups, the first `more` of which have one more
// than the others; a tile at least for each wave.
struct Runs {
  int each, more, runs;
  __device__ Runs(int each, int more) : each(each), more(more), runs(0) {}
  __device__ Runs(int tiles, int groups, int ways) {
    runs = max(1, min(groups, (tiles + ways - 1) / ways));
    each = tiles / runs, more = tiles - each * runs;
  }
  __device__ int begin(int run) const { return run * each + min(run, more); }
  __device__ int of(int tile) const {
    const int wide = more * (each + 1);
    return tile < wide ? tile / (each + 1) : more + (tile - wide) / each;
  }
};

// the row of q and out of a request's row under a key head
__device__ __forceinline__ int64_t ruled_row(const AttentionArgs &a, int q_at, int kv_head, int row) {
  const int token = row / a.rule.heads_each, head = row - token * a.rule.heads_each;
  return ((int64_t)(q_at + token) * a.kv_heads + kv_head) * a.rule.heads_each + head;
}

__device__ __forceinline__ bf16x8 as_bf16(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }
// four E4M3 bytes -> two words of two bf16, times scale
__device__ __forceinline__ void widen4(uint32_t v, float scale, uint32_t &a, uint32_t &b) {
  a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, false));
  b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, true));
}
// eight E2M1 codes, the first in the lowest four bits -> four words of two bf16, times scale
__device__ __forceinline__ u32x4 widen8(uint32_t v, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 3))};
}
// whether one of two bf16 is an infinity or NaN
__device__ __forceinline__ bool not_finite(uint32_t v) { return (v & 0x7F80u) == 0x7F80u || (v & 0x7F800000u) == 0x7F800000u; }
// out tanh(in x).  Small arguments by the series (its next term is 62/2835 of the eighth power, 2^-29 of the result), since 1 - 2 / (1 + e^2y) loses
// their digits; beyond, it is off by 2^-23, so by 2^-20 of the result.
__device__ __forceinline__ float capped(float x, float in, float out) {
  const float y = x * in, y2 = y * y;
  const float small = y * (1.0f + y2 * (-1.0f / 3 + y2 * (2.0f / 15 + y2 * (-17.0f / 315))));
  const float large = 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(2.88539008177792681472f * y));
  return out * (fabsf(y) < 0.125f ? small : large);
}
// A head's slope to base 2.  Magnitudes beyond 1e28 are taken for that: either leaves all the weight to the nearest (or farthest) key, and times 2^31
// tokens it is still finite, where infinities would be NaN at distance 0 or beside one another.
__device__ __forceinline__ float slope_of(const AttentionArgs &a, int head) {
  return 1.44269504088896340736f * fminf(fmaxf(a.rule.slopes[head], -1e28f), 1e28f);
}
typedef const __attribute__((address_space(4))) int *uniform_ints;      // read by scalar loads

// `bytes` bytes from p as a raw buffer; all three the same in every lane
__device__ __forceinline__ __amdgpu_buffer_rsrc_t records(const void *base, int64_t at, int bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base) + at;
  const uint64_t u = (uint32_t)__builtin_amdgcn_readfirstlane((int)p) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(p >> 32)) << 32;
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(u), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
template <int N, bool ONCE>
__device__ __forceinline__ auto buffer_load(__amdgpu_buffer_rsrc_t r, int at) {
  if constexpr (N == 16) return __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, LOAD_POLICY<ONCE>);
  else if constexpr (N == 8) return __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, LOAD_POLICY<ONCE>);
  else if constexpr (N == 4) return __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, LOAD_POLICY<ONCE>);
  else return __builtin_amdgcn_raw_buffer_load_b16(r, at, 0, LOAD_POLICY<ONCE>);
}

// Over the four lanes l, l ^ 16, l ^ 32, l ^ 48 of a column: the rows of 16 lanes (then the halves of the wave) of a register with itself
// exchanged, so that each lane has its own and the other's
template <class F>
__device__ __forceinline__ float over_column(float v, F &&op) {
  const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = op(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
  const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
}

// DP: head_dim rounded up to what the operands hold.  WAYS: 4, the waves take turns at the tiles of a column; 1, each has a column
// of its own and all of its tiles in the run.  RT: products side by side, for up to 16 query heads each.  SOLO: a workgroup for each
// (request, columns that it works on), which is its run.  RULED: scores and new tokens by a.rule.
template <int DP, int FMT, bool ONCE, int WAYS, int RT, bool SOLO, bool RULED>
__device__ __forceinline__ void attention_body(const AttentionArgs &a) {
  constexpr int E = DP < 128 ? DP / 16 : 8;         // consecutive values of V in a lane
  constexpr int NH = DP / (16 * E);                 // such pieces of a row
  constexpr bool SCALED = FMT != FMT_BF16;
  constexpr int BITS = FMT == FMT_BF16 ? 16 : FMT == FMT_MXFP8 ? 8 : 4, ROWS = ATT_ROWS * RT;
  constexpr int KW = DP * BITS / 32 < 16 ? DP * BITS / 32 : 16;   // bytes of a lane's load of K
  constexpr int KL = DP * BITS / (32 * KW);         // such loads of a lane for a group of 16 rows of K
  constexpr int KE = KW * 8 / BITS;                 // values of one
  constexpr int KS = DP / 32;                       // k-steps of S
  constexpr int VW = E * BITS / 8;                  // bytes of a lane's load of V
  constexpr int SCALE_OF = 4 * BITS;                // bytes of elements for one of scales
  __shared__ f32x4 o_all[WAYS][ATT_ROWS][WAYS > 1 ? 4 * E + 1 : 1];       // a piece of O at a time
  __shared__ float m_all[WAYS][ROWS], l_all[WAYS][ROWS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
  // (key head, rows) of a request, as many at a time as the workgroup works on
  const int columns = (a.kv_heads * a.row_groups + ATT_WAVES / WAYS - 1) / (ATT_WAVES / WAYS), way = WAYS > 1 ? wave : 0;
  const uniform_ints lengths = (uniform_ints)(uintptr_t)a.lengths;

  // one (request, column), as far as it lies in the run: its tiles first ... last - 1 of `tiles`; end: the place behind them
  struct Segment {
    int b, column, tiles, length, kv_head, rows_at, first, last, end;
    int q_at, fresh, position, prefix, prefix_tiles, skip;            // RULED: its first row, and see Reach
  };
  // rows of a request under a key head; the tile at place i of the row of its tiles
  auto rows_in = [&](const Segment &s) { return RULED ? s.fresh * a.rule.heads_each : a.group; };
  auto tile_at = [](const Segment &s, int i) { return RULED && i >= s.prefix_tiles ? i + s.skip : i; };
  const int run = (int)blockIdx.x;
  int run_begin = 0, run_end = 0, tiles_each = 1, tiles_more = 0;
  // (all of it the same in every lane of a wave, which the compiler does not see through the loops: scalar registers)
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  auto place_column = [&](Segment &s, int column) {
    s.column = uniform(column);
    column = uniform(WAYS == 1 ? column * ATT_WAVES + wave : column);
    s.kv_head = a.row_groups == 1 ? column : uniform(column / a.row_groups), s.rows_at = column - s.kv_head * a.row_groups;
    if (s.kv_head >= a.kv_heads) s.kv_head = 0, s.rows_at = a.row_groups;      // (no column: no tile of it is there, and no row)
  };
  auto take_request = [&](Segment &s, int b, int length) {
    s.b = uniform(b), s.length = uniform(length), s.tiles = (s.length + ATT_TILE - 1) / ATT_TILE;
  };
  auto rows_by = [&](auto starts, int b) { return starts ? rows_of_request(a, starts[b], starts[b + 1]) : make_int2(b, b + 1); };
  auto take_ruled = [&](Segment &s, int b) {
    s.b = uniform(b);
    const int2 rows = rows_by((uniform_ints)(uintptr_t)a.rule.starts, s.b);
    const Reach r = reach_of(a, lengths[s.b], rows.y - rows.x, a.rule.prefix ? ((uniform_ints)(uintptr_t)a.rule.prefix)[s.b] : 0);
    s.q_at = uniform(rows.x), s.length = uniform(r.length), s.tiles = uniform(r.tiles), s.fresh = uniform(r.fresh), s.position = uniform(r.first);
    s.prefix = uniform(r.prefix), s.prefix_tiles = uniform(r.prefix_tiles), s.skip = uniform(r.skip);
  };
  auto reach_at = [&](int b) {                      // by a lane
    const int2 rows = rows_by(a.rule.starts, b);
    return reach_of(a, a.lengths[b], rows.y - rows.x, a.rule.prefix ? a.rule.prefix[b] : 0);
  };
  auto places_of = [](int tiles) { return tiles ? tiles + att_setup(WAYS) : 0; };
  // the one behind s, which the run goes on with
  auto behind_of = [&](Segment s) {
    int column = s.column + 1;
    if (column == columns) {
      do {
        if constexpr (RULED) take_ruled(s, s.b + 1);
        else take_request(s, s.b + 1, length_of(a, lengths[s.b + 1]));
      } while (s.tiles == 0);
      column = 0;
    }
    place_column(s, column);
    s.end += att_setup(WAYS);
    s.first = 0, s.last = min(run_end - s.end, s.tiles), s.end += s.last;
    return s;
  };
  // requests without tokens: zeros, and nothing to join
  auto zeros = [&] {
    if constexpr (RULED) {
      for (int b = run; b < a.B; b += gridDim.x) {
        Segment s;
        take_ruled(s, b);
        if (s.tiles) continue;
        if (a.by_item)
          for (int x = tid; x < columns; x += 256) a.cuts[b * columns + x] = Cut{0, 0, -1, 0, 1, 0};
        const int64_t row = (int64_t)a.kv_heads * a.rule.heads_each * a.dim / 8;
        for (int64_t x = tid; x < s.fresh * row; x += 256) reinterpret_cast<u32x4 *>(a.out)[s.q_at * row + x] = u32x4{0, 0, 0, 0};
      }
      return;
    }
    for (int b = run; b < a.B; b += gridDim.x)
      if (length_of(a, lengths[b]) == 0) {
        if (a.by_item)
          for (int x = tid; x < columns; x += 256) a.cuts[b * columns + x] = Cut{0, 0, -1, 0, 1, 0};
        for (int x = tid; x < a.kv_heads * a.group * a.dim / 8; x += 256)
          reinterpret_cast<u32x4 *>(a.out + (int64_t)b * a.kv_heads * a.group * a.dim)[x] = u32x4{0, 0, 0, 0};
      }
  };
  Segment seg;
  if constexpr (SOLO) {
    const int b = blockIdx.x / columns, column = blockIdx.x - b * columns;
    if constexpr (RULED) {
      take_ruled(seg, b);
      seg.first = 0, seg.last = seg.tiles, seg.end = 0;
    } else {
      const int length = length_of(a, lengths[b]), tiles = (length + ATT_TILE - 1) / ATT_TILE;
      seg = Segment{b, 0, tiles, length, 0, 0, 0, tiles, 0};      // (end: that of no run)
    }
    place_column(seg, column);
  } else {
    // places of one column, request by request: every wave adds them up, a lane those of `per` requests (eight loads at a time)
    const int per = (a.B + 63) / 64;
    // (RULED: tiles instead)
    auto length_at = [&](int b) {
      if constexpr (RULED) return b < a.B ? reach_at(b).tiles : 0;
      else return b < a.B ? length_of(a, a.lengths[b]) : 0;
    };
    auto tiles_in = [](int length) { return RULED ? length : (length + ATT_TILE - 1) / ATT_TILE; };
    int mine = 0, length = 0;
    if (per == 1) {
      length = length_at(lane);
      mine = places_of(tiles_in(length));
    } else {
      for (int i0 = 0; i0 < per; i0 += 8) {
        int read[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) read[i] = i0 + i < per ? length_at(lane * per + i0 + i) : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) mine += places_of(tiles_in(read[i]));
      }
    }
    int sum = wave_sum(mine);
    const int total = __builtin_amdgcn_readlane(sum, 63);
    const Runs runs(total * columns, gridDim.x, WAYS);
    run_begin = uniform(runs.begin(min(run, runs.runs))), run_end = uniform(runs.begin(min(run + 1, runs.runs)));
    if (run_begin == run_end) {                     // (fewer tiles than workgroups)
      if (tid == 0 && !a.by_item) a.cuts[run] = Cut{0, 0, -1, 0, 1, 0};
      zeros();
      return;
    }
    // the lane whose requests the run begins in; then the request, 64 of them at a time
    int owner = __builtin_ctzll(__ballot(run_begin < sum * columns)), before = __builtin_amdgcn_readlane(sum - mine, owner), b = owner;
    if (per > 1) {
      for (int b0 = owner * per;; b0 += 64) {
        length = length_at(b0 + lane);
        mine = places_of(tiles_in(length));
        sum = before + wave_sum(mine);
        const uint64_t behind_it = __ballot(run_begin < sum * columns);
        if (behind_it) {
          owner = __builtin_ctzll(behind_it), b = b0 + owner;
          before = __builtin_amdgcn_readlane(sum - mine, owner);
          break;
        }
        before = __builtin_amdgcn_readlane(sum, 63);
      }
    }
    if constexpr (RULED) take_ruled(seg, b);
    else take_request(seg, b, __builtin_amdgcn_readlane(length, owner));
    const int into = run_begin - before * columns, column = uniform(into / places_of(seg.tiles));
    place_column(seg, column);
    // tile t of a column has the place att_setup + t from its beginning
    const int tile0 = run_begin - into + column * places_of(seg.tiles) + att_setup(WAYS);
    seg.first = max(run_begin - tile0, 0), seg.last = min(run_end - tile0, seg.tiles), seg.end = tile0 + seg.last;
    if (seg.last <= 0) {                            // (the run ends ahead of the first tile)
      if (tid == 0 && !a.by_item) a.cuts[run] = Cut{0, 0, -1, 0, 1, 0};
      zeros();
      return;
    }
    tiles_each = uniform(runs.each), tiles_more = uniform(runs.more);
  }

  // what a lane reads of a group of 16 tokens, in bytes from its first token
  const int k_at = n * a.token_bytes + KW * g, v_at = 4 * g * a.token_bytes + VW * n;
  // Q^T as the B operand: column n, the i of this lane's K values
  bf16x8 q[RT][KS];
  int position[RT], low[RT];                        // RULED: of this lane's column, and the first token that its window holds
  float slope[RT];
  auto load_q = [&](const Segment &s) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = s.rows_at * ROWS + rt * ATT_ROWS + n;       // query head of this lane's column within the group
      const uint16_t *from = a.q + s.b * a.q_stride + (int64_t)(s.kv_head * a.group + row) * a.q_head_stride;
      if constexpr (RULED) {
        const int token = row / a.rule.heads_each, head = s.kv_head * a.rule.heads_each + row - token * a.rule.heads_each;
        position[rt] = s.position + token;
        low[rt] = a.rule.window && position[rt] >= a.rule.window ? position[rt] - a.rule.window + 1 : 0;
        slope[rt] = a.rule.slopes && row < rows_in(s) ? slope_of(a, head) : 0.0f;
        from = a.q + (int64_t)(s.q_at + token) * a.q_stride + (int64_t)head * a.q_head_stride;
      }
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        const int i = 4 * KE * (8 * t / KE) + KE * g + 8 * t % KE;
        u32x4 v = {0, 0, 0, 0};
        if (row < rows_in(s) && i < a.dim) v = *reinterpret_cast<const u32x4 *>(from + i);
        q[rt][t] = as_bf16(v);
      }
    }
  };
  // the pages of a tile's two groups of 16 tokens, and where in them the groups begin; how many of a group are tokens; where they lie, in bytes
  struct Pages {
    int page[2], in_page[2];
  };
  auto look_up = [&](const Segment &s, int tile) {
    Pages p;
    const uniform_ints table = (uniform_ints)(uintptr_t)(a.tables + s.b * a.table_stride);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int t16 = max(min(2 * tile_at(s, tile) + u, (s.length - 1) / 16), 0), entry = (int)((uint64_t)(uint32_t)t16 * (uint64_t)a.page16_magic >> 38);
      p.page[u] = s.length > 0 ? table[entry] : -1;
      p.in_page[u] = 16 * (t16 - entry * (a.page_size / 16));
    }
    return p;
  };
  struct Place {
    int count[2], bytes[2];                         // tokens; bytes of the cache from the first to the end of the last
    int64_t at[2];
  };
  // Where the groups of a wave's next 32 tiles of a segment lie, a lane each.  The lanes work out together what takes a wave alone 100 scalar
  // instructions for a tile; the tile's own then reads it lane by lane.
  struct Window {
    int page, t16, left, count, bytes;
    uint32_t at_lo, at_hi;
  };
  auto look_ahead = [&](const Segment &s, int tile0) {            // its first; the pages are on the way
    Window w;
    const int tile = tile0 + lane / 2 * WAYS;
    w.t16 = 2 * tile_at(s, tile) + (lane & 1);
    const int entry = (int)((uint64_t)(uint32_t)max(w.t16, 0) * (uint64_t)a.page16_magic >> 38);
    const bool rows = RULED ? s.rows_at * ROWS < rows_in(s) && s.rows_at < a.row_groups : s.rows_at < a.row_groups;
    w.left = tile < s.last && rows ? max(s.length - 16 * w.t16, 0) : 0;
    w.page = w.left ? a.tables[s.b * a.table_stride + entry] : -1;
    return w;
  };
  auto work_out = [&](const Segment &s, Window &w) {
    const int entry = (int)((uint64_t)(uint32_t)max(w.t16, 0) * (uint64_t)a.page16_magic >> 38);
    const bool there = (uint32_t)w.page < (uint32_t)a.pages;      // (a page that is none: as a number without a sign past all others)
    w.count = there ? min(w.left, 16) : 0;
    w.bytes = w.count ? (w.count - 1) * a.token_bytes + a.dim * BITS / 8 : 0;
    const int64_t at = (there ? w.page : 0) * a.page_bytes + (s.kv_head * a.head_bytes + (int64_t)(16 * (w.t16 - entry * (a.page_size / 16)) * a.token_bytes));
    w.at_lo = (uint32_t)at, w.at_hi = (uint32_t)(at >> 32);
  };
  auto place_at = [&](const Window &w, int i) {
    Place p;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      p.count[u] = __builtin_amdgcn_readlane(w.count, 2 * i + u), p.bytes[u] = __builtin_amdgcn_readlane(w.bytes, 2 * i + u);
      p.at[u] = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(w.at_hi, 2 * i + u) << 32 | (uint32_t)__builtin_amdgcn_readlane(w.at_lo, 2 * i + u));
    }
    return p;
  };
  auto place = [&](const Segment &s, int tile, const Pages &p) {
    Place w;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int t = tile_at(s, tile) * ATT_TILE + 16 * u;
      // (a page that is none: as a number without a sign past all others)
      const bool rows = RULED ? s.rows_at * ROWS < rows_in(s) && s.rows_at < a.row_groups : s.rows_at < a.row_groups;
      const int left = tile < s.last && (uint32_t)p.page[u] < (uint32_t)a.pages && rows ? s.length - t : 0;
      w.count[u] = max(min(left, 16), 0);
      w.bytes[u] = w.count[u] ? (w.count[u] - 1) * a.token_bytes + a.dim * BITS / 8 : 0;
      w.at[u] = (left > 0 ? p.page[u] : 0) * a.page_bytes + (s.kv_head * a.head_bytes + (int64_t)(p.in_page[u] * a.token_bytes));
    }
    return w;
  };
  auto rows_of = [&](const char *base, const Place &p, int u) {
    return records(base, p.at[u], p.bytes[u]);
  };
  auto scales_of = [&](const uint8_t *base, const Place &p, int u) {
    return records(base, p.at[u] / SCALE_OF, p.bytes[u] / SCALE_OF);
  };
  uint32_t k[2][KL][KW / 4];
  uint32_t v[2][NH][4][(VW + 3) / 4];
  uint8_t k_scales[2][KL], v_scales[2][NH][4];
  auto load_k = [&](const Place &p) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const __amdgpu_buffer_rsrc_t r = rows_of(a.k, p, u);
#pragma unroll
      for (int s = 0; s < KL; ++s)
      {
        const auto x = buffer_load<KW, ONCE>(r, 4 * KE * s + KE * g < a.dim ? k_at + 4 * KW * s : ATT_FAR);
#pragma unroll
        for (int c = 0; c < KW / 4; ++c) k[u][s][c] = x[c];
      }
      if constexpr (SCALED) {
        const __amdgpu_buffer_rsrc_t rs = scales_of(a.k_scales, p, u);
#pragma unroll
        for (int s = 0; s < KL; ++s)
          k_scales[u][s] = __builtin_amdgcn_raw_buffer_load_b8(rs, 4 * KE * s + KE * g < a.dim ? (k_at + 4 * KW * s) / SCALE_OF : ATT_FAR, 0, 0);
      }
    }
  };
  auto load_v = [&](const Place &p) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const __amdgpu_buffer_rsrc_t r = rows_of(a.v, p, u);
      __amdgpu_buffer_rsrc_t rs;
      if constexpr (SCALED) rs = scales_of(a.v_scales, p, u);
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int where = v_at + e * a.token_bytes + 16 * VW * h;
          const bool in = 16 * E * h + E * n < a.dim;
          const auto x = buffer_load<VW, ONCE>(r, in ? where : ATT_FAR);
          if constexpr (VW <= 4) v[u][h][e][0] = x;
          else
#pragma unroll
            for (int c = 0; c < VW / 4; ++c) v[u][h][e][c] = x[c];
          if constexpr (SCALED) v_scales[u][h][e] = __builtin_amdgcn_raw_buffer_load_b8(rs, in ? where / SCALE_OF : ATT_FAR, 0, 0);
        }
    }
  };

  Pages pages = look_up(seg, seg.first + way);
  Place here = place(seg, seg.first + way, pages);
  load_q(seg);
  __builtin_amdgcn_sched_barrier(0);                // (K ahead of V, as in the loop, whose waits count them)
  load_k(here);
  __builtin_amdgcn_sched_barrier(0);
  load_v(here);
  if constexpr (!SOLO) zeros();
  for (int second = 0;; second = 1) {               // second: the run's second segment, or a later one
    const bool whole = seg.first == 0 && seg.last == seg.tiles;
    // what comes behind this segment: its first tile is on the way when this one's last is worked on
    Segment behind = seg;
    behind.last = 0;                                // (no tile of it is there)
    if (!SOLO && seg.end < run_end) behind = behind_of(seg);
    const bool more = !SOLO && behind.last > 0;
    if (!SOLO && tid == 0 && (a.by_item ? seg.first == 0 : !more)) {
      a.cuts[a.by_item ? seg.b * columns + seg.column : run] = Cut{
          seg.b, seg.column, seg.first == 0 && !whole ? 2 * run + second : -1, seg.end - seg.last + seg.tiles - 1, tiles_each, tiles_more};
    }
    Pages pages_behind = look_up(behind, behind.first + way);
    Window window = look_ahead(seg, seg.first + way + WAYS), window_behind = look_ahead(seg, seg.first + way + 33 * WAYS);
    int window_at = 32;
    f32x4 o[RT][NH * E];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      m[rt] = -INFINITY, l[rt] = 0.0f;
#pragma unroll
      for (int i = 0; i < NH * E; ++i) o[rt][i] = f32x4{0, 0, 0, 0};
    }
    if (seg.first + way >= seg.last) {             // (nothing for this wave)
      here = place(behind, behind.first + way, pages_behind);
      load_k(here);
      __builtin_amdgcn_sched_barrier(0);
      load_v(here);
    }
    // Q is there from here on: a wait for it inside the loop would be one for all loads, in every round
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int t = 0; t < KS; ++t) asm volatile("" : "+v"(q[rt][t]));
    for (int tile = seg.first + way; tile < seg.last; tile += WAYS) {
      Place next;
      if (window_at == 32) {
        if (tile != seg.first + way) window = window_behind, window_behind = look_ahead(seg, tile + 33 * WAYS);
        work_out(seg, window), window_at = 0;
      }
      if (tile + WAYS < seg.last) next = place_at(window, window_at++);
      else next = place(behind, behind.first + way, pages_behind);
      f32x4 st[RT][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) st[rt][u] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KL; ++s) {
          if constexpr (FMT == FMT_MXFP4) {
            const float scale = __uint_as_float((uint32_t)k_scales[u][s] << 23);
#pragma unroll
            for (int e = 0; e < KE / 8; ++e) {
              const u32x4 w = widen8(k[u][s][e], scale);
#pragma unroll
              for (int rt = 0; rt < RT; ++rt)
                st[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(w), q[rt][KE / 8 * s + e], st[rt][u], 0, 0, 0);
            }
          } else if constexpr (FMT == FMT_MXFP8) {
            const float scale = __uint_as_float((uint32_t)k_scales[u][s] << 23);
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) widen4(k[u][s][e], scale, w[2 * e], w[2 * e + 1]);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
              st[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(u32x4{w[0], w[1], w[2], w[3]}), q[rt][2 * s], st[rt][u], 0, 0, 0);
              st[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(u32x4{w[4], w[5], w[6], w[7]}), q[rt][2 * s + 1], st[rt][u], 0, 0, 0);
            }
          } else {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
              st[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(u32x4{k[u][s][0], k[u][s][1], k[u][s][2], k[u][s][3]}), q[rt][s], st[rt][u], 0, 0, 0);
          }
        }
      }
      load_k(next);
      if constexpr (SOLO) __builtin_amdgcn_sched_barrier(0);       // (else some of them wait for V: 333 tokens 6.6 -> 7.0 us)
      // p as two bf16 parts, the first the next below p (its bits less one, cut off) and the second what is left, rounded: p to 2^-16, so the
      // output's own rounding is the only one to bf16 that shows.  Both are positive where p is, so that an infinite v stays infinite, and
      // both zero where p is: masked tokens, and weights that are nothing in 32 bits, however large their v.
      u32x4 pt[RT], pt_rest[RT];
      // (RULED) this lane's first token of the tile's, and whether every row sees all of those
      const int t0 = tile_at(seg, tile) * ATT_TILE + 4 * g;
      bool seen = true;
      if constexpr (RULED) {
        const int tile0 = tile_at(seg, tile) * ATT_TILE, last = seg.position + seg.fresh - 1;
        seen = tile0 + ATT_TILE <= seg.prefix || (tile0 + ATT_TILE - 1 <= seg.position && (!a.rule.window || last < a.rule.window || tile0 > last - a.rule.window));
      }
      auto sees = [&](int rt, int e) {              // whether this lane's column sees its token e
        const int t = t0 + 16 * (e / 4) + e % 4;
        return (t <= position[rt] && t >= low[rt]) || t < seg.prefix;
      };
      const bool masked = !seen || here.count[0] + here.count[1] < ATT_TILE;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float p[8];
        if (RULED && a.rule.cap_out > 0.0f) {
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = capped(st[rt][e / 4][e % 4], a.rule.cap_in, a.rule.cap_out);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = st[rt][e / 4][e % 4] * a.scale_log2;
        }
        if (RULED && a.rule.slopes) {
          const float from = (float)(position[rt] - t0);          // (both below 2^24, or their distance rounded, as it would be)
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] -= slope[rt] * fabsf(from - (float)(16 * (e / 4) + e % 4));
        }
        if (masked) {
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = 4 * g + e % 4 < here.count[e / 4] && (!RULED || seen || sees(rt, e)) ? p[e] : -INFINITY;
        }
        float top = p[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, p[e]);
        top = over_column(top, [](float x, float y) { return fmaxf(x, y); });
        // The weights' base moves where they would pass 2^ATT_SLACK, so that most tiles leave O alone; m is that base, which the joins know as the maximum.
        const bool moves = top > m[rt] + ATT_SLACK;
        if (__any(moves)) {
          const float m_new = moves ? top : m[rt], alpha = moves ? __builtin_amdgcn_exp2f(m[rt] - top) : 1.0f;
          m[rt] = m_new;
          l[rt] *= alpha;
#pragma unroll
          for (int i = 0; i < NH * E; ++i) o[rt][i] *= alpha;
        }
        // (nothing but masked tokens so far: everything below is 0)
        const float base = m[rt] == -INFINITY ? 0.0f : m[rt];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(p[e] - base);
          l[rt] += p[e];
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t lo = __builtin_elementwise_sub_sat(__float_as_uint(p[2 * c]), 1u), hi = __builtin_elementwise_sub_sat(__float_as_uint(p[2 * c + 1]), 1u);
          pt[rt][c] = __builtin_amdgcn_perm(hi, lo, 0x07060302);
          const bf16x2 rest = {(__bf16)(p[2 * c] - __uint_as_float(lo & 0xFFFF0000u)), (__bf16)(p[2 * c + 1] - __uint_as_float(hi & 0xFFFF0000u))};
          pt_rest[rt][c] = __builtin_bit_cast(uint32_t, rest);
        }
      }
      auto widen_v = [&](int h, uint32_t (&w)[8][E / 2]) {            // 8 tokens, E values each
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (FMT == FMT_MXFP4) {
            const float scale = __uint_as_float((uint32_t)v_scales[e / 4][h][e % 4] << 23);
            const u32x4 x = widen8(v[e / 4][h][e % 4][0], scale);
#pragma unroll
            for (int c = 0; c < E / 2; ++c) w[e][c] = x[c];
          } else if constexpr (FMT == FMT_MXFP8) {
            const float scale = __uint_as_float((uint32_t)v_scales[e / 4][h][e % 4] << 23);
#pragma unroll
            for (int c = 0; c < E / 4; ++c) widen4(v[e / 4][h][e % 4][c], scale, w[e][2 * c], w[e][2 * c + 1]);
          } else {
#pragma unroll
            for (int c = 0; c < E / 2; ++c) w[e][c] = v[e / 4][h][e % 4][c];
          }
        }
      };
      auto operand = [](const uint32_t (&w)[8][E / 2], int j) {
        u32x4 vt;
#pragma unroll
        for (int c = 0; c < 4; ++c)
          vt[c] = __builtin_amdgcn_perm(w[2 * c + 1][j / 2], w[2 * c][j / 2], j % 2 ? 0x07060302 : 0x05040100);
        return as_bf16(vt);
      };
      bool apart = false;                           // (RULED) a token that not every row sees has a value that is not finite
      if constexpr (RULED)
        if (!seen) {
          uint32_t bad = 0;
#pragma unroll
          for (int h = 0; h < NH; ++h) {
            uint32_t w[8][E / 2];
            widen_v(h, w);
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
              for (int c = 0; c < E / 2; ++c) bad |= not_finite(w[e][c]);
            __builtin_amdgcn_sched_barrier(0);
          }
          apart = __any(bad != 0);
        }
      if (RULED && apart) {
        // 0 times that is no 0: a row at a time, with nothing in the place of what it does not see
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int j = 0; j < E; ++j) {
              uint32_t w[8][E / 2];
              widen_v(h, w);
              const u32x4 there = __builtin_bit_cast(u32x4, operand(w, j));
#pragma nounroll
              for (int row = 0; row < ATT_ROWS; ++row) {
                const int row_position = __builtin_amdgcn_readlane(position[rt], row), row_low = __builtin_amdgcn_readlane(low[rt], row);
                const u32x4 nothing = {0, 0, 0, 0}, p_row = n == row ? pt[rt] : nothing, rest_row = n == row ? pt_rest[rt] : nothing;
                u32x4 vt = there;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  const int t = t0 + 16 * (e / 4) + e % 4;
                  if (!((t <= row_position && t >= row_low) || t < seg.prefix)) vt[e / 2] &= e % 2 ? 0x0000FFFFu : 0xFFFF0000u;
                }
                f32x4 x = {0, 0, 0, 0};
                x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(vt), as_bf16(p_row), x, 0, 0, 0);
                x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(vt), as_bf16(rest_row), x, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[rt][h * E + j][r] += n == row ? x[r] : 0.0f;
              }
              __builtin_amdgcn_sched_barrier(0);
            }
      } else {
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          uint32_t w[8][E / 2];
          widen_v(h, w);
#pragma unroll
          for (int j = 0; j < E; ++j) {
            const bf16x8 vt = operand(w, j);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
              o[rt][h * E + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, as_bf16(pt[rt]), o[rt][h * E + j], 0, 0, 0);
              o[rt][h * E + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, as_bf16(pt_rest[rt]), o[rt][h * E + j], 0, 0, 0);
            }
          }
        }
      }
      load_v(next);
      here = next;
    }
    const int rows = min(ROWS, rows_in(seg) - seg.rows_at * ROWS);
    uint16_t *const out = a.out + ((int64_t)seg.b * a.kv_heads * a.group + seg.kv_head * a.group + seg.rows_at * ROWS) * a.dim;
    auto out_row = [&](int row) { return RULED ? a.out + ruled_row(a, seg.q_at, seg.kv_head, seg.rows_at * ROWS + row) * a.dim : out + row * a.dim; };
    const int64_t part = ((int64_t)(run * 2 + second) * (ATT_WAVES / WAYS) + (WAYS == 1 ? wave : 0)) * ROWS;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      // The lanes of a column hold the sums of their own tokens.
      l[rt] = over_column(l[rt], [](float x, float y) { return x + y; });
      const int at = rt * ATT_ROWS;                 // the first row; lane (n, g), o[h E + j][r] = O[row at + n][16 E h + E (4 g + r) + j]
      if constexpr (WAYS == 1) {
        const float inverse = l[rt] != 0.0f ? 1.0f / l[rt] : 0.0f;
        if (at + n < rows && !whole && g == 0) a.part_ml[2 * (part + at + n)] = m[rt], a.part_ml[2 * (part + at + n) + 1] = l[rt];
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int i = 16 * E * h + E * (4 * g + r);
            if (at + n >= rows || i >= a.dim) continue;
#pragma unroll
            for (int j = 0; j < E; j += 4) {
              f32x4 x = {o[rt][h * E + j][r], o[rt][h * E + j + 1][r], o[rt][h * E + j + 2][r], o[rt][h * E + j + 3][r]};
              if (whole) {
                x *= inverse;
                *reinterpret_cast<bf16x4 *>(out_row(at + n) + i + j) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
              } else {
                *reinterpret_cast<f32x4 *>(a.part + (part + at + n) * a.dim + i + j) = x;
              }
            }
          }
      } else {
        // the waves' put together
        if (g == 0) m_all[wave][at + n] = m[rt], l_all[wave][at + n] = l[rt];
#pragma unroll
        for (int h = 0; h < NH; ++h) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < E; j += 4)
              o_all[wave][n][(E * (4 * g + r) + j) / 4] =
                  f32x4{o[rt][h * E + j][r], o[rt][h * E + j + 1][r], o[rt][h * E + j + 2][r], o[rt][h * E + j + 3][r]};
          __syncthreads();
          const int begin = 16 * E * h, quads = min(16 * E, a.dim - begin) / 4;
          for (int x = tid; x < min(rows - at, ATT_ROWS) * quads; x += 256) {
            const int r = x / quads, c = x - r * quads, row = at + r;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < WAYS; ++w) top = fmaxf(top, m_all[w][row]);
            const float base = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f;
            f32x4 value = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < WAYS; ++w) {
              const float f = __builtin_amdgcn_exp2f(m_all[w][row] - base);
              sum += f * l_all[w][row];
              value += f * o_all[w][r][c];
            }
            if (whole) {
              value *= sum != 0.0f ? 1.0f / sum : 0.0f;
              *reinterpret_cast<bf16x4 *>(out_row(row) + begin + 4 * c) = bf16x4{(__bf16)value[0], (__bf16)value[1], (__bf16)value[2], (__bf16)value[3]};
            } else {
              *reinterpret_cast<f32x4 *>(a.part + (part + row) * a.dim + begin + 4 * c) = value;
              if (begin + c == 0) a.part_ml[2 * (part + row)] = top, a.part_ml[2 * (part + row) + 1] = sum;
            }
          }
          if (rt + 1 < RT || h + 1 < NH || more) __syncthreads();
        }
      }
    }
    if (!more) break;
    seg = behind;
    load_q(seg);
  }
}

// What is not whole within a run, put together in the order of the tokens.  A thread takes four values of a query head and every
// so many-th of its parts, in one pass like the waves above; a workgroup's threads for the same values are put together in LDS.
// many: values, by fours, that a workgroup takes.
template <bool RULED>
__device__ __forceinline__ void attention_join_body(const AttentionArgs &a, int together, int many) {
  __shared__ f32x4 values[ATT_JOIN];
  __shared__ float m_all[ATT_JOIN], l_all[ATT_JOIN];
  const Cut cut = a.cuts[blockIdx.x];
  if (cut.place < 0) return;
  const int parts = Runs(cut.each, cut.more).of(cut.last_tile) - cut.place / 2 + 1;
  const int tid = threadIdx.x, quads = a.dim / 4, rows = min(a.rows, a.group);
  const int all = together * rows * quads, here = min(all, many), ways = blockDim.x / here, way = tid / here;
  const int x = blockIdx.y * many + (tid - way * here), c = x % quads, r = x / quads % rows, w = x / quads / rows;
  const int column = cut.column * together + w, kv_head = column / a.row_groups, row = (column - kv_head * a.row_groups) * a.rows + r;
  int rows_there = a.group, q_at = 0;
  if constexpr (RULED) {
    const int2 there = a.rule.starts ? rows_of_request(a, a.rule.starts[cut.b], a.rule.starts[cut.b + 1]) : make_int2(cut.b, cut.b + 1);
    q_at = there.x, rows_there = min(there.y - there.x, a.rule.most) * a.rule.heads_each;
  }
  const bool real = x < all && way < ways && row < rows_there && kv_head < a.kv_heads;
  float m = -INFINITY, l = 0.0f;
  f32x4 v = {0, 0, 0, 0};
  if (real) {
#pragma unroll 4
    for (int i = way; i < parts; i += ways) {
      const int64_t at = ((int64_t)(i ? (cut.place / 2 + i) * 2 : cut.place) * together + w) * a.rows + r;
      const float mi = a.part_ml[2 * at], li = a.part_ml[2 * at + 1];
      const f32x4 vi = *reinterpret_cast<const f32x4 *>(a.part + at * a.dim + 4 * c);
      const float top = fmaxf(m, mi), base = top == -INFINITY ? 0.0f : top;
      const float f = __builtin_amdgcn_exp2f(m - base), fi = __builtin_amdgcn_exp2f(mi - base);
      m = top;
      l = l * f + li * fi;
      v = v * f + vi * fi;
    }
  }
  m_all[tid] = m, l_all[tid] = l, values[tid] = v;
  __syncthreads();
  if (!real || way > 0) return;
  float top = m;
  for (int i = 1; i < ways; ++i) top = fmaxf(top, m_all[tid + i * here]);
  const float base = top == -INFINITY ? 0.0f : top, f = __builtin_amdgcn_exp2f(m - base);
  l *= f;
  v *= f;
  for (int i = 1; i < ways; ++i) {
    const float fi = __builtin_amdgcn_exp2f(m_all[tid + i * here] - base);
    l += l_all[tid + i * here] * fi;
    v += values[tid + i * here] * fi;
  }
  v *= l != 0.0f ? 1.0f / l : 0.0f;
  uint16_t *out = a.out + ((int64_t)(cut.b * a.kv_heads + kv_head) * a.group + row) * a.dim;
  if constexpr (RULED) out = a.out + ruled_row(a, q_at, kv_head, row) * a.dim;
  *reinterpret_cast<bf16x4 *>(out + 4 * c) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
}


// What a call's sizes and pointers are for the kernels, but for its workspace and the cut into workgroups (paged_attention.hip).
AttentionArgs attention_args(const torq_kv_cache_t &cache, const void *q, int64_t q_stride, int64_t q_head_stride, int heads,
                             const int32_t *block_tables, int64_t table_stride, int width, const int32_t *lengths, int64_t B, float scale,
                             void *out, const torq_scores_t *scores, const int32_t *starts, int most, int64_t tokens);

// How a call is cut into workgroups, and the kernels of the other files.
struct AttentionPlan {
  int ways, groups, rows;
  bool solo, by_item;
  int64_t items;
};
void go_attention4(const AttentionPlan &plan, const AttentionArgs &a, bool once, hipStream_t stream);
void go_scored_bf16(const AttentionPlan &plan, const AttentionArgs &a, bool once, hipStream_t stream);
void go_scored_mxfp8(const AttentionPlan &plan, const AttentionArgs &a, bool once, hipStream_t stream);
void go_scored_mxfp4(const AttentionPlan &plan, const AttentionArgs &a, bool once, hipStream_t stream);

}  // namespace torq
