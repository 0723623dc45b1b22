// torq_paged_attention: one new token of each request over its pages (and what torq_chunk_attention runs for few rows): its kernels for bf16 and
// MXFP8 caches without a rule, the joins, and who runs which.
//
// The mathematics, the layout and what was measured stand in paged_attention_body.h, whose kernels run MXFP4 and rules.  This one is apart from those and
// differs in two things: the weights' base is the maximum so far, so that it moves and O is multiplied with every tile, and a tile's pages are looked up by
// scalar instructions, a tile ahead.  It stays since the outputs that callers have of these formats stay so to the bit, and the other way would gain
// little where a tile is two or four times the bytes: this one / that one, us, 16 requests of 1000 to 8192 tokens 55.5 / 54.8, one of 131072 87.9 /
// 87.2, 77 with 20 heads of 80 86.3 / 86.2, 45 in MXFP8 313 / 306, one of 333 6.2 / 6.2.  A fault of one is to be looked for in the other.
#include <algorithm>
#include <cfloat>

#include "paged_attention_body.h"

namespace torq {

// DP: head_dim rounded up to what the operands hold.  WAYS: 4, the waves take turns at the tiles of a column; 1, each has a column
// of its own and all of its tiles in the run.  RT: products side by side, for up to 16 query heads each.  SOLO: a workgroup for each
// (request, columns that it works on), which is its run.
template <int DP, bool F8, bool ONCE, int WAYS, int RT, bool SOLO>
__global__ void __launch_bounds__(256) paged_attention_kernel(AttentionArgs a) {
  constexpr int KS = DP / 32;                       // k-steps of S
  constexpr int E = DP < 128 ? DP / 16 : 8;         // consecutive values of V in a lane
  constexpr int NH = DP / (16 * E);                 // such pieces of a row
  constexpr int BYTES = F8 ? 1 : 2, ROWS = ATT_ROWS * RT;
  constexpr int KL = DP * BYTES / 64;               // 16-byte loads of a lane for a group of 16 rows of K
  __shared__ f32x4 o_all[WAYS][ATT_ROWS][WAYS > 1 ? 4 * E + 1 : 1];       // a piece of O at a time
  __shared__ float m_all[WAYS][ROWS], l_all[WAYS][ROWS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
  // (key head, rows) of a request, as many at a time as the workgroup works on
  const int columns = (a.kv_heads * a.row_groups + ATT_WAVES / WAYS - 1) / (ATT_WAVES / WAYS), way = WAYS > 1 ? wave : 0;
  const uniform_ints lengths = (uniform_ints)(uintptr_t)a.lengths;

  // one (request, column), as far as it lies in the run: its tiles first ... last - 1 of `tiles`; end: the place behind them
  struct Segment {
    int b, column, tiles, length, kv_head, rows_at, first, last, end;
  };
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
  auto places_of = [](int tiles) { return tiles ? tiles + att_setup(WAYS) : 0; };
  // the one behind s, which the run goes on with
  auto behind_of = [&](Segment s) {
    int column = s.column + 1;
    if (column == columns) {
      do take_request(s, s.b + 1, length_of(a, lengths[s.b + 1]));
      while (s.tiles == 0);
      column = 0;
    }
    place_column(s, column);
    s.end += att_setup(WAYS);
    s.first = 0, s.last = min(run_end - s.end, s.tiles), s.end += s.last;
    return s;
  };
  // requests without tokens: zeros, and nothing to join
  auto zeros = [&] {
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
    const int length = length_of(a, lengths[b]), tiles = (length + ATT_TILE - 1) / ATT_TILE;
    seg = Segment{b, 0, tiles, length, 0, 0, 0, tiles, 0};      // (end: that of no run)
    place_column(seg, column);
  } else {
    // places of one column, request by request: every wave adds them up, a lane those of `per` requests (eight loads at a time)
    const int per = (a.B + 63) / 64;
    auto length_at = [&](int b) { return b < a.B ? length_of(a, a.lengths[b]) : 0; };
    int mine = 0, length = 0;
    if (per == 1) {
      length = length_at(lane);
      mine = places_of((length + ATT_TILE - 1) / ATT_TILE);
    } else {
      for (int i0 = 0; i0 < per; i0 += 8) {
        int read[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) read[i] = i0 + i < per ? length_at(lane * per + i0 + i) : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) mine += places_of((read[i] + ATT_TILE - 1) / ATT_TILE);
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
        mine = places_of((length + ATT_TILE - 1) / ATT_TILE);
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
    take_request(seg, b, __builtin_amdgcn_readlane(length, owner));
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
  const int k_at = n * a.token_bytes + 16 * g, v_at = 4 * g * a.token_bytes + E * n * BYTES;
  // Q^T as the B operand: column n, the i of this lane's K values
  bf16x8 q[RT][KS];
  auto load_q = [&](const Segment &s) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = s.rows_at * ROWS + rt * ATT_ROWS + n;       // query head of this lane's column within the group
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        const int i = F8 ? 64 * (t / 2) + 16 * g + 8 * (t % 2) : 32 * t + 8 * g;
        u32x4 v = {0, 0, 0, 0};
        if (row < a.group && i < a.dim)
          v = *reinterpret_cast<const u32x4 *>(a.q + s.b * a.q_stride + (int64_t)(s.kv_head * a.group + row) * a.q_head_stride + i);
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
      const int t16 = max(min(2 * tile + u, (s.length - 1) / 16), 0), entry = (int)((uint64_t)(uint32_t)t16 * (uint64_t)a.page16_magic >> 38);
      p.page[u] = s.length > 0 ? table[entry] : -1;
      p.in_page[u] = 16 * (t16 - entry * (a.page_size / 16));
    }
    return p;
  };
  struct Place {
    int count[2];
    int64_t at[2];
  };
  auto place = [&](const Segment &s, int tile, const Pages &p) {
    Place w;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int t = tile * ATT_TILE + 16 * u;
      // (a page that is none: as a number without a sign past all others)
      const int left = tile < s.last && (uint32_t)p.page[u] < (uint32_t)a.pages && s.rows_at < a.row_groups ? s.length - t : 0;
      w.count[u] = max(min(left, 16), 0);
      w.at[u] = (left > 0 ? p.page[u] : 0) * a.page_bytes + (s.kv_head * a.head_bytes + (int64_t)(p.in_page[u] * a.token_bytes));
    }
    return w;
  };
  auto rows_of = [&](const char *base, const Place &p, int u) {
    return records(base, p.at[u], p.count[u] ? (p.count[u] - 1) * a.token_bytes + a.dim * BYTES : 0);
  };
  auto scales_of = [&](const uint8_t *base, const Place &p, int u) {
    return records(base, p.at[u] / 32, p.count[u] ? (p.count[u] - 1) * (a.token_bytes / 32) + a.dim / 32 : 0);
  };
  u32x4 k[2][KL];
  uint32_t v[2][NH][4][E * BYTES / 4];
  uint8_t k_scales[2][KL], v_scales[2][NH][4];
  auto load_k = [&](const Place &p) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const __amdgpu_buffer_rsrc_t r = rows_of(a.k, p, u);
#pragma unroll
      for (int s = 0; s < KL; ++s)
        k[u][s] = buffer_load<16, ONCE>(r, (64 * s + 16 * g) < a.dim * BYTES ? k_at + 64 * s : ATT_FAR);
      if constexpr (F8) {
        const __amdgpu_buffer_rsrc_t rs = scales_of(a.k_scales, p, u);
#pragma unroll
        for (int s = 0; s < KL; ++s)
          k_scales[u][s] = __builtin_amdgcn_raw_buffer_load_b8(rs, 64 * s + 16 * g < a.dim ? (k_at + 64 * s) / 32 : ATT_FAR, 0, 0);
      }
    }
  };
  auto load_v = [&](const Place &p) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const __amdgpu_buffer_rsrc_t r = rows_of(a.v, p, u);
      __amdgpu_buffer_rsrc_t rs;
      if constexpr (F8) rs = scales_of(a.v_scales, p, u);
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int where = v_at + e * a.token_bytes + 16 * E * h * BYTES;
          const bool in = 16 * E * h + E * n < a.dim;
          const auto x = buffer_load<E * BYTES, ONCE>(r, in ? where : ATT_FAR);
          if constexpr (E * BYTES == 4) v[u][h][e][0] = x;
          else
#pragma unroll
            for (int c = 0; c < E * BYTES / 4; ++c) v[u][h][e][c] = x[c];
          if constexpr (F8) v_scales[u][h][e] = __builtin_amdgcn_raw_buffer_load_b8(rs, in ? where / 32 : ATT_FAR, 0, 0);
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
    pages = look_up(seg, seg.first + way + WAYS);
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
      if (tile + WAYS < seg.last) next = place(seg, tile + WAYS, pages);
      else next = place(behind, behind.first + way, pages_behind);
      pages = look_up(seg, tile + 2 * WAYS);
      f32x4 st[RT][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) st[rt][u] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KL; ++s) {
          if constexpr (F8) {
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
              st[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(k[u][s]), q[rt][s], st[rt][u], 0, 0, 0);
          }
        }
      }
      load_k(next);
      if constexpr (SOLO) __builtin_amdgcn_sched_barrier(0);       // (else some of them wait for V: 333 tokens 6.6 -> 7.0 us)
      // p as two bf16 parts, the first the next below p (its bits less one, cut off) and the second what is left, rounded: p to 2^-16, so the
      // output's own rounding is the only one to bf16 that shows.  Both are positive where p is, so that an infinite v stays infinite, and
      // both zero where p is: masked tokens, and weights that are nothing in 32 bits, however large their v.
      u32x4 pt[RT], pt_rest[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float m_new = m[rt], p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = 4 * g + e % 4 < here.count[e / 4] ? st[rt][e / 4][e % 4] * a.scale_log2 : -INFINITY;
          m_new = fmaxf(m_new, p[e]);
        }
        m_new = over_column(m_new, [](float x, float y) { return fmaxf(x, y); });
        // (nothing but masked tokens so far: everything below is 0)
        const float base = m_new == -INFINITY ? 0.0f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m[rt] - base);
        m[rt] = m_new;
        l[rt] *= alpha;
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
#pragma unroll
        for (int i = 0; i < NH * E; ++i) o[rt][i] *= alpha;
      }
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        uint32_t w[8][E / 2];                       // 8 tokens, E values each
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (F8) {
            const float scale = __uint_as_float((uint32_t)v_scales[e / 4][h][e % 4] << 23);
#pragma unroll
            for (int c = 0; c < E / 4; ++c) widen4(v[e / 4][h][e % 4][c], scale, w[e][2 * c], w[e][2 * c + 1]);
          } else {
#pragma unroll
            for (int c = 0; c < E / 2; ++c) w[e][c] = v[e / 4][h][e % 4][c];
          }
        }
#pragma unroll
        for (int j = 0; j < E; ++j) {
          u32x4 vt;
#pragma unroll
          for (int c = 0; c < 4; ++c)
            vt[c] = __builtin_amdgcn_perm(w[2 * c + 1][j / 2], w[2 * c][j / 2], j % 2 ? 0x07060302 : 0x05040100);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            o[rt][h * E + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(vt), as_bf16(pt[rt]), o[rt][h * E + j], 0, 0, 0);
            o[rt][h * E + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(vt), as_bf16(pt_rest[rt]), o[rt][h * E + j], 0, 0, 0);
          }
        }
      }
      load_v(next);
      here = next;
    }
    const int rows = min(ROWS, a.group - seg.rows_at * ROWS);
    uint16_t *const out = a.out + ((int64_t)seg.b * a.kv_heads * a.group + seg.kv_head * a.group + seg.rows_at * ROWS) * a.dim;
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
                *reinterpret_cast<bf16x4 *>(out + (at + n) * a.dim + i + j) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
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
              *reinterpret_cast<bf16x4 *>(out + row * a.dim + begin + 4 * c) = bf16x4{(__bf16)value[0], (__bf16)value[1], (__bf16)value[2], (__bf16)value[3]};
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

// The joins of parts, without a rule (those of every format) and with one.
__global__ void __launch_bounds__(ATT_JOIN) paged_attention_join_kernel(AttentionArgs a, int together, int many) {
  attention_join_body<false>(a, together, many);
}
__global__ void __launch_bounds__(ATT_JOIN) scored_attention_join_kernel(AttentionArgs a, int together, int many) {
  attention_join_body<true>(a, together, many);
}

namespace {
int bits_of(const torq_kv_cache_t &cache) { return cache.format == FMT_BF16 ? 16 : cache.format == FMT_MXFP8 ? 8 : 4; }
// Query heads of a column: 32 where there are more than 16, the registers hold two products side by side, and there are columns
// enough without the second 16.  24 heads for each of 8 key heads of 128, 1, 4, 16 requests of 1000 to 8192 tokens with 16 / 32:
// 12.3 / 13.1, 28.9 / 26.4, 79.8 / 65.6 us (32 heads 83.1 / 68.6, heads of 64 49.1 / 39.2, MXFP8 up to 32768 199 / 139); for one
// key head, 1 request of 60000, 64 of up to 8192: 23.2 / 26.3, 53.0 / 39.1; 333 tokens, 8 key heads, 1, 4, 16 requests 6.9 / 8.2, 7.6 / 8.2, 10.8 / 9.5.
int rows_of(const torq_kv_cache_t &cache, int heads, int64_t B) {
  return heads / cache.heads > ATT_ROWS && cache.head_dim <= 128 && B * cache.heads >= 32 ? 2 * ATT_ROWS : ATT_ROWS;
}
int row_groups_of(const torq_kv_cache_t &cache, int heads, int64_t B) {
  const int rows = rows_of(cache, heads, B);
  return (heads / cache.heads + rows - 1) / rows;
}
// Past the cache: rows of whole lines that one workgroup reads, and more of them than the cache holds, as far as the tables can tell.  Without /
// with the hint, from HBM and the same cache again, us: 67 MB 21.7 / 20.7, 19.5 / 19.6; 134 MB 33.9 / 30.9, 28.4 / 29.4; 268 MB 57.8 / 52.1,
// 47.8 / 50.8; 537 MB 104.7 / 94.2, 104.8 / 93.2; MXFP8 69 MB 23.9 / 23.5, 20.7 / 22.2, 277 MB 61.4 / 58.7, 52.0 / 57.9.  Rows that share lines
// lose: heads of 80 168 MB 40.1 / 42.7, of 96 in MXFP8, tokens outermost, 208 MB 70.8 / 83.6.
bool once_of(const torq_kv_cache_t &cache, int heads, int64_t B, int width) {
  if (row_groups_of(cache, heads, B) > 1) return false;
  const double pages = (double)std::min<int64_t>(cache.pages, B * (int64_t)width);
  const int row = cache.head_dim * bits_of(cache) / 8;
  return row % 128 == 0 && 2.0 * pages * cache.page_size * cache.heads * row > ONE_PASS_WEIGHT_BYTES;
}
AttentionPlan plan_of(const torq_kv_cache_t &cache, int heads, int64_t B, int width) {
  AttentionPlan p;
  p.rows = rows_of(cache, heads, B);
  const int64_t columns = (int64_t)cache.heads * row_groups_of(cache, heads, B), tiles = ((int64_t)width * cache.page_size + ATT_TILE - 1) / ATT_TILE;
  // Every request within so few tokens that a workgroup each is done before runs would be made out and joined.  In runs / a workgroup each, us: 333
  // tokens, 8 key heads, 1, 16, 64 requests 9.3 / 6.7, 13.9 / 8.0, 20.2 / 17.0; 900 to 1000 tokens, 1, 4, 16, 64, 256 of them 9.9 / 12.1, 13.5 / 13.3,
  // 20.5 / 14.3, 50.0 / 44.0, 175 / 165, ragged (1 to 1000) 9.9 / 9.1, 10.7 / 10.2, 17.5 / 13.4, 32.2 / 34.3, 101 / 100; up to 2000, ragged, 16, 64 of
  // them 23.3 / 25.2, 53.7 / 65.7
  // (and within a launch, which runs always are)
  p.solo = (tiles <= 16 || (tiles <= 32 && B * columns >= 128)) && B * columns <= most_workgroups(256);
  bool own;                                         // each wave has a column of its own
  const bool alone = cache.head_dim > 128, mx = cache.format != FMT_BF16;
  const int64_t idle = -columns & (ATT_WAVES - 1), workgroups = B * (columns + idle) / ATT_WAVES;
  auto busy = [&](int eighths) { return 8 * columns >= eighths * (columns + idle); };
  if (p.solo) {
    // It saves the putting together, where there are columns for the waves of all CUs (a workgroup's are of one request, so that some have
    // none where its columns are no multiple of four) and few tiles of each; over 128, where a CU has one workgroup at a time, also of more,
    // if their rounds of the CUs are whole.  All four / one each, us:
    //   columns  tokens       head_dim  key heads  bf16         MXFP8
    //   512      20 to 128    128       8          7.6 / 8.8    7.1 / 8.2
    //   1024     20 to 128    128       8          11.3 / 10.3  10.7 / 8.7
    //   1024     20 to 128    128       7          11.5 / 14.5  11.6 / 12.0
    //   4096     20 to 128    128       7                       31.8 / 24.1
    //   4096     60 to 160    128       8          49.0 / 47.9
    //   4096     60 to 192    128       8          53.5 / 55.3
    //   4096     60 to 256    128       8          62.9 / 68.4  49.2 / 45.1
    //   4096     60 to 192    64        8          31.6 / 30.4
    //   8192     60 to 256    64        8          68.5 / 66.1
    //   512      100 to 128   256       8          17.0 / 14.9  11.6 / 12.3
    //   512      130 to 256   256       8          24.7 / 32.9  15.3 / 18.9
    //   1024     100 to 128   256       8          32.6 / 22.9  19.2 / 14.3
    //   1024     130 to 256   256       8          47.1 / 40.9  30.9 / 25.7
    //   2048     60 to 160    256       3          66.0 / 52.9  43.3 / 40.2
    //   2048     60 to 160    256       2          65.0 / 56.1  43.2 / 45.0
    //   2048     60 to 160    256       1          66.0 / 81.5  42.8 / 69.1
    //   2048     60 to 256    256       3          84.1 / 74.9  52.0 / 54.1
    //   1024     1 to 320     256       8          47.3 / 44.2  26.8 / 23.3
    //   1024     1 to 512     256       8          61.7 / 67.4  41.5 / 42.0
    //   1024     460 to 512   256       8          91.6 / 83.5  53.2 / 48.0
    //   1280     160 to 320   256       8          66.8 / 73.7  41.9 / 51.0
    //   2048     300 to 1000  256       8          246 / 260
    //   2048     900 to 1000  256       8          337 / 320
    const int64_t rounds = (workgroups + 255) / 256;
    own = alone ? (tiles <= 6 ? workgroups >= 128 && busy(mx ? 6 : 4) : tiles <= 16 && busy(7) && 8 * workgroups >= 7 * 256 * rounds)
                : tiles <= (mx || cache.head_dim <= 64 ? 8 : 5) && (mx ? busy(6) : idle == 0) && B * columns >= (tiles <= 4 ? 768 : 2048);
  } else if (row_groups_of(cache, heads, B) > 1) {
    // Two columns of 16, 8 key heads, 1, 4, 16 requests: 12.5 / 15.7, 33.8 / 28.9, 102 / 80 us.  In MXFP8, where it is the vector instructions that
    // idle waves leave to others: 64 and 128 requests of 1000 to 4000, 24 query heads of 256 for one key head 39 / 49, 66 / 93, 40 of 128 31 / 39,
    // 44 / 62, for three 59 / 70, 87 / 121; of 256 for three 88 / 105, but from 128 requests on 184 / 174
    own = !mx || busy(7) ? B * columns >= 64 : alone && columns > 2 && B * columns >= ATT_WAYS_ITEMS;
  } else {
    own = idle == 0 && (alone || heads / cache.heads <= 2) && B * columns >= ATT_WAYS_ITEMS;
  }
  p.ways = own ? 1 : ATT_WAVES;
  // workgroups: three, two or one for each CU by the registers that a wave takes.  head_dim 64 with 512, 768, 1024: 64 requests of 100 to
  // 3000 tokens 52.3, 50.1, 49.6 us, 16 long ones 34.6, 35.4, 35.8; 128: 16 58.3, 59.4, 64.6; 256 with 256, 512, 768: 64.9, 72.6, 79.9
  const int64_t full = cache.head_dim <= 64 ? 768 : cache.head_dim <= 128 ? 512 : 256;
  p.items = B * ((columns + ATT_WAVES / p.ways - 1) / (ATT_WAVES / p.ways));
  const int64_t groups = (p.items * (tiles + att_setup(p.ways)) + p.ways - 1) / p.ways;      // by the longest that the tables hold
  p.groups = p.solo ? (int)p.items : (int)(groups < 1 ? 1 : groups < full ? groups : full);
  p.by_item = p.items < p.groups;
  return p;
}
size_t cuts_bytes(const AttentionPlan &p) { return (p.by_item ? (size_t)p.items : (size_t)p.groups) * sizeof(Cut); }
size_t part_rows(const AttentionPlan &p) { return (size_t)p.groups * 2 * (ATT_WAVES / p.ways) * p.rows; }
}  // namespace

size_t paged_attention_workspace_bytes(const torq_kv_cache_t &cache, int heads, int64_t B, int width) {
  const AttentionPlan p = plan_of(cache, heads, B, width);
  return p.solo ? 0 : cuts_bytes(p) + part_rows(p) * (cache.head_dim + 2) * sizeof(float);
}

AttentionArgs attention_args(const torq_kv_cache_t &cache, const void *q, int64_t q_stride, int64_t q_head_stride, int heads,
                             const int32_t *block_tables, int64_t table_stride, int width, const int32_t *lengths, int64_t B, float scale,
                             void *out, const torq_scores_t *scores, const int32_t *starts, int most, int64_t tokens) {
  if (cache.pages == 0) width = 0;                  // no token has a page: nothing of the cache is touched
  const int bits = bits_of(cache), each = heads / cache.heads;
  const torq_scores_t plain = {}, &rule = scores ? *scores : plain;
  const float log2e = 1.44269504088896340736f;
  AttentionArgs a{};
  a.k = (const char *)cache.k, a.v = (const char *)cache.v, a.k_scales = cache.k_scales, a.v_scales = cache.v_scales;
  a.page_bytes = cache.page_stride * bits / 8, a.head_bytes = cache.head_stride * bits / 8, a.token_bytes = (int)(cache.token_stride * bits / 8);
  a.pages = (int)cache.pages, a.page_size = cache.page_size, a.page16_magic = ((int64_t)1 << 38) / (cache.page_size / 16) + 1;
  a.q = (const uint16_t *)q, a.q_stride = q_stride, a.q_head_stride = q_head_stride, a.out = (uint16_t *)out;
  a.tables = block_tables, a.lengths = lengths, a.table_stride = table_stride, a.most = (int64_t)width * cache.page_size;
  a.B = (int)B, a.kv_heads = cache.heads, a.group = (int)std::min<int64_t>((int64_t)each * most, 0x7FFFFFFF), a.dim = cache.head_dim, a.scale_log2 = scale * log2e;
  a.rule = ScoreArgs{0.0f, 0.0f, rule.slopes, rule.prefix, starts, rule.window, most, each, tokens};
  if (rule.cap > 0.0f) a.rule.cap_in = std::max(-FLT_MAX, std::min(FLT_MAX, scale / rule.cap)), a.rule.cap_out = rule.cap * log2e;
  return a;
}

hipError_t launch_paged_attention(const torq_kv_cache_t &cache, const void *q, int64_t q_stride, int64_t q_head_stride, int heads,
                                  const int32_t *block_tables, int64_t table_stride, int width, const int32_t *lengths,
                                  int64_t B, float scale, void *out, void *workspace, const torq_scores_t *scores,
                                  const int32_t *starts, int most, int64_t tokens, hipStream_t stream) {
  const int rows = heads * most;                    // a request's new tokens' heads
  const AttentionPlan plan = plan_of(cache, rows, B, width);
  const bool f8 = cache.format == FMT_MXFP8, once = once_of(cache, rows, B, width);
  AttentionArgs a = attention_args(cache, q, q_stride, q_head_stride, heads, block_tables, table_stride, width, lengths, B, scale, out, scores, starts,
                                   most, tokens);
  a.rows = plan.rows, a.row_groups = row_groups_of(cache, rows, B);
  a.cuts = (Cut *)workspace, a.by_item = plan.by_item;
  a.part = (float *)((uintptr_t)workspace + cuts_bytes(plan)), a.part_ml = a.part + part_rows(plan) * cache.head_dim;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(plan.groups), dim3(256), 0, stream, a); };
  auto of_hint = [&](auto dp, auto of8, auto hint) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool F8 = decltype(of8)::value, ONCE = decltype(hint)::value;
    auto of_launch = [&](auto solo) {
      constexpr bool SOLO = decltype(solo)::value;
      if constexpr (DP <= 128)
        if (plan.rows > ATT_ROWS) {
          // (a column for each wave: short tables, or lines that are read more than once)
          if (plan.ways == 1) return go(paged_attention_kernel<DP, F8, false, 1, 2, SOLO>);
          return go(paged_attention_kernel<DP, F8, ONCE, ATT_WAVES, 2, SOLO>);
        }
      plan.ways > 1 ? go(paged_attention_kernel<DP, F8, ONCE, ATT_WAVES, 1, SOLO>) : go(paged_attention_kernel<DP, F8, ONCE, 1, 1, SOLO>);
    };
    plan.solo ? of_launch(std::true_type{}) : of_launch(std::false_type{});
  };
  auto of_format = [&](auto dp, auto of8) {
    // (rows of up to 64 bytes never go past the cache)
    if constexpr (!(decltype(of8)::value && decltype(dp)::value == 64))
      if (once) return of_hint(dp, of8, std::true_type{});
    of_hint(dp, of8, std::false_type{});
  };
  auto of_dim = [&](auto dp) { f8 ? of_format(dp, std::true_type{}) : of_format(dp, std::false_type{}); };
  // (a rule that says nothing is none)
  const bool ruled = starts || (scores && (scores->cap > 0.0f || scores->slopes || scores->window || scores->prefix));
  if (ruled) (cache.format == FMT_BF16 ? go_scored_bf16 : f8 ? go_scored_mxfp8 : go_scored_mxfp4)(plan, a, once, stream);
  else if (cache.format == FMT_MXFP4) go_attention4(plan, a, once, stream);
  else if (cache.head_dim <= 64) of_dim(std::integral_constant<int, 64>{});
  else if (cache.head_dim <= 128) of_dim(std::integral_constant<int, 128>{});
  else of_dim(std::integral_constant<int, 256>{});
  if (!plan.solo) {
    // fewer (request, key head)s than runs: many parts each, over more threads; else two or three, one for most runs
    const int together = ATT_WAVES / plan.ways, values = together * std::min(a.rows, a.group) * (a.dim / 4);
    const int threads = plan.by_item ? ATT_JOIN : 256, many = plan.by_item ? 64 : 256;
    hipLaunchKernelGGL(ruled ? scored_attention_join_kernel : paged_attention_join_kernel, dim3(plan.by_item ? (unsigned)plan.items : (unsigned)plan.groups, (values + many - 1) / many),
                       dim3(threads), 0, stream, a, together, many);
  }
  return hipGetLastError();
}

}  // namespace torq
