// torq_paged_attention: one new token of each request over its pages, out = softmax(scale q K^T) V for each head.
//
// The query heads of a key head are the columns of one matrix product, up to 16 at a time, so K and V are read once for all of
// them: HBM-bound, 2 (bf16) or 1 1/32 (MXFP8) bytes for 2 heads / kv_heads flops.
//
// Work: the tokens of every (request, key head) in tiles of 32, all of them in one row of tiles, cut into equal runs, one for each
// workgroup: lengths may be as ragged as they like, and the host need not know them (every workgroup adds them up itself).  A run goes through one or
// several (request, key head)s.  The four waves of a workgroup take turns at the tiles, each with a softmax of its own in one pass (running
// maximum m, sum l, unnormalised O), put together in LDS at the end of a (request, key head).  What lies whole within a run is written as output, the
// others' O, m and l go to the workspace, two at most for a run, and a second kernel joins them in the order of the tokens.
//
// A tile goes through the matrix cores transposed, and nothing of it passes between lanes but the column maxima:
//   S^T [token][head] = K [token][i] Q^T [i][head]           v_mfma_f32_16x16x32_bf16, two groups of 16 tokens
//   lane (n = l % 16, g = l / 16) then holds head n's S for tokens 4g + r of both groups, r < 4
//   O^T [i][head] += V^T [i][token] P^T [token][head]        the k index of this product runs over the 32 tokens in the order in
//                                                            which the lanes hold them, so P^T is already its B operand
// Its A operand wants 8 tokens of one i in a lane.  The lane loads, for its 8 tokens, E consecutive values of V (coalesced
// rows), and pairs of them are put together by v_perm_b32: slot j holds V[its tokens][E * (l % 16) + j].
// In MXFP8 the elements are widened to bf16 with their scale in one instruction (exact: 4 bits of significand).
//
// K and V of a wave's next tile are on their way while it works on this one, K from the moment that S is there, V from the
// moment that O is.  The loads are buffer loads over the 16 tokens of a group (a group lies in one page) as far as they are tokens of
// the request: what is past the length, in no page or past the last tile has no records, costs no traffic and comes back as
// zeros, so the loop knows no other case (and a NaN behind the length is not read).
#include "torq_device.h"
#include "torq_internal.h"

namespace torq {

constexpr int ATT_TILE = 32;          // tokens of a wave's step
constexpr int ATT_WAVES = 4;
constexpr int ATT_ROWS = 16;          // query heads of a workgroup
constexpr int ATT_GROUPS = 768;       // workgroups, three for each CU
constexpr int ATT_FAR = 0x7FFFFF00;   // an offset past every buffer

struct AttentionArgs {
  const char *k, *v;
  const uint8_t *k_scales, *v_scales;
  int64_t pages, page_stride, head_stride;
  int token_bytes;                    // from a token to the next
  const uint16_t *q;
  int64_t q_stride, q_head_stride;
  const int *tables, *lengths;
  int64_t table_stride, page16_magic; // t / page_size = (t / 16) * page16_magic >> 38
  int64_t most;                       // width * page_size
  int B, page_size, kv_heads, group, row_groups, dim;
  float scale_log2;                   // scale * log2(e): the softmax is taken to base 2
  uint16_t *out;
  float *part, *part_ml;              // [run][2][16][dim] and [run][2][16][2]: O, and m and l, of a (request, key head) not whole in a run
  int *before;                        // [B + 1]: tiles of one key head ahead of each request
};

// The runs: `tiles` tiles over `runs` workgroups, the first `more` of which have one more than the others.
struct Runs {
  int each, more, runs;
  __device__ Runs(int tiles, int groups) {
    runs = max(1, min(groups, (tiles + ATT_WAVES - 1) / ATT_WAVES));
    each = tiles / runs, more = tiles - each * runs;
  }
  __device__ int begin(int run) const { return run * each + min(run, more); }
  __device__ int of(int tile) const {
    const int wide = more * (each + 1);
    return tile < wide ? tile / (each + 1) : more + (tile - wide) / each;
  }
};

__device__ __forceinline__ bf16x8 as_bf16(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }
// four E4M3 bytes -> two words of two bf16, times scale
__device__ __forceinline__ void widen4(uint32_t v, float scale, uint32_t &a, uint32_t &b) {
  a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, false));
  b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, true));
}
typedef const __attribute__((address_space(4))) int *uniform_ints;      // read by scalar loads
typedef __attribute__((__vector_size__(2 * sizeof(unsigned)))) unsigned u32x2;

// `bytes` bytes from p as a raw buffer; all three the same in every lane
__device__ __forceinline__ __amdgpu_buffer_rsrc_t records(const void *base, int64_t at, int bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base) + at;
  const uint64_t u = (uint32_t)__builtin_amdgcn_readfirstlane((int)p) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(p >> 32)) << 32;
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(u), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
template <int N>
__device__ __forceinline__ auto buffer_load(__amdgpu_buffer_rsrc_t r, int at) {
  if constexpr (N == 16) return __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0);
  else if constexpr (N == 8) return __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, 0);
  else return __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
}

__device__ __forceinline__ int tiles_of(const AttentionArgs &a, int b) {
  const int64_t n = a.lengths[b];
  return (int)(((n < 0 ? 0 : n < a.most ? n : a.most) + ATT_TILE - 1) / ATT_TILE);
}

// DP: head_dim rounded up to what the operands hold.
template <int DP, bool F8>
__global__ void __launch_bounds__(256) paged_attention_kernel(AttentionArgs a) {
  constexpr int KS = DP / 32;                       // k-steps of S
  constexpr int E = DP < 128 ? DP / 16 : 8;         // consecutive values of V in a lane
  constexpr int NH = DP / (16 * E);                 // such pieces of a row
  constexpr int BYTES = F8 ? 1 : 2;
  constexpr int KL = DP * BYTES / 64;               // 16-byte loads of a lane for a group of 16 rows of K
  __shared__ float o_all[ATT_WAVES][ATT_ROWS][16 * E + 4];      // a piece of O at a time
  __shared__ float m_all[ATT_WAVES][ATT_ROWS], l_all[ATT_WAVES][ATT_ROWS];
  __shared__ int wave_tiles[ATT_WAVES], found_b, found_before;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
  const int columns = a.kv_heads * a.row_groups;    // (key head, rows) of a request

  // tiles of one column, request by request: a thread adds up `per` of them
  const int per = (a.B + 255) / 256;
  int mine = 0;
  for (int i = 0; i < per; ++i)
    if (tid * per + i < a.B) mine += tiles_of(a, tid * per + i);
  int sum = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(sum, o);
    if (lane >= o) sum += up;
  }
  if (lane == 63) wave_tiles[wave] = sum;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < ATT_WAVES; ++w) {
    if (w < wave) sum += wave_tiles[w];
    total += wave_tiles[w];
  }
  total = __builtin_amdgcn_readfirstlane(total);
  if (blockIdx.x == 0) {                            // (for the join)
    int at = sum - mine;
    for (int i = 0; i < per; ++i)
      if (tid * per + i < a.B) {
        a.before[tid * per + i] = at;
        at += tiles_of(a, tid * per + i);
      }
    if (tid == 0) a.before[a.B] = total;
  }
  const Runs runs(total * columns, gridDim.x);
  if ((int)blockIdx.x >= runs.runs) return;
  const int run_begin = runs.begin(blockIdx.x), run_end = runs.begin(blockIdx.x + 1);
  if (run_begin == run_end) return;                 // (nothing at all)
  // the request in which the run begins
  if ((sum - mine) * columns <= run_begin && run_begin < sum * columns) {
    int at = sum - mine, b = tid * per;
    for (int t; (at + (t = tiles_of(a, b))) * columns <= run_begin; ++b) at += t;
    found_b = b, found_before = at;
  }
  __syncthreads();
  int b = __builtin_amdgcn_readfirstlane(found_b), before = __builtin_amdgcn_readfirstlane(found_before);
  const uniform_ints lengths = (uniform_ints)(uintptr_t)a.lengths;

  // what a lane reads of a group of 16 tokens, in bytes from its first token
  const int k_at = n * a.token_bytes + 16 * g, v_at = 4 * g * a.token_bytes + E * n * BYTES;

  for (int at = run_begin; at < run_end;) {
    // one (request, key head, rows), as far as it lies in the run
    int length = lengths[b];
    length = length < 0 ? 0 : length < a.most ? length : (int)a.most;
    const int tiles = (length + ATT_TILE - 1) / ATT_TILE;
    if (at >= (before + tiles) * columns) {
      before += tiles;
      ++b;
      continue;
    }
    const int column = (at - before * columns) / tiles, rows_at = column % a.row_groups, kv_head = column / a.row_groups;
    const int column_begin = before * columns + column * tiles;
    const int first = at - column_begin, last = min(run_end - column_begin, tiles);     // tiles of it
    const uniform_ints table = (uniform_ints)(uintptr_t)(a.tables + b * a.table_stride);
    const int row = rows_at * ATT_ROWS + n;         // query head of this lane's column within the group
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
    // the pages of a tile's two groups of 16 tokens; how many of a group are tokens; where they lie, in bytes
    auto look_up = [&](int tile, int (&page)[2]) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int t16 = min(2 * tile + u, (length - 1) / 16);
        page[u] = table[(int)((uint64_t)t16 * (uint64_t)a.page16_magic >> 38)];
      }
    };
    struct Place {
      int count[2];
      int64_t at[2];
    };
    auto place = [&](int tile, const int (&page)[2]) {
      Place p;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int t = tile * ATT_TILE + 16 * u, t16 = 2 * tile + u;
        const int in_page = (t16 - (int)((uint64_t)t16 * (uint64_t)a.page16_magic >> 38) * (a.page_size / 16)) * 16;
        const bool there = tile < last && t < length && page[u] >= 0 && page[u] < a.pages;
        p.count[u] = there ? min(length - t, 16) : 0;
        p.at[u] = ((there ? page[u] : 0) * a.page_stride + kv_head * a.head_stride) * BYTES + (int64_t)in_page * a.token_bytes;
      }
      return p;
    };
    auto rows_of = [&](const char *base, const Place &p, int u) {
      const int bytes = p.count[u] ? (p.count[u] - 1) * a.token_bytes + a.dim * BYTES : 0;
      return records(base, p.at[u], bytes);
    };
    u32x4 k[2][KL];
    uint32_t v[2][NH][4][E * BYTES / 4];
    uint32_t k_scales[2][KL], v_scales[2][NH][4];
    auto load_k = [&](const Place &p) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const __amdgpu_buffer_rsrc_t r = rows_of(a.k, p, u);
#pragma unroll
        for (int s = 0; s < KL; ++s)
          k[u][s] = buffer_load<16>(r, (64 * s + 16 * g) < a.dim * BYTES ? k_at + 64 * s : ATT_FAR);
        if constexpr (F8) {
          const int bytes = p.count[u] ? (p.count[u] - 1) * (a.token_bytes / 32) + a.dim / 32 : 0;
          const __amdgpu_buffer_rsrc_t rs = records(a.k_scales, p.at[u] / 32, bytes);
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
        if constexpr (F8) {
          const int bytes = p.count[u] ? (p.count[u] - 1) * (a.token_bytes / 32) + a.dim / 32 : 0;
          rs = records(a.v_scales, p.at[u] / 32, bytes);
        }
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int where = v_at + e * a.token_bytes + 16 * E * h * BYTES;
            const bool in = 16 * E * h + E * n < a.dim;
            const auto x = buffer_load<E * BYTES>(r, in ? where : ATT_FAR);
            if constexpr (E * BYTES == 4) v[u][h][e][0] = x;
            else
#pragma unroll
              for (int c = 0; c < E * BYTES / 4; ++c) v[u][h][e][c] = x[c];
            if constexpr (F8) v_scales[u][h][e] = __builtin_amdgcn_raw_buffer_load_b8(rs, in ? where / 32 : ATT_FAR, 0, 0);
          }
      }
    };
    f32x4 o[NH * E];
#pragma unroll
    for (int i = 0; i < NH * E; ++i) o[i] = f32x4{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;

    int page[2];
    look_up(first + wave, page);
    Place here = place(first + wave, page);
    load_k(here);
    __builtin_amdgcn_sched_barrier(0);              // (in the order of the loop's own, whose waits count them)
    load_v(here);
    look_up(first + wave + ATT_WAVES, page);
    for (int tile = first + wave; tile < last; tile += ATT_WAVES) {
      const Place next = place(tile + ATT_WAVES, page);
      look_up(tile + 2 * ATT_WAVES, page);
      f32x4 st[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        st[u] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KL; ++s) {
          if constexpr (F8) {
            const float scale = __uint_as_float(k_scales[u][s] << 23);
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) widen4(k[u][s][e], scale, w[2 * e], w[2 * e + 1]);
            st[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(u32x4{w[0], w[1], w[2], w[3]}), q[2 * s], st[u], 0, 0, 0);
            st[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(u32x4{w[4], w[5], w[6], w[7]}), q[2 * s + 1], st[u], 0, 0, 0);
          } else {
            st[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(k[u][s]), q[s], st[u], 0, 0, 0);
          }
        }
      }
      load_k(next);
      float m_new = m, p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = 4 * g + e % 4 < here.count[e / 4] ? st[e / 4][e % 4] * a.scale_log2 : -INFINITY;
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
        uint32_t w[8][E / 2];                       // 8 tokens, E values each
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (F8) {
            const float scale = __uint_as_float(v_scales[e / 4][h][e % 4] << 23);
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
          o[h * E + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(vt), as_bf16(pt), o[h * E + j], 0, 0, 0);
          o[h * E + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(vt), as_bf16(pt_rest), o[h * E + j], 0, 0, 0);
        }
      }
      load_v(next);
      here = next;
    }
    // the lanes of a column hold the sums of their own tokens
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) m_all[wave][n] = m, l_all[wave][n] = l;
    const int rows = min(ATT_ROWS, a.group - rows_at * ATT_ROWS);
    const bool whole = first == 0 && last == tiles;
    uint16_t *const out = a.out + ((int64_t)b * a.kv_heads * a.group + kv_head * a.group + rows_at * ATT_ROWS) * a.dim;
    // where the run begins within a column: its first place in the workspace, else its second
    const int64_t part = ((int64_t)blockIdx.x * 2 + (at == run_begin ? 0 : 1)) * ATT_ROWS;
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      // lane (n, g), o[h E + j][r] = O[head n][16 E h + E (4 g + r) + j]
#pragma unroll
      for (int j = 0; j < E; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) o_all[wave][n][E * (4 * g + r) + j] = o[h * E + j][r];
      __syncthreads();
      const int begin = 16 * E * h, count = min(16 * E, a.dim - begin);
      for (int x = tid; x < rows * count; x += 256) {
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
        if (whole) {
          const __bf16 y = (__bf16)(sum != 0.0f ? value / sum : 0.0f);
          out[r * a.dim + begin + i] = __builtin_bit_cast(uint16_t, y);
        } else {
          a.part[(part + r) * a.dim + begin + i] = value;
          if (begin + i == 0) a.part_ml[2 * (part + r)] = top, a.part_ml[2 * (part + r) + 1] = sum;
        }
      }
      __syncthreads();
    }
    at = column_begin + last;
  }
}

// What is not whole within a run, put together in the order of the runs; zeros for a request without tokens.  A workgroup for each (request,
// query head): its lanes take four values each of the parts of every few runs, which are put together in LDS.
__global__ void __launch_bounds__(256) paged_attention_join_kernel(AttentionArgs a, int groups) {
  __shared__ float factor[ATT_GROUPS], reduced[256 / 64];
  __shared__ f32x4 values[256];
  const int tid = threadIdx.x, heads = a.kv_heads * a.group, columns = a.kv_heads * a.row_groups;
  const int b = blockIdx.x / heads, head = blockIdx.x - b * heads, kv_head = head / a.group, r = head % a.group % ATT_ROWS;
  const int column = kv_head * a.row_groups + head % a.group / ATT_ROWS;
  const int before = a.before[b], tiles = a.before[b + 1] - before;
  uint16_t *const out = a.out + (int64_t)blockIdx.x * a.dim;
  if (tiles == 0) {
    if (tid < a.dim) out[tid] = 0;
    return;
  }
  const Runs runs(a.before[a.B] * columns, groups);
  const int begin = before * columns + column * tiles, run0 = runs.of(begin), count = runs.of(begin + tiles - 1) - run0 + 1;
  if (count == 1) return;
  // the first part is its run's second place unless the run begins with it
  const int first = runs.begin(run0) == begin ? 2 * run0 : 2 * run0 + 1;
  auto place = [&](int i) { return (int64_t)(i ? 2 * (run0 + i) : first) * ATT_ROWS + r; };
  auto over_group = [&](float v, auto op) {         // of all threads, in a fixed order
#pragma unroll
    for (int o = 32; o; o >>= 1) v = op(v, __shfl_xor(v, o));
    __syncthreads();
    if ((tid & 63) == 0) reduced[tid >> 6] = v;
    __syncthreads();
    return op(op(reduced[0], reduced[1]), op(reduced[2], reduced[3]));
  };
  float m[ATT_GROUPS / 256], top = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < ATT_GROUPS / 256; ++i) {
    m[i] = tid + 256 * i < count ? a.part_ml[2 * place(tid + 256 * i)] : -INFINITY;
    top = fmaxf(top, m[i]);
  }
  top = over_group(top, [](float x, float y) { return fmaxf(x, y); });
  const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
  for (int i = 0; i < ATT_GROUPS / 256; ++i)
    if (tid + 256 * i < count) {
      const float f = __builtin_amdgcn_exp2f(m[i] - base);
      factor[tid + 256 * i] = f;
      sum += f * a.part_ml[2 * place(tid + 256 * i) + 1];
    }
  sum = over_group(sum, [](float x, float y) { return x + y; });
  // lanes: values 4 c ... 4 c + 3 of every `apart`-th part
  const int quads = a.dim / 4, apart = 256 / quads, c = tid % quads, from = tid / quads;
  f32x4 v = {0, 0, 0, 0};
  if (from < apart)
#pragma unroll 4
    for (int i = from; i < count; i += apart)
      v += factor[i] * *reinterpret_cast<const f32x4 *>(a.part + place(i) * a.dim + 4 * c);
  values[tid] = v;
  __syncthreads();
  if (tid < quads) {
    for (int i = 1; i < apart; ++i) v += values[tid + i * quads];
    bf16x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (__bf16)(sum != 0.0f ? v[e] / sum : 0.0f);
    *reinterpret_cast<bf16x4 *>(out + 4 * tid) = y;
  }
}

namespace {
int row_groups_of(const torq_kv_cache_t &cache, int heads) { return (heads / cache.heads + ATT_ROWS - 1) / ATT_ROWS; }
// Workgroups: a tile at least for each wave, by the longest that the tables hold
int groups_of(const torq_kv_cache_t &cache, int heads, int64_t B, int width) {
  const int64_t most = (int64_t)width * cache.page_size;
  const int64_t tiles = B * cache.heads * row_groups_of(cache, heads) * ((most + ATT_TILE - 1) / ATT_TILE);
  const int64_t groups = (tiles + ATT_WAVES - 1) / ATT_WAVES;
  return (int)(groups < 1 ? 1 : groups < ATT_GROUPS ? groups : ATT_GROUPS);
}
size_t before_bytes(int64_t B) { return ((size_t)(B + 1) * sizeof(int) + 255) & ~(size_t)255; }
}  // namespace

size_t paged_attention_workspace_bytes(const torq_kv_cache_t &cache, int heads, int64_t B, int width) {
  return before_bytes(B) + (size_t)groups_of(cache, heads, B, width) * 2 * ATT_ROWS * (cache.head_dim + 2) * sizeof(float);
}

hipError_t launch_paged_attention(const torq_kv_cache_t &cache, const void *q, int64_t q_stride, int64_t q_head_stride, int heads,
                                  const int32_t *block_tables, int64_t table_stride, int width, const int32_t *lengths,
                                  int64_t B, float scale, void *out, void *workspace, hipStream_t stream) {
  const int row_groups = row_groups_of(cache, heads), groups = groups_of(cache, heads, B, width);
  if (cache.pages == 0) width = 0;                  // no token has a page: nothing of the cache is touched
  const int page16 = cache.page_size / 16;
  float *const part = (float *)((char *)workspace + before_bytes(B));
  AttentionArgs a{(const char *)cache.k, (const char *)cache.v, cache.k_scales, cache.v_scales, cache.pages, cache.page_stride,
                  cache.head_stride, (int)cache.token_stride * (cache.format == FMT_BF16 ? 2 : 1), (const uint16_t *)q, q_stride,
                  q_head_stride, block_tables, lengths, table_stride, ((int64_t)1 << 38) / page16 + 1,
                  (int64_t)width * cache.page_size, (int)B, cache.page_size, cache.heads, heads / cache.heads, row_groups,
                  cache.head_dim, scale * 1.44269504088896340736f, (uint16_t *)out, part, part + (size_t)groups * 2 * ATT_ROWS * cache.head_dim,
                  (int *)workspace};
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(groups), dim3(256), 0, stream, a); };
  const bool f8 = cache.format == FMT_MXFP8;
  if (cache.head_dim <= 64) go(f8 ? paged_attention_kernel<64, true> : paged_attention_kernel<64, false>);
  else if (cache.head_dim <= 128) go(f8 ? paged_attention_kernel<128, true> : paged_attention_kernel<128, false>);
  else go(f8 ? paged_attention_kernel<256, true> : paged_attention_kernel<256, false>);
  hipLaunchKernelGGL(paged_attention_join_kernel, dim3((unsigned)(B * heads)), dim3(256), 0, stream, a, groups);
  return hipGetLastError();
}

}  // namespace torq
