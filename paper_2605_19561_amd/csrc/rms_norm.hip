// torq_add_rms_norm: s = x + residual, out = s / sqrt(mean(s^2) + eps) * weight, to bf16 or MXFP8.  One pass over the data:
// HBM-bound, 8 bytes a value with a residual and bf16 out, 7 1/32 to MXFP8.  Measured: [8192, 8192] 79.4 us (6.8 TB/s), [2048, 5120]
// to MXFP8 13.4 us (5.5 TB/s), one row of 4096 3.1 us in a graph.
//
// 16 to 1024 lanes take a row; its s stay in registers between the sum of squares and the product, so x and residual are read once.
// A lane holds 8 consecutive values (16-byte loads and stores), four lanes a block of MXFP8.
#include "torq_device.h"
#include "torq_internal.h"

namespace torq {

__device__ __forceinline__ void unpack8(u32x4 v, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16_bits_to_f32(v[i] & 0xFFFFu);
    f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
  }
}
template <bool ONCE>
__device__ __forceinline__ u32x4 load16(const u32x4 *p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool ONCE>
__device__ __forceinline__ void store16(u32x4 *p, u32x4 v) {
  if constexpr (ONCE) __builtin_nontemporal_store(v, p);
  else *p = v;
}
__device__ __forceinline__ u32x4 pack8_bf16(const float (&f)[8]) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)f[i];
  return __builtin_bit_cast(u32x4, v);
}

// x and residual of more than this are read with the non-temporal hint (see ONE_PASS_INPUT_BYTES; outputs as large as the inputs
// leave less of the cache to them, so the line is lower).  us without / with the hint, from HBM and with x just written (with the
// writing): [2048, 5120] to MXFP8, 42 MB 13.4 / 16.1; [4096, 8192] 134 MB 42.5 / 43.3, 72.3 / 62.0; [6144, 8192] 73.2 / 62.1, 107.8 /
// 103.2; [8192, 8192] 95.5 / 79.4, 144.9 / 136.2, to MXFP8 85.5 / 74.3, 135.2 / 127.8; [16384, 8192] written 286.7 / 283.4
// residual_out goes past the cache with them: out is what comes next, residual_out a layer later.  [8192, 8192] called in turn with one
// set of outputs 94.4 -> 80.3, to MXFP8 84.5 -> 74.6, [16384, 8192] with outputs of their own 187 -> 156.
constexpr double ONE_PASS_NORM_BYTES = 120.0 * 1024 * 1024;

// TPR: lanes of a row, CH: pieces of 8 values that each of them holds.
template <int TPR, int CH, int FMT, bool ONCE>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) add_rms_norm_kernel(const u32x4 *x, const u32x4 *residual, const u32x4 *weight,
                                                                            int64_t M, int n8, float inv_d, float eps,
                                                                            u32x4 *residual_out, void *out, uint8_t *scales) {
  constexpr int WG = TPR > 256 ? TPR : 256, ROWS = WG / TPR;
  __shared__ float sums[WG / 64];
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
  const int lane = threadIdx.x % TPR;
  if (ROWS > 1 && row >= M) return;                 // (no barrier where a workgroup has several rows)
  const int64_t at = row * n8 + lane;
  float s[CH][8], total = 0.0f;
  u32x4 xs[CH], rs[CH], ws[CH];                     // (the weights too ahead of the sum: a row alone waits for memory once)
#pragma unroll
  for (int c = 0; c < CH; ++c)
    if (c * TPR + lane < n8) {
      xs[c] = load16<ONCE>(x + at + c * TPR);
      if (residual) rs[c] = load16<ONCE>(residual + at + c * TPR);
      ws[c] = weight[c * TPR + lane];
    }
#pragma unroll
  for (int c = 0; c < CH; ++c)
    if (c * TPR + lane < n8) {
      unpack8(xs[c], s[c]);
      if (residual) {
        float r[8];
        unpack8(rs[c], r);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[c][e] += r[e];
        store16<ONCE>(residual_out + at + c * TPR, pack8_bf16(s[c]));
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) total += s[c][e] * s[c][e];
    }
#pragma unroll
  for (int o = (TPR < 64 ? TPR : 64) / 2; o; o >>= 1) total += __shfl_xor(total, o);
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = total;
    __syncthreads();
    total = 0.0f;
#pragma unroll
    for (int w = 0; w < WG / 64; ++w) total += sums[w];
  }
  const float r = 1.0f / sqrtf(total * inv_d + eps);
#pragma unroll
  for (int c = 0; c < CH; ++c)
    if (c * TPR + lane < n8) {
      float w[8];
      unpack8(ws[c], w);
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] *= s[c][e] * r;
      if constexpr (FMT == FMT_BF16) {
        static_cast<u32x4 *>(out)[at + c * TPR] = pack8_bf16(w);
      } else {
        const uint32_t byte = mxfp8_scale_from_amax(quad_amax_nan(amax8_nan(w)));
        static_cast<uint2 *>(out)[at + c * TPR] = pack8_e4m3(w, byte);
        if ((lane & 3) == 0) scales[(at + c * TPR) >> 2] = (uint8_t)byte;
      }
    }
}

hipError_t launch_add_rms_norm(const void *x, const void *residual, const void *weight, int64_t M, int d, float eps,
                               int format, void *residual_out, void *out, uint8_t *scales, hipStream_t stream) {
  const int n8 = d / 8;
  const bool once = (residual ? 4.0 : 2.0) * (double)M * d > ONE_PASS_NORM_BYTES;
  auto go = [&](auto tpr, auto ch) {
    constexpr int TPR = decltype(tpr)::value, CH = decltype(ch)::value, WG = TPR > 256 ? TPR : 256, ROWS = WG / TPR;
    auto kernel = format == FMT_BF16 ? (once ? add_rms_norm_kernel<TPR, CH, FMT_BF16, true> : add_rms_norm_kernel<TPR, CH, FMT_BF16, false>)
                                     : (once ? add_rms_norm_kernel<TPR, CH, FMT_MXFP8, true> : add_rms_norm_kernel<TPR, CH, FMT_MXFP8, false>);
    constexpr int64_t MOST = most_workgroups(WG) * ROWS;       // rows of one launch
    for (int64_t m = 0; m < M; m += MOST) {
      const int64_t rows = M - m < MOST ? M - m : MOST;
      const size_t at = (size_t)m * d * 2;
      hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + ROWS - 1) / ROWS)), dim3(WG), 0, stream, (const u32x4 *)((const char *)x + at),
                         residual ? (const u32x4 *)((const char *)residual + at) : nullptr, (const u32x4 *)weight, rows, n8,
                         1.0f / (float)d, eps, residual ? (u32x4 *)((char *)residual_out + at) : nullptr,
                         (void *)((char *)out + (format == FMT_BF16 ? at : at / 2)), scales ? scales + (size_t)m * (d / 32) : nullptr);
    }
    return hipGetLastError();
  };
  using std::integral_constant;
  // Lanes of a row: short rows share a workgroup, without a barrier, and a long one's loads are spread over more of the CU.  With 256
  // lanes for every row, against this: [65536, 128] 30.6 -> 7.3 us, [500000, 64] to MXFP8 387 -> 47, [1, 28672] 10.3 -> 4.7,
  // [2300, 25600] to MXFP8 53 -> 38.
  if (n8 <= 16) return go(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  if (n8 <= 32) return go(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  if (n8 <= 64) return go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (n8 <= 128) return go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  if (n8 <= 256) return go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (n8 <= 512) return go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  if (n8 <= 1024) return go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  if (n8 <= 2048) return go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  return go(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

}  // namespace torq
