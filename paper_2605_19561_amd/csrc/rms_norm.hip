// torq_add_rms_norm: s = x + residual, out = s / sqrt(mean(s^2) + eps) * weight, to bf16 or MXFP8.  One pass over the data:
// HBM-bound, 8 bytes a value with a residual and bf16 out, 7 1/32 to MXFP8.
//
// A workgroup takes a row; its s stay in registers between the sum of squares and the product, so x and residual are read once.
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
__device__ __forceinline__ u32x4 pack8_bf16(const float (&f)[8]) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)f[i];
  return __builtin_bit_cast(u32x4, v);
}

// CH: pieces of 8 values that a lane of the 256 holds.
template <int CH, int FMT>
__global__ void __launch_bounds__(256) add_rms_norm_kernel(const u32x4 *x, const u32x4 *residual, const u32x4 *weight, int n8,
                                                           float inv_d, float eps, u32x4 *residual_out, void *out,
                                                           uint8_t *scales) {
  __shared__ float sums[4];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  x += row * n8;
  float s[CH][8], total = 0.0f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int i = c * 256 + tid;
    if (i >= n8) break;
    unpack8(x[i], s[c]);
    if (residual) {
      float r[8];
      unpack8(residual[row * n8 + i], r);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[c][e] += r[e];
      residual_out[row * n8 + i] = pack8_bf16(s[c]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) total += s[c][e] * s[c][e];
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
  if ((tid & 63) == 0) sums[tid >> 6] = total;
  __syncthreads();
  total = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  const float r = 1.0f / sqrtf(total * inv_d + eps);
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int i = c * 256 + tid;
    if (i >= n8) break;
    float w[8];
    unpack8(weight[i], w);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] *= s[c][e] * r;
    if constexpr (FMT == FMT_BF16) {
      static_cast<u32x4 *>(out)[row * n8 + i] = pack8_bf16(w);
    } else {
      const uint32_t byte = mxfp8_scale_from_amax(quad_amax_nan(amax8_nan(w)));
      static_cast<uint2 *>(out)[row * n8 + i] = pack8_e4m3(w, byte);
      if ((tid & 3) == 0) scales[(row * n8 + i) >> 2] = (uint8_t)byte;
    }
  }
}

hipError_t launch_add_rms_norm(const void *x, const void *residual, const void *weight, int64_t M, int d, float eps,
                               int format, void *residual_out, void *out, uint8_t *scales, hipStream_t stream) {
  const int n8 = d / 8, ch = (n8 + 255) / 256;
  auto go = [&](auto kernel) {
    for (int64_t m = 0; m < M; m += 1 << 30) {      // rows of one launch: the grid's limit is 2^31 - 1
      const int64_t rows = M - m < (1 << 30) ? M - m : 1 << 30;
      const size_t at = (size_t)m * d * 2;
      hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(256), 0, stream, (const u32x4 *)((const char *)x + at),
                         residual ? (const u32x4 *)((const char *)residual + at) : nullptr, (const u32x4 *)weight, n8,
                         1.0f / (float)d, eps, residual ? (u32x4 *)((char *)residual_out + at) : nullptr,
                         (void *)((char *)out + (format == FMT_BF16 ? at : at / 2)), scales ? scales + (size_t)m * (d / 32) : nullptr);
    }
    return hipGetLastError();
  };
  auto of_format = [&](auto chunks) {
    constexpr int CH = decltype(chunks)::value;
    return format == FMT_BF16 ? go(add_rms_norm_kernel<CH, FMT_BF16>) : go(add_rms_norm_kernel<CH, FMT_MXFP8>);
  };
  if (ch <= 1) return of_format(std::integral_constant<int, 1>{});
  if (ch <= 2) return of_format(std::integral_constant<int, 2>{});
  if (ch <= 4) return of_format(std::integral_constant<int, 4>{});
  if (ch <= 8) return of_format(std::integral_constant<int, 8>{});
  return of_format(std::integral_constant<int, 16>{});
}

}  // namespace torq
