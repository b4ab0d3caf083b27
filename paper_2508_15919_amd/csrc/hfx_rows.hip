// Rows of a step between its attention calls: the root-mean-square norm of the residual stream, with its addition, and rows in 8 bits.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/hfxattn.h"
#include "hfx_device.h"
#include "hfx_launch.h"

namespace hfx {

__device__ __forceinline__ void widen8(const u32x4& v, float* x) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    x[2 * w] = __builtin_bit_cast(float, v[w] << 16);
    x[2 * w + 1] = __builtin_bit_cast(float, v[w] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4 narrow8(const float* x) {
  u32x4 v;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const bf16x2 r = {(__bf16)x[2 * w], (__bf16)x[2 * w + 1]};
    v[w] = __builtin_bit_cast(unsigned, r);
  }
  return v;
}
__device__ __forceinline__ unsigned magnitude_bits(float x) { return __builtin_bit_cast(unsigned, x) & 0x7fffffffu; }

// The largest `top` (bits of magnitudes: a NaN has larger ones than any number) and the sum of `sum` over the T threads of a workgroup.
template <int T, bool Sum>
__device__ __forceinline__ void reduce_row(unsigned& top, double& sum) {
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    top = max(top, (unsigned)__shfl_xor((int)top, s, 64));
    if constexpr (Sum) sum += __shfl_xor(sum, s, 64);
  }
  if constexpr (T > 64) {
    __shared__ double part_sum[T / 64];
    __shared__ unsigned part_top[T / 64];
    const int wave = (int)threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
      part_top[wave] = top;
      if constexpr (Sum) part_sum[wave] = sum;
    }
    __syncthreads();
    top = 0;
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < T / 64; ++i) {
      top = max(top, part_top[i]);
      if constexpr (Sum) sum += part_sum[i];
    }
  }
}

// Factor from values to codes, and what the largest magnitude stands for.  A largest magnitude below 2^-100 counts as that, so that the factor is finite; a row
// with something that is not finite has NaN for its scale, and codes of zero.
struct Scaling {
  float factor, top;
};
__device__ __forceinline__ Scaling scaling_of(unsigned top_bits) {
  if (top_bits >= 0x7f800000u) return {0.0f, __builtin_nanf("")};
  const float top = fmaxf(__builtin_bit_cast(float, top_bits), 0x1p-100f);
  return {127.0f / top, top};
}
// Eight codes: the product rounded to fp32, then to the nearest whole number, ties to even.
__device__ __forceinline__ uint2 to_codes(const float* v, float factor) {
  unsigned w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int c[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e] = factor == 0.0f ? 0 : (int)__builtin_rintf(v[4 * h + e] * factor);
    w[h] = (unsigned)(c[0] & 255) | (unsigned)(c[1] & 255) << 8 | (unsigned)(c[2] & 255) << 16 | (unsigned)c[3] << 24;
  }
  return make_uint2(w[0], w[1]);
}

// One workgroup of T threads per row, eight values of it to a thread at a time; the first P of those stay in registers between the two passes, the ones behind
// (rows of more than 8 T P values) are read again.  The row of x and the residual is rounded to bf16 before anything else is formed from it: the norm is that of
// the stream as it is kept.  Squares of bf16 numbers are exact in fp32 but may pass its range, and are summed in 64 bits.  A value's code is the
// nearest to h w 127 / top: the norm's own factor r is in the scale alone, top r / 127, so that codes do not depend on the order of the sum.
template <int T, int P>
__global__ __launch_bounds__(T) void rms_norm_kernel(const RmsNorm a) {
  const long row = blockIdx.x;
  const uint16_t* const x = a.x + row * a.x_stride;
  const uint16_t* const residual = a.residual ? a.residual + row * a.residual_stride : nullptr;
  uint16_t* const kept = a.residual ? a.sum + row * a.cols : nullptr;
  float h[P][8];
  unsigned top = 0;
  double sum = 0.0;
  auto first = [&](int c, float* v) {
    widen8(*reinterpret_cast<const u32x4*>(x + c), v);
    if (residual) {
      float z[8];
      widen8(*reinterpret_cast<const u32x4*>(residual + c), z);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += z[e];
      const u32x4 r = narrow8(v);
      *reinterpret_cast<u32x4*>(kept + c) = r;
      widen8(r, v);
    }
    float w[8];
    widen8(*reinterpret_cast<const u32x4*>(a.weight + c), w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sum += (double)v[e] * (double)v[e];
      top = max(top, magnitude_bits(v[e] * w[e]));
    }
  };
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int c = (p * T + (int)threadIdx.x) * 8;
    if (c < a.cols) first(c, h[p]);
  }
  for (int c = (P * T + (int)threadIdx.x) * 8; c < a.cols; c += T * 8) {
    float v[8];
    first(c, v);
  }
  reduce_row<T, true>(top, sum);
  const double r = 1.0 / __builtin_sqrt(sum / (double)a.cols + (double)a.eps);
  const float rf = (float)r;
  const Scaling s = scaling_of(top);
  if (a.codes && threadIdx.x == 0) a.scales[row] = (float)((double)s.top * r / 127.0);
  auto second = [&](int c, const float* v) {
    float w[8], y[8];
    widen8(*reinterpret_cast<const u32x4*>(a.weight + c), w);
    if (a.codes) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = v[e] * w[e];
      *reinterpret_cast<uint2*>(a.codes + row * a.cols + c) = to_codes(y, s.factor);
    }
    if (a.out) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = v[e] * rf * w[e];
      *reinterpret_cast<u32x4*>(a.out + row * a.cols + c) = narrow8(y);
    }
  };
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int c = (p * T + (int)threadIdx.x) * 8;
    if (c < a.cols) second(c, h[p]);
  }
  for (int c = (P * T + (int)threadIdx.x) * 8; c < a.cols; c += T * 8) {
    float v[8];
    widen8(*reinterpret_cast<const u32x4*>((kept ? kept : x) + c), v);
    second(c, v);
  }
}

// Rows through an activation, times other rows, to bf16 and to 8 bits.  Laid out as the norm.
template <int T, int P>
__global__ __launch_bounds__(T) void quantise_rows_kernel(const QuantiseRows a) {
  const long row = blockIdx.x;
  const uint16_t* const x = a.x + row * a.x_stride;
  const uint16_t* const times = a.times ? a.times + row * a.times_stride : nullptr;
  float held[P][8];
  unsigned top = 0;
  double none = 0.0;
  auto value = [&](int c, float* v) {
    widen8(*reinterpret_cast<const u32x4*>(x + c), v);
    if (a.activation == HFX_ACT_SILU) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float t = expf(-fabsf(v[e]));      // (that of -v alone passes fp32's range where the result is still a normal number)
        v[e] = (v[e] < 0.0f ? v[e] * t : v[e]) / (1.0f + t);
      }
    }
    if (times) {
      float z[8];
      widen8(*reinterpret_cast<const u32x4*>(times + c), z);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= z[e];
    }
  };
  auto first = [&](int c, float* v) {
    value(c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, magnitude_bits(v[e]));
    if (a.out) *reinterpret_cast<u32x4*>(a.out + row * a.cols + c) = narrow8(v);
  };
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int c = (p * T + (int)threadIdx.x) * 8;
    if (c < a.cols) first(c, held[p]);
  }
  for (int c = (P * T + (int)threadIdx.x) * 8; c < a.cols; c += T * 8) {
    float v[8];
    first(c, v);
  }
  if (!a.codes) return;
  reduce_row<T, false>(top, none);
  const Scaling s = scaling_of(top);
  if (threadIdx.x == 0) a.scales[row] = s.top / 127.0f;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int c = (p * T + (int)threadIdx.x) * 8;
    if (c < a.cols) *reinterpret_cast<uint2*>(a.codes + row * a.cols + c) = to_codes(held[p], s.factor);
  }
  for (int c = (P * T + (int)threadIdx.x) * 8; c < a.cols; c += T * 8) {
    float v[8];
    value(c, v);
    *reinterpret_cast<uint2*>(a.codes + row * a.cols + c) = to_codes(v, s.factor);
  }
}

hipError_t launch_rms_norm(const RmsNorm& a, int rows, hipStream_t stream) {
  if (a.cols <= 1024) return launch(rms_norm_kernel<64, 2>, dim3(rows), 64, stream, a);
  if (a.cols <= 8192) return launch(rms_norm_kernel<256, 4>, dim3(rows), 256, stream, a);
  return launch(rms_norm_kernel<1024, 4>, dim3(rows), 1024, stream, a);
}

hipError_t launch_quantise_rows(const QuantiseRows& a, int rows, hipStream_t stream) {
  if (a.cols <= 1024) return launch(quantise_rows_kernel<64, 2>, dim3(rows), 64, stream, a);
  if (a.cols <= 8192) return launch(quantise_rows_kernel<256, 4>, dim3(rows), 256, stream, a);
  return launch(quantise_rows_kernel<1024, 4>, dim3(rows), 1024, stream, a);
}

}  // namespace hfx
