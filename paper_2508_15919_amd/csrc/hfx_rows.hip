// Rows of a step between its attention calls: the root-mean-square norm of the residual stream, with its addition, and rows in 8 bits.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

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

// What the lanes of a wavefront hold, with the lanes that differ in the lowest bits: two neighbours, four, eight, sixteen.
template <int Step>
__device__ __forceinline__ int neighbours(int x) {
  constexpr int kControl[4] = {0xb1, 0x4e, 0x141, 0x140};      // exchanges in fours; half a row of 16, and a row, the other way round
  return __builtin_amdgcn_mov_dpp(x, kControl[Step], 0xf, 0xf, true);
}
template <int Step>
__device__ __forceinline__ double neighbours(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const unsigned low = (unsigned)neighbours<Step>((int)u), high = (unsigned)neighbours<Step>((int)(u >> 32));
  return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}
__device__ __forceinline__ double lane_of(double x, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const unsigned low = (unsigned)__builtin_amdgcn_readlane((int)u, lane), high = (unsigned)__builtin_amdgcn_readlane((int)(u >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}

// The largest `top` (bits of magnitudes: a NaN has larger ones than any number) and the sum of `sum` over the T threads of a workgroup.
template <int T, bool Sum>
__device__ __forceinline__ void reduce_row(unsigned& top, double& sum) {
  auto step = [&](auto i) {
    constexpr int kStep = decltype(i)::value;
    top = max(top, (unsigned)neighbours<kStep>((int)top));
    if constexpr (Sum) sum += neighbours<kStep>(sum);
  };
  step(std::integral_constant<int, 0>());
  step(std::integral_constant<int, 1>());
  step(std::integral_constant<int, 2>());
  step(std::integral_constant<int, 3>());
  const unsigned t = top;
  top = max(max((unsigned)__builtin_amdgcn_readlane((int)t, 0), (unsigned)__builtin_amdgcn_readlane((int)t, 16)),
            max((unsigned)__builtin_amdgcn_readlane((int)t, 32), (unsigned)__builtin_amdgcn_readlane((int)t, 48)));
  if constexpr (Sum) sum = (lane_of(sum, 0) + lane_of(sum, 16)) + (lane_of(sum, 32) + lane_of(sum, 48));
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

// 16 bytes of a row that is read or written once; Past: past the caches.
template <bool Past>
__device__ __forceinline__ u32x4 load_piece(const uint16_t* p) {
  const u32x4* v = reinterpret_cast<const u32x4*>(p);
  return Past ? __builtin_nontemporal_load(v) : *v;
}
template <bool Past>
__device__ __forceinline__ void store_piece(uint16_t* p, const u32x4& x) {
  u32x4* v = reinterpret_cast<u32x4*>(p);
  if constexpr (Past) __builtin_nontemporal_store(x, v);
  else *v = x;
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
// Eight codes: the product rounded to fp32, then to the nearest whole number, ties to even: added to 1.5 2^23, whose unit in the last place is one, it leaves its
// lowest eight bits at the end of the sum.
__device__ __forceinline__ uint2 to_codes(const float* v, float factor) {
#pragma clang fp contract(off)
  if (factor == 0.0f) return make_uint2(0, 0);
  unsigned w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    unsigned c[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float t = v[4 * h + e] * factor;
      c[e] = __builtin_bit_cast(unsigned, t + 12582912.0f);
    }
    const unsigned low = __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400u), high = __builtin_amdgcn_perm(c[3], c[2], 0x04000c0cu);
    w[h] = low | high;
  }
  return make_uint2(w[0], w[1]);
}

// v / (1 + e^-v), as v t / (1 + t) below zero and v / (1 + t) above, t = e^-|v|: t = 2^p (1 + q ln 2) with p the product of -|v| and log2 e rounded and q what it lost, the quotient by a
// reciprocal and one correction (an IEEE division and expf take three times the instructions, and rows of 8192 gated values were bound by them: 2500 of them 27 us).  Past 80, where 1 + t is
// 1 and t leaves the range of normal numbers, 2^(p + 64) takes the place of 2^p, of a p that ends at -200 log2 e, and the product with v the rest.  Which form a value takes goes by itself alone;
// Far: there are such values among the wavefront's.
template <bool Far>
__device__ __forceinline__ float silu_of(float v) {
#pragma clang fp contract(off)
  constexpr float kLog2e = 0x1.715476p+0f, kLog2eRest = 0x1.4ae0cp-26f, kLn2 = 0x1.62e43p-1f;
  const bool far = Far && !(fabsf(v) <= 80.0f);
  const float a = Far ? fmaxf(-fabsf(v), -200.0f) : -fabsf(v), p = a * kLog2e, q = __builtin_fmaf(a, kLog2eRest, __builtin_fmaf(a, kLog2e, -p));
  float t = __builtin_amdgcn_exp2f(far ? p + 64.0f : p);
  t = __builtin_fmaf(t, q * kLn2, t);
  const float n = v < 0.0f ? (far ? v * t * 0x1p-64f : v * t) : v, d = 1.0f + t, r = __builtin_amdgcn_rcpf(d), y = n * r;
  return far ? n : __builtin_fmaf(__builtin_fmaf(-d, y, n), r, y);
}
__device__ __forceinline__ void silu(float* v) {
  float most = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[e]));
  if (__builtin_expect(__any(!(most <= 80.0f)), 0)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = silu_of<true>(v[e]);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = silu_of<false>(v[e]);
}

// a^(-1/2), by the hardware's estimate and two steps of Newton's method (a square root and divisions in 64 bits are chains of forty dependent operations).
__device__ __forceinline__ double inverse_root(double a) {
  double y = __builtin_amdgcn_rsq(a);
  if (a > 0.0 && a < __builtin_inf()) {
#pragma unroll
    for (int i = 0; i < 2; ++i) y = __builtin_fma(y * 0.5, __builtin_fma(-a * y, y, 1.0), y);
  }
  return y;
}

// One workgroup of T threads per row, eight values of it to a thread at a time; the first P of those stay in registers between the two passes, the ones behind
// (rows of more than 8 T P values) are read again.  The row of x and the residual is rounded to bf16 before anything else is formed from it: the norm is that of
// the stream as it is kept.  Squares of bf16 numbers are exact in fp32 but may pass its range, and are summed in 64 bits.  A value's code is the
// nearest to h w 127 / top: the norm's own factor r is in the scale alone, top r / 127, so that codes do not depend on the order of the sum.
// Bound by memory on many rows (8224 of 4096 with the sum and a bf16 result, 270 MB, 43.6 us, 6.2 TB/s; a plain copy has 4.9), by the chain of launch, loads, reduction and stores on few: 4 rows 2.7 us a call in a
// captured graph.
template <int T, int P, bool Past>
__global__ __launch_bounds__(T) void rms_norm_kernel(const RmsNorm a) {
  const long row = blockIdx.x;
  const uint16_t* const x = a.x + row * a.x_stride;
  const uint16_t* const residual = a.residual ? a.residual + row * a.residual_stride : nullptr;
  uint16_t* const kept = a.residual ? a.sum + row * a.cols : nullptr;
  float h[P][8];
  u32x4 weight[P];
  unsigned top = 0;
  double sum = 0.0;
  auto first = [&](int c, float* v, u32x4& wide) {
    wide = *reinterpret_cast<const u32x4*>(a.weight + c);
    widen8(load_piece<Past>(x + c), v);
    if (residual) {
      float z[8];
      widen8(load_piece<Past>(residual + c), z);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += z[e];
      const u32x4 r = narrow8(v);
      store_piece<Past>(kept + c, r);
      widen8(r, v);
    }
    float w[8];
    widen8(wide, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sum += (double)v[e] * (double)v[e];
      top = max(top, magnitude_bits(v[e] * w[e]));
    }
  };
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int c = (p * T + (int)threadIdx.x) * 8;
    if (c < a.cols) first(c, h[p], weight[p]);
  }
  for (int c = (P * T + (int)threadIdx.x) * 8; c < a.cols; c += T * 8) {
    float v[8];
    u32x4 w;
    first(c, v, w);
  }
  reduce_row<T, true>(top, sum);
  const double r = inverse_root(__builtin_fma(sum, a.part, (double)a.eps));
  const float up = r > 0x1p100 ? 0x1p64f : 1.0f, rf = (float)(r / (double)up);      // (rows of the smallest numbers, without eps, have an r past the range of fp32)
  const Scaling s = scaling_of(top);
  if (a.codes && threadIdx.x == 0) a.scales[row] = (float)((double)s.top * r * (1.0 / 127.0));
  auto second = [&](int c, const float* v, const u32x4& wide) {
    float w[8], y[8];
    widen8(wide, w);
    if (a.codes) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = v[e] * w[e];
      *reinterpret_cast<uint2*>(a.codes + row * a.cols + c) = to_codes(y, s.factor);
    }
    if (a.out) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = v[e] * up * rf * w[e];
      *reinterpret_cast<u32x4*>(a.out + row * a.cols + c) = narrow8(y);
    }
  };
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int c = (p * T + (int)threadIdx.x) * 8;
    if (c < a.cols) second(c, h[p], weight[p]);
  }
  for (int c = (P * T + (int)threadIdx.x) * 8; c < a.cols; c += T * 8) {
    float v[8];
    widen8(*reinterpret_cast<const u32x4*>((kept ? kept : x) + c), v);
    second(c, v, *reinterpret_cast<const u32x4*>(a.weight + c));
  }
}

// Rows through an activation, times other rows, to bf16 and to 8 bits.  Laid out as the norm, and bound as it is: 2500 gated rows of 8192 (102 MB) 20.2 us, 5.1
// TB/s; 64 of them 3.3 to 3.4 us a call in a captured graph.
template <int T, int P, bool Past>
__global__ __launch_bounds__(T) void quantise_rows_kernel(const QuantiseRows a) {
  const long row = blockIdx.x;
  const uint16_t* const x = a.x + row * a.x_stride;
  const uint16_t* const times = a.times ? a.times + row * a.times_stride : nullptr;
  float held[P][8];
  unsigned top = 0;
  double none = 0.0;
  auto value = [&](int c, float* v) {
    widen8(load_piece<Past>(x + c), v);
    if (a.activation == HFX_ACT_SILU) silu(v);
    if (times) {
      float z[8];
      widen8(load_piece<Past>(times + c), z);
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

// Threads and pieces for rows of `cols` values: one piece to a thread up to 4096, two up to 16384, four and from there on a second reading.  (8224 rows of 4096: 512 threads of one piece
// 48.9 us, 256 of two 52.9, 128 of four 54.6, 1024 of one 65.2; four rows 3.2, 3.7, 4.9 and 3.3.  8224 rows of 1024: 128 of one 17.1, 64 of two 17.3, 256 of one 19.9.  2500 gated rows of 8192: 512 of two
// 22.0, 1024 of one 26.8, 256 of four 23.5.)  Up to 256 rows on
// their way to 8 bits, each on a unit of its own, take 1024 of one from 4112 to 8192 values, with an activation, a factor, both or neither: with 512 of two 64 rows of 8192 3.60 and 3.29 us (gated), 2.46 and
// 2.33 (plain), of 4112 3.16 and 2.91, 2.34 and 2.16; 256 of 8192 3.80 and 3.57, 2.66 and 2.59.  384 plain rows of 8192 2.93 and 3.10, gated 5.50 and 5.44.  The norm's rows do not: 64 of 8192 3.5 and 3.7.
// Rows of more than 32 MB in all go past the caches where nobody reads them soon: what comes in, and the sum, which the next norm reads (1024 rows of 4096, 29 MB in 8 bits, with a reader of the
// sum behind it 15.3 -> 13.1 us; 8224 rows alone 46.7 -> 44.3; 512 rows 8.9 -> 9.3).  What the next call reads, codes and results, stays in reach.
template <class A, class Pick>
static hipError_t launch_rows(const A& a, int rows, long bytes, hipStream_t stream, Pick pick) {
  const bool past = bytes > (32l << 20);
  auto run = [&](auto threads, auto pieces) {
    constexpr int T = decltype(threads)::value;
    return launch(past ? pick(threads, pieces, std::true_type()) : pick(threads, pieces, std::false_type()), dim3((unsigned)rows), (unsigned)T, stream, a);
  };
  const auto one = std::integral_constant<int, 1>();
  const auto two = std::integral_constant<int, 2>();
  const auto four = std::integral_constant<int, 4>();
  if (a.cols <= 512) return run(std::integral_constant<int, 64>(), one);
  if (a.cols <= 1024) return run(std::integral_constant<int, 128>(), one);
  if (a.cols <= 2048) return run(std::integral_constant<int, 256>(), one);
  if (a.cols <= 4096) return run(std::integral_constant<int, 512>(), one);
  if constexpr (std::is_same_v<A, QuantiseRows>)
    if (rows <= 256 && a.cols <= 8192) return run(std::integral_constant<int, 1024>(), one);
  if (a.cols <= 8192) return run(std::integral_constant<int, 512>(), two);
  if (a.cols <= 16384) return run(std::integral_constant<int, 1024>(), two);
  return run(std::integral_constant<int, 1024>(), four);
}

hipError_t launch_rms_norm(RmsNorm a, int rows, hipStream_t stream) {
  a.part = 1.0 / a.cols;
  return launch_rows(a, rows, (long)rows * a.cols * ((a.residual ? 6 : 2) + (a.out ? 2 : 0) + (a.codes ? 1 : 0)), stream, [](auto t, auto p, auto past) {
    return rms_norm_kernel<decltype(t)::value, decltype(p)::value, decltype(past)::value>;
  });
}

hipError_t launch_quantise_rows(const QuantiseRows& a, int rows, hipStream_t stream) {
  return launch_rows(a, rows, (long)rows * a.cols * ((a.times ? 4 : 2) + (a.out ? 2 : 0) + (a.codes ? 1 : 0)), stream, [](auto t, auto p, auto past) {
    return quantise_rows_kernel<decltype(t)::value, decltype(p)::value, decltype(past)::value>;
  });
}

}  // namespace hfx
