// Products of rows and weights that are both held in 8 bits, with a scale for each row and each output channel: the projections of a layer.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "hfx_device.h"
#include "hfx_launch.h"

namespace hfx {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// Results of one lane: four channels n .. n + 3 of row m.
template <bool Fp32>
__device__ __forceinline__ void store_results(const MatmulRows& a, int m, int n, float row_scale, int c0, int c1, int c2, int c3) {
#pragma clang fp contract(off)
  const int c[4] = {c0, c1, c2, c3};
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int at = min(n + e, a.n - 1);
    y[e] = (float)c[e] * row_scale * a.weight_scales[at];
    if (a.bias) y[e] += __builtin_bit_cast(float, (unsigned)a.bias[at] << 16);
  }
  const long to = (long)m * a.out_stride + n;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < a.n) {
      if constexpr (Fp32) static_cast<float*>(a.out)[to + e] = y[e];
      else static_cast<__bf16*>(a.out)[to + e] = (__bf16)y[e];
    }
}

// A wavefront's 32 channels by 32 rows, straight from memory: a lane has 16 values of one channel and of one row.
template <bool Fp32>
__global__ __launch_bounds__(64) void matmul_rows_plain_kernel(const MatmulRows a) {
  const int lane = threadIdx.x, j = lane >> 5;
  const long tiles_n = (a.n + 31) / 32, tiles = tiles_n * ((a.rows + 31) / 32);
  for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
  const int n0 = (int)(tile % tiles_n) * 32, m0 = (int)(tile / tiles_n) * 32;
  const int8_t* const w = a.weight + (long)min(n0 + (lane & 31), a.n - 1) * a.weight_stride;
  const int8_t* const x = a.codes + (long)min(m0 + (lane & 31), a.rows - 1) * a.codes_stride;
  i32x16 acc = {};
  for (int k = 0; k < a.k; k += 32) {
    const bool in = k + 16 * j < a.k;
    i32x4 fw = *reinterpret_cast<const i32x4*>(w + (in ? k + 16 * j : 0));
    i32x4 fx = *reinterpret_cast<const i32x4*>(x + (in ? k + 16 * j : 0));
    if (!in) fx = i32x4{0, 0, 0, 0};
    acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw, fx, acc, 0, 0, 0);
  }
  const int m = m0 + (lane & 31);
  if (m >= a.rows) continue;
  const float scale = a.scales[m];
#pragma unroll
  for (int q = 0; q < 4; ++q) store_results<Fp32>(a, m, n0 + 8 * q + 4 * j, scale, acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
  }
}

hipError_t launch_matmul_rows(const MatmulRows& a, bool fp32, hipStream_t stream) {
  const dim3 grid((unsigned)std::min<long>((a.n + 31l) / 32 * ((a.rows + 31l) / 32), 1 << 20));
  return launch(fp32 ? matmul_rows_plain_kernel<true> : matmul_rows_plain_kernel<false>, grid, 64, stream, a);
}

}  // namespace hfx
