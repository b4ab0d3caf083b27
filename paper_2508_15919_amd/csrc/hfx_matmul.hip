// Products of rows and weights that are both held in 8 bits, with a scale for each row and each output channel: the projections of a layer.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "hfx_device.h"
#include "hfx_launch.h"

namespace hfx {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// Four channels n .. n + 3 of row m.
template <bool Fp32>
__device__ __forceinline__ void store_results(const MatmulRows& a, int m, int n, float row_scale, const i32x4& c) {
#pragma clang fp contract(off)
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int at = min(n + e, a.n - 1);
    y[e] = (float)c[e] * row_scale * a.weight_scales[at];
    if (a.bias) y[e] += __builtin_bit_cast(float, (unsigned)a.bias[at] << 16);
  }
  const long to = (long)m * a.out_stride + n;
  if (n + 3 < a.n && (a.out_stride & 3) == 0) {
    if constexpr (Fp32) *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + to) = f32x4{y[0], y[1], y[2], y[3]};
    else *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.out) + to) = bf16x4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < a.n) {
      if constexpr (Fp32) static_cast<float*>(a.out)[to + e] = y[e];
      else static_cast<__bf16*>(a.out)[to + e] = (__bf16)y[e];
    }
}

// ---------------------------------------------------------------- few rows
// 16 channels by up to 16 R rows, the sum cut into steps of 128 that W wavefronts take in turn; weights and rows go straight to registers.  A lane has 32 bytes in a
// row of a step, which two matrix instructions take one half each (any order of the values will do that is the same in both operands), so that
// four lanes ask for a whole line.
template <int R, int W, bool Fp32>
__global__ __launch_bounds__(64 * W) void matmul_few_kernel(const MatmulRows a) {
  __shared__ i32x4 part[W][R][64];
  constexpr int U = 4;                              // steps whose loads are in flight together
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), r = lane & 15, j = lane >> 4;
  const int n0 = (int)blockIdx.x * 16;
  const int8_t* const w = a.weight + (long)min(n0 + r, a.n - 1) * a.weight_stride;
  const int8_t* x[R];
#pragma unroll
  for (int i = 0; i < R; ++i) x[i] = a.codes + (long)min(16 * i + r, a.rows - 1) * a.codes_stride;
  i32x4 acc[R] = {};
  const i32x4 zero = {0, 0, 0, 0};
  for (int s0 = wave * 128; s0 < a.k; s0 += U * W * 128) {
    i32x4 fw[U][2], fx[U][R][2];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = s0 + u * W * 128 + 32 * j + 16 * h, at = k < a.k ? k : 0;
        fw[u][h] = *reinterpret_cast<const i32x4*>(w + at);
#pragma unroll
        for (int i = 0; i < R; ++i) fx[u][i][h] = *reinterpret_cast<const i32x4*>(x[i] + at);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool in = s0 + u * W * 128 + 32 * j + 16 * h < a.k;
#pragma unroll
        for (int i = 0; i < R; ++i) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u][h], in ? fx[u][i][h] : zero, acc[i], 0, 0, 0);
      }
  }
#pragma unroll
  for (int i = 0; i < R; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  if (wave >= R) return;
  i32x4 c = part[0][wave][lane];
#pragma unroll
  for (int i = 1; i < W; ++i) c += part[i][wave][lane];
  const int m = 16 * wave + r;
  if (m < a.rows) store_results<Fp32>(a, m, n0 + 4 * j, a.scales[m], c);
}

// ---------------------------------------------------------------- tiles
// Copies 64 pieces of 16 bytes to LDS, lane after lane from `lds` on.
__device__ __forceinline__ void copy_to_lds(const int8_t* base, unsigned offset, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(offset), "s"(base), "s"(lds) : "memory", "m0");
}

// A workgroup's BN channels by BM rows.  Stages of 128 values of the sum go straight from memory to LDS, S of them in a ring; a row's eight 16-byte pieces
// are permuted by bits 1 to 3 of its number, so that 16 lanes that read the same piece of 16 rows meet all banks.  (WN channels by WM rows, and of a
// stage one part of K, belong to a wavefront.)
template <int BN, int BM, int WN, int WM, int K, int S, bool Fp32>
__global__ __launch_bounds__(BN / WN * (BM / WM) * K * 64) void matmul_tile_kernel(const MatmulRows a, int tiles_n, int tiles_m) {
  constexpr int kWaves = BN / WN * (BM / WM) * K, kBytes = (BN + BM) * 128;
  constexpr int LN = BN / 8 / kWaves, LM = BM / 8 / kWaves, TN = WN / 32, TM = WM / 32;
  static_assert(LN * 8 * kWaves == BN && LM * 8 * kWaves == BM, "each wavefront copies whole blocks of eight rows of both");
  __shared__ __attribute__((aligned(1024))) char smem[S * kBytes];
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  const int kpart = wave % K, wn = wave / K % (BN / WN), wm = wave / K / (BN / WN);

  int tile_n, tile_m;
  {
    const unsigned b = blockIdx.x;
    tile_n = b % (unsigned)tiles_n;
    tile_m = b / (unsigned)tiles_n;
  }
  const int n0 = tile_n * BN, m0 = tile_m * BM;
  const int8_t* const weight = a.weight + (long)n0 * a.weight_stride;
  const int8_t* const codes = a.codes + (long)m0 * a.codes_stride;
  const unsigned lds0 = (unsigned)(uintptr_t)smem;

  // block i of eight rows: this lane copies piece `lane % 8` of its place, row lane / 8
  const int stages = (a.k + 127) / 128;
  unsigned off_n[LN], off_m[LM];
  auto offsets = [&](int values) {                  // of a stage with so many values; pieces behind them are piece 0 again
#pragma unroll
    for (int i = 0; i < LN; ++i) {
      const int row = (wave + i * kWaves) * 8 + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
      off_n[i] = (unsigned)min(row, a.n - 1 - n0) * (unsigned)a.weight_stride + (unsigned)(piece * 16 < values ? piece * 16 : 0);
    }
#pragma unroll
    for (int i = 0; i < LM; ++i) {
      const int row = (wave + i * kWaves) * 8 + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
      off_m[i] = (unsigned)min(row, a.rows - 1 - m0) * (unsigned)a.codes_stride + (unsigned)(piece * 16 < values ? piece * 16 : 0);
    }
  };
  auto copy = [&](int stage, int slot) {
    if (stage == stages - 1 && (a.k & 127) != 0) offsets(a.k & 127);
    const unsigned to = lds0 + slot * kBytes;
#pragma unroll
    for (int i = 0; i < LN; ++i) copy_to_lds(weight + (long)stage * 128, off_n[i], to + (wave + i * kWaves) * 1024);
#pragma unroll
    for (int i = 0; i < LM; ++i) copy_to_lds(codes + (long)stage * 128, off_m[i], to + BN * 128 + (wave + i * kWaves) * 1024);
  };
  offsets(128);

  i32x16 acc[TN][TM] = {};
  const int swizzle = (lane >> 1) & 7, half = lane >> 5;
  const int at_n = (wn * WN + (lane & 31)) * 128, at_m = BN * 128 + (wm * WM + (lane & 31)) * 128;
  auto multiply = [&](const char* from, int kk, int values) {
    const int piece = ((2 * kk + half) ^ swizzle) * 16;
    i32x4 fn[TN], fm[TM];
#pragma unroll
    for (int t = 0; t < TN; ++t) fn[t] = *reinterpret_cast<const i32x4*>(from + at_n + t * 4096 + piece);
#pragma unroll
    for (int t = 0; t < TM; ++t) fm[t] = *reinterpret_cast<const i32x4*>(from + at_m + t * 4096 + piece);
    if (values < 128) {
      const int keep = (2 * kk + half) * 16 < values ? -1 : 0;
#pragma unroll
      for (int t = 0; t < TM; ++t) fm[t] &= i32x4{keep, keep, keep, keep};
    }
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int u = 0; u < TM; ++u) acc[t][u] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fn[t], fm[u], acc[t][u], 0, 0, 0);
  };

#pragma unroll
  for (int s = 0; s < S - 1; ++s)
    if (s < stages) copy(s, s);
  // Stage s is here and the place of the one before it free: on with the copies.
  auto next = [&](int s, int slot) {
    if (s + S - 2 < stages) HFX_WAIT_VMCNT((S - 2) * (LN + LM));      // the stages behind it may still be on their way
    else HFX_WAIT_VMCNT(0);
    ring_barrier();
    if (s + S - 1 < stages) copy(s + S - 1, slot == 0 ? S - 1 : slot - 1);
    return smem + slot * kBytes;
  };
  int slot = 0;
  const int whole = a.k >> 7;
  for (int s = 0; s < whole; ++s) {
    const char* const from = next(s, slot);
#pragma unroll
    for (int kk = 0; kk < 4; kk += K) multiply(from, kk + kpart, 128);
    slot = slot == S - 1 ? 0 : slot + 1;
  }
  if (whole < stages) {
    const char* const from = next(whole, slot);
#pragma unroll 1
    for (int kk = kpart; kk < 4; kk += K) multiply(from, kk, a.k & 127);
  }

  if constexpr (K > 1) {                            // the parts of a stage are joined in LDS
    __syncthreads();
    i32x4* const sums = reinterpret_cast<i32x4*>(smem) + (wave / K) * (TN * TM * 4 * 64) + lane;
    for (int p = 1; p < K; ++p) {
      if (kpart == p) {
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
          for (int u = 0; u < TM; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const i32x4 c = {acc[t][u][4 * q], acc[t][u][4 * q + 1], acc[t][u][4 * q + 2], acc[t][u][4 * q + 3]};
              i32x4* const to = sums + ((t * TM + u) * 4 + q) * 64;
              *to = p == 1 ? c : *to + c;
            }
      }
      __syncthreads();
    }
    if (kpart != 0) return;
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int u = 0; u < TM; ++u)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const i32x4 c = sums[((t * TM + u) * 4 + q) * 64];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[t][u][4 * q + e] += c[e];
        }
  }

#pragma unroll
  for (int u = 0; u < TM; ++u) {
    const int m = m0 + wm * WM + u * 32 + (lane & 31);
    if (m < a.rows) {
      const float scale = a.scales[m];
#pragma unroll
      for (int t = 0; t < TN; ++t) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const i32x4 c = {acc[t][u][4 * q], acc[t][u][4 * q + 1], acc[t][u][4 * q + 2], acc[t][u][4 * q + 3]};
          store_results<Fp32>(a, m, n0 + wn * WN + t * 32 + 8 * q + 4 * half, scale, c);
        }
        asm volatile("" ::: "memory");
      }
    }
  }
}

template <int BN, int BM, int WN, int WM, int K, int S>
static hipError_t launch_tiles(const MatmulRows& a, bool fp32, hipStream_t stream) {
  constexpr unsigned kThreads = BN / WN * (BM / WM) * K * 64;
  const int tiles_n = (a.n + BN - 1) / BN, tiles_m = (a.rows + BM - 1) / BM;
  return launch(fp32 ? matmul_tile_kernel<BN, BM, WN, WM, K, S, true> : matmul_tile_kernel<BN, BM, WN, WM, K, S, false>, dim3((unsigned)tiles_n * (unsigned)tiles_m),
                kThreads, stream, a, tiles_n, tiles_m);
}

template <int R, int W>
static hipError_t launch_few(const MatmulRows& a, bool fp32, hipStream_t stream) {
  return launch(fp32 ? matmul_few_kernel<R, W, true> : matmul_few_kernel<R, W, false>, dim3((a.n + 15) / 16), 64 * W, stream, a);
}

#ifdef HFX_PROBE
int g_variant = -1;
extern "C" void hfx_probe_variant(int v) { g_variant = v; }
static hipError_t probe(const MatmulRows& a, bool fp32, hipStream_t stream) {
  switch (g_variant) {
    case 0: return launch_few<1, 8>(a, fp32, stream);
    case 1: return launch_few<2, 8>(a, fp32, stream);
    case 2: return launch_few<4, 8>(a, fp32, stream);
    case 3: return launch_few<1, 16>(a, fp32, stream);
    case 4: return launch_few<1, 4>(a, fp32, stream);
    case 10: return launch_tiles<256, 256, 128, 64, 1, 2>(a, fp32, stream);
    case 11: return launch_tiles<256, 128, 64, 64, 1, 2>(a, fp32, stream);
    case 12: return launch_tiles<128, 128, 64, 32, 1, 2>(a, fp32, stream);
    case 13: return launch_tiles<128, 128, 64, 64, 1, 2>(a, fp32, stream);
    case 14: return launch_tiles<64, 64, 32, 32, 1, 4>(a, fp32, stream);
    case 15: return launch_tiles<64, 64, 32, 32, 2, 4>(a, fp32, stream);
    case 16: return launch_tiles<32, 64, 32, 32, 2, 4>(a, fp32, stream);
    case 17: return launch_tiles<32, 32, 32, 32, 4, 4>(a, fp32, stream);
    case 18: return launch_tiles<32, 32, 32, 32, 4, 8>(a, fp32, stream);
    case 19: return launch_tiles<64, 32, 32, 32, 2, 4>(a, fp32, stream);
    case 20: return launch_tiles<32, 64, 32, 64, 4, 6>(a, fp32, stream);
    case 21: return launch_tiles<64, 128, 32, 64, 1, 3>(a, fp32, stream);
    case 22: return launch_tiles<128, 256, 64, 64, 1, 2>(a, fp32, stream);
    case 23: return launch_tiles<256, 256, 64, 128, 1, 2>(a, fp32, stream);
    case 24: return launch_tiles<64, 64, 64, 64, 4, 4>(a, fp32, stream);
    case 25: return launch_tiles<64, 64, 32, 64, 4, 4>(a, fp32, stream);
    case 26: return launch_tiles<64, 128, 64, 64, 4, 3>(a, fp32, stream);
    case 27: return launch_tiles<128, 64, 64, 32, 2, 3>(a, fp32, stream);
    case 28: return launch_tiles<64, 128, 32, 64, 2, 3>(a, fp32, stream);
  }
  return hipErrorInvalidValue;
}
#endif

hipError_t launch_matmul_rows(const MatmulRows& a, bool fp32, hipStream_t stream) {
#ifdef HFX_PROBE
  if (g_variant >= 0) return probe(a, fp32, stream);
#endif
  if (a.rows <= 16) return launch_few<1, 8>(a, fp32, stream);
  if (a.rows <= 32) return launch_few<2, 8>(a, fp32, stream);
  if ((long)a.rows * a.n <= 64l * 64 * 512) return launch_tiles<64, 64, 32, 32, 1, 4>(a, fp32, stream);
  if ((long)a.rows * a.n <= 128l * 128 * 512) return launch_tiles<128, 128, 64, 32, 1, 2>(a, fp32, stream);
  return launch_tiles<256, 256, 128, 64, 1, 2>(a, fp32, stream);
}

}  // namespace hfx
