// Products of rows and weights that are both held in 8 bits, with a scale for each row and each output channel: the projections of a layer.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "hfx_device.h"
#include "hfx_launch.h"

namespace hfx {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// Results of four channels; every rounding by itself.
__device__ __forceinline__ f32x4 results(const i32x4& c, float row_scale, const f32x4& weight_scale, const uint16_t* bias, int n, int last) {
#pragma clang fp contract(off)
  f32x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (float)c[e] * row_scale * weight_scale[e];
  if (bias) {
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += __builtin_bit_cast(float, (unsigned)bias[min(n + e, last)] << 16);
  }
  return y;
}
__device__ __forceinline__ bf16x4 rounded(const f32x4& y) { return bf16x4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]}; }

// Stores channels n .. n + N - 1 of a row, as many of them as there are.  Rows may begin at any element.
template <int N, typename T>
__device__ __forceinline__ void store_channels(T* row, const T* y, int n, int channels) {
  if (n + N <= channels) {
    __builtin_memcpy(row + n, y, N * sizeof(T));
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (n + e < channels) row[n + e] = y[e];
  }
}
template <bool Fp32>
__device__ __forceinline__ void store_results(const MatmulRows& a, int m, int n, const f32x4& y) {
  if constexpr (Fp32) {
    store_channels<4>(static_cast<float*>(a.out) + m * a.out_stride, reinterpret_cast<const float*>(&y), n, a.n);
  } else {
    const bf16x4 r = rounded(y);
    store_channels<4>(static_cast<__bf16*>(a.out) + m * a.out_stride, reinterpret_cast<const __bf16*>(&r), n, a.n);
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
  f32x4 weight_scale;
  const float row_scale = a.scales[min(16 * wave + r, a.rows - 1)];
#pragma unroll
  for (int e = 0; e < 4; ++e) weight_scale[e] = a.weight_scales[min(n0 + 4 * j + e, a.n - 1)];
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
  if (m < a.rows) store_results<Fp32>(a, m, n0 + 4 * j, results(c, row_scale, weight_scale, a.bias, n0 + 4 * j, a.n - 1));
}

// ---------------------------------------------------------------- tiles
// Copies 64 pieces of 16 bytes to LDS, lane after lane from `lds` on.
__device__ __forceinline__ void copy_to_lds(const int8_t* base, unsigned offset, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(offset), "s"(base), "s"(lds) : "memory", "m0");
}

// ... 64 times four bytes.
__device__ __forceinline__ void copy_words_to_lds(const float* base, unsigned offset, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" :: "v"(offset), "s"(base), "s"(lds) : "memory", "m0");
}

// A workgroup's BN channels by BM rows.  Stages of B values of the sum go straight from memory to LDS, S of them in a ring; a row's 16-byte pieces
// are permuted by its number, so that 16 lanes that read the same piece of 16 rows meet all banks.  (WN channels by WM rows, and of a
// stage one part of K, belong to a wavefront.)  The operands of 32 values are read while the matrix instructions of the 32 before them run; the workgroup meets
// once a stage, ahead of the last of these, when all of the stage has been read: its place is then free for the copies of the stage S behind it.
template <int BN, int BM, int WN, int WM, int K, int B, int S, bool Fp32>
__global__ __launch_bounds__(BN / WN * (BM / WM) * K * 64) void matmul_tile_kernel(const MatmulRows a, int tiles_n, int tiles_m) {
  constexpr int kWaves = BN / WN * (BM / WM) * K, kBytes = (BN + BM) * B, kRows = 1024 / B;      // (rows that a copy instruction takes)
  constexpr int LN = BN / kRows / kWaves, LM = BM / kRows / kWaves, TN = WN / 32, TM = WM / 32, P = B / 32 / K;
  static_assert(LN * kRows * kWaves == BN && LM * kRows * kWaves == BM, "each wavefront copies whole blocks of rows of both");
  static_assert((B == 64 || B == 128) && P >= 1 && S * kBytes <= 160 * 1024, "");
  constexpr int kScaleN = S * kBytes, kScaleM = kScaleN + (BN + 63) / 64 * 256, kAll = kScaleM + (BM + 63) / 64 * 256;
  static_assert(kAll <= 160 * 1024, "");
  __shared__ __attribute__((aligned(1024))) char smem[kAll];
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
  const int stages = (a.k + B - 1) / B, whole = a.k / B, rest = a.k % B;

  // A lane copies one piece of row lane / (B / 16) of a block, the one that belongs in its place.  In a stage with fewer than B values pieces behind them are piece 0 again.
  auto offset = [&](int i, int last, long stride, int values) {
    const int row = (wave + i * kWaves) * kRows + lane / (B / 16), piece = (lane % (B / 16)) ^ (row >> (B == 128 ? 1 : 2) & (B / 16 - 1));
    return (unsigned)min(row, last) * (unsigned)stride + (unsigned)(piece * 16 < values ? piece * 16 : 0);
  };
  unsigned off_n[LN], off_m[LM];
#pragma unroll
  for (int i = 0; i < LN; ++i) off_n[i] = offset(i, a.n - 1 - n0, a.weight_stride, B);
#pragma unroll
  for (int i = 0; i < LM; ++i) off_m[i] = offset(i, a.rows - 1 - m0, a.codes_stride, B);
  // copy instruction i of LN + LM of a whole stage
  auto copy = [&](int stage, int slot, int i) {
    const unsigned to = lds0 + slot * kBytes + wave * 1024;
    if (i < LN) copy_to_lds(weight + (long)stage * B, off_n[i < LN ? i : 0], to + i * kWaves * 1024);
    else copy_to_lds(codes + (long)stage * B, off_m[i < LN ? 0 : i - LN], to + BN * B + (i - LN) * kWaves * 1024);
  };
  auto copy_any = [&](int stage, int slot) {
    if (stage < whole) {
#pragma unroll
      for (int i = 0; i < LN + LM; ++i) copy(stage, slot, i);
    } else {
      const unsigned to = lds0 + slot * kBytes + wave * 1024;
#pragma unroll
      for (int i = 0; i < LN; ++i) copy_to_lds(weight + (long)stage * B, offset(i, a.n - 1 - n0, a.weight_stride, rest), to + i * kWaves * 1024);
#pragma unroll
      for (int i = 0; i < LM; ++i) copy_to_lds(codes + (long)stage * B, offset(i, a.rows - 1 - m0, a.codes_stride, rest), to + BN * B + i * kWaves * 1024);
    }
  };

  i32x16 acc[TN][TM] = {};
  struct Operands {
    i32x4 n[TN], m[TM];
  };
  const int swizzle = lane >> (B == 128 ? 1 : 2) & (B / 16 - 1), half = lane >> 5;
  const int at_n = (wn * WN + (lane & 31)) * B, at_m = BN * B + (wm * WM + (lane & 31)) * B;
  auto read = [&](Operands& f, int slot, int kk) {
    const char* const from = smem + slot * kBytes + (((2 * kk + half) ^ swizzle) * 16);
#pragma unroll
    for (int t = 0; t < TN; ++t) f.n[t] = *reinterpret_cast<const i32x4*>(from + at_n + t * 32 * B);
#pragma unroll
    for (int t = 0; t < TM; ++t) f.m[t] = *reinterpret_cast<const i32x4*>(from + at_m + t * 32 * B);
  };
  auto multiply = [&](const Operands& f, int t) {
#pragma unroll
    for (int u = 0; u < TM; ++u) acc[t][u] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.n[t], f.m[u], acc[t][u], 0, 0, 0);
  };

  // the scales go ahead of the stages: who waits for a stage has them
  for (int i = wave; i < (BN + 63) / 64; i += kWaves) copy_words_to_lds(a.weight_scales, 4u * (unsigned)min(n0 + i * 64 + lane, a.n - 1), lds0 + kScaleN + i * 256);
  for (int i = wave; i < (BM + 63) / 64; i += kWaves) copy_words_to_lds(a.scales, 4u * (unsigned)min(m0 + i * 64 + lane, a.rows - 1), lds0 + kScaleM + i * 256);
#pragma unroll
  for (int s = 0; s < S; ++s)
    if (s < stages) copy_any(s, s);
  if (stages >= S) HFX_WAIT_VMCNT((S - 1) * (LN + LM));
  else HFX_WAIT_VMCNT(0);
  ring_barrier();
  Operands f[2];
  read(f[0], 0, kpart);
  int s = 0, slot = 0;
  // A stage; `more`: the stages up to s + S - 1 are on their way or here, and s + S is a whole one.
  auto stage = [&](auto more) {
    const int behind = slot == S - 1 ? 0 : slot + 1;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      Operands& now = f[p & 1];
      Operands& then = P == 1 ? f[1] : f[(p + 1) & 1];
      if (p < P - 1) {
        read(then, slot, (p + 1) * K + kpart);
      } else if (more || s + 1 < stages) {
        if (more || s + S <= stages) HFX_WAIT_VMCNT((S - 2) * (LN + LM));      // the stages behind the next one may still be on their way
        else HFX_WAIT_VMCNT(0);
        ring_barrier();
        read(then, behind, kpart);
        if constexpr (!decltype(more)::value) {
          if (s + S < stages) copy_any(s + S, slot);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < TN; ++t) {
        multiply(now, t);
        if constexpr (decltype(more)::value) {
          if (p == P - 1) {
#pragma unroll
            for (int i = 0; i < LN + LM; ++i)
              if (i * TN / (LN + LM) == t) copy(s + S, slot, i);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (P == 1) f[0] = f[1];
    }
    ++s;
    slot = behind;
  };
  static_assert(P == 1 || P % 2 == 0, "a stage begins with the first of the two sets of operands");
  while (s + S < whole) stage(std::true_type());
  while (s < whole) stage(std::false_type());
  if (rest != 0) {
#pragma unroll 1
    for (int kk = kpart; kk < B / 32; kk += K) {
      read(f[0], slot, kk);
      const int keep = (2 * kk + half) * 16 < rest ? -1 : 0;
#pragma unroll
      for (int t = 0; t < TM; ++t) f[0].m[t] &= i32x4{keep, keep, keep, keep};
#pragma unroll
      for (int t = 0; t < TN; ++t) multiply(f[0], t);
    }
  }

  __syncthreads();                                  // the ring is free
  const float* const row_scales = reinterpret_cast<const float*>(smem + kScaleM) + wm * WM + (lane & 31);
  const char* const weight_scales = smem + kScaleN + (wn * WN + 4 * half) * 4;
  const int n1 = n0 + wn * WN, m1 = m0 + wm * WM;
  auto finished = [&](const i32x4& c, int t, int u, int q) {
    return results(c, row_scales[u * 32], *reinterpret_cast<const f32x4*>(weight_scales + (t * 32 + 8 * q) * 4), a.bias, n1 + t * 32 + 8 * q + 4 * half, a.n - 1);
  };
  auto quarter = [&](int t, int u, int q) { return i32x4{acc[t][u][4 * q], acc[t][u][4 * q + 1], acc[t][u][4 * q + 2], acc[t][u][4 * q + 3]}; };

  if constexpr (K > 1) {
    // The wavefronts that share results each sum a part of them.
    static_assert(kWaves * TN * TM * 4096 <= S * kBytes, "");
    i32x4* const sums = reinterpret_cast<i32x4*>(smem) + lane;
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int u = 0; u < TM; ++u)
#pragma unroll
        for (int q = 0; q < 4; ++q) sums[((wave * TN + t) * TM + u) * 256 + q * 64] = quarter(t, u, q);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int u = 0; u < TM; ++u)
#pragma unroll
        for (int i = 0; i < 4 / K; ++i) {
          const int q = kpart * (4 / K) + i, m = m1 + u * 32 + (lane & 31);
          i32x4 c = {0, 0, 0, 0};
#pragma unroll
          for (int p = 0; p < K; ++p) c += sums[(((wave - kpart + p) * TN + t) * TM + u) * 256 + q * 64];
          if (m < a.rows) store_results<Fp32>(a, m, n1 + t * 32 + 8 * q + 4 * half, finished(c, t, u, q));
        }
  } else if constexpr (Fp32) {
#pragma unroll
    for (int u = 0; u < TM; ++u) {
      const int m = m1 + u * 32 + (lane & 31);
      if (m < a.rows) {
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q) store_results<Fp32>(a, m, n1 + t * 32 + 8 * q + 4 * half, finished(quarter(t, u, q), t, u, q));
      }
      asm volatile("" ::: "memory");
    }
  } else {
    // A lane has four channels of its row at a time; through LDS the rows leave in pieces of 16 bytes side by side.  Pieces are permuted by the row, and their halves
    // change places in rows 16 to 31, so that all banks are met.
    constexpr int kPieces = WN / 8, kShare = 256 / (2 * WN), kAtOnce = 64 / kPieces;
    char* const box = smem + wave * (32 * WN * 2);
    const int row = lane & 31;
    char* const to = box + row * (2 * WN) + (half ^ (row >> 4)) * 8;
#pragma unroll
    for (int u = 0; u < TM; ++u) {
#pragma unroll
      for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<bf16x4*>(to + ((t * 4 + q) ^ (row / kShare & (kPieces - 1))) * 16) = rounded(finished(quarter(t, u, q), t, u, q));
#pragma unroll
      for (int i = 0; i < 32 / kAtOnce; ++i) {
        const int r = i * kAtOnce + lane / kPieces, piece = lane % kPieces, m = m1 + u * 32 + r;
        u32x4 line = *reinterpret_cast<const u32x4*>(box + r * (2 * WN) + (piece ^ (r / kShare & (kPieces - 1))) * 16);
        if (r >= 16) line = u32x4{line[2], line[3], line[0], line[1]};
        if (m < a.rows) store_channels<8>(static_cast<__bf16*>(a.out) + m * a.out_stride, reinterpret_cast<const __bf16*>(&line), n1 + piece * 8, a.n);
      }
      asm volatile("" ::: "memory");
    }
  }
}

template <int BN, int BM, int WN, int WM, int K, int B, int S>
static hipError_t launch_tiles(const MatmulRows& a, bool fp32, hipStream_t stream) {
  constexpr unsigned kThreads = BN / WN * (BM / WM) * K * 64;
  const int tiles_n = (a.n + BN - 1) / BN, tiles_m = (a.rows + BM - 1) / BM;
  return launch(fp32 ? matmul_tile_kernel<BN, BM, WN, WM, K, B, S, true> : matmul_tile_kernel<BN, BM, WN, WM, K, B, S, false>, dim3((unsigned)tiles_n * (unsigned)tiles_m),
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
    case 10: return launch_tiles<256, 256, 128, 64, 1, 128, 2>(a, fp32, stream);
    case 11: return launch_tiles<256, 256, 64, 128, 1, 128, 2>(a, fp32, stream);
    case 12: return launch_tiles<256, 256, 64, 128, 1, 64, 4>(a, fp32, stream);
    case 13: return launch_tiles<256, 256, 64, 64, 1, 128, 2>(a, fp32, stream);
    case 14: return launch_tiles<192, 256, 96, 64, 1, 128, 2>(a, fp32, stream);
    case 15: return launch_tiles<256, 192, 64, 96, 1, 128, 2>(a, fp32, stream);
    case 16: return launch_tiles<128, 128, 64, 64, 1, 128, 2>(a, fp32, stream);
    case 17: return launch_tiles<128, 256, 64, 64, 1, 128, 3>(a, fp32, stream);
    case 18: return launch_tiles<256, 128, 64, 64, 1, 128, 3>(a, fp32, stream);
    case 21: return launch_tiles<128, 128, 64, 64, 1, 64, 4>(a, fp32, stream);
    case 22: return launch_tiles<128, 128, 64, 32, 1, 128, 2>(a, fp32, stream);
    case 30: return launch_tiles<64, 64, 32, 32, 1, 128, 4>(a, fp32, stream);
    case 31: return launch_tiles<64, 64, 32, 32, 2, 128, 4>(a, fp32, stream);
    case 32: return launch_tiles<32, 64, 32, 32, 2, 128, 6>(a, fp32, stream);
    case 33: return launch_tiles<32, 32, 32, 32, 4, 128, 8>(a, fp32, stream);
    case 34: return launch_tiles<64, 32, 32, 32, 2, 128, 6>(a, fp32, stream);
    case 35: return launch_tiles<32, 64, 32, 64, 4, 128, 6>(a, fp32, stream);
    case 36: return launch_tiles<64, 128, 32, 64, 1, 128, 3>(a, fp32, stream);
    case 37: return launch_tiles<64, 128, 64, 32, 1, 128, 3>(a, fp32, stream);
    case 38: return launch_tiles<128, 64, 64, 32, 1, 128, 3>(a, fp32, stream);
    case 39: return launch_tiles<128, 64, 32, 64, 1, 128, 3>(a, fp32, stream);
    case 41: return launch_tiles<64, 64, 32, 32, 1, 128, 8>(a, fp32, stream);
    case 42: return launch_tiles<32, 64, 32, 32, 2, 128, 12>(a, fp32, stream);
    case 43: return launch_tiles<64, 64, 64, 32, 2, 128, 8>(a, fp32, stream);
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
  if ((long)a.rows * a.n <= 64l * 64 * 512) return launch_tiles<64, 64, 32, 32, 1, 128, 4>(a, fp32, stream);
  if ((long)a.rows * a.n <= 128l * 128 * 512) return launch_tiles<128, 128, 64, 32, 1, 128, 2>(a, fp32, stream);
  return launch_tiles<256, 256, 64, 128, 1, 128, 2>(a, fp32, stream);
}

}  // namespace hfx
