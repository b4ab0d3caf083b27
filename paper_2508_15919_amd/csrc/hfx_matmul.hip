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

// ... eight in bf16.
__device__ __forceinline__ void store_line(const MatmulRows& a, int m, int n, const u32x4& line) {
  __bf16* const row = static_cast<__bf16*>(a.out) + m * a.out_stride;
  if (a.past && n + 8 <= a.n) __builtin_nontemporal_store(line, reinterpret_cast<u32x4*>(row + n));
  else store_channels<8>(row, reinterpret_cast<const __bf16*>(&line), n, a.n);
}

// ---------------------------------------------------------------- few rows
// 16 N channels by 16 R rows to a workgroup, the sum cut into steps of 128 that its W wavefronts take in turn; both operands go straight to registers, U steps ahead.  A lane
// has 32 bytes in a row of a step, which two matrix instructions take one half each (any order of the values will do that is the same in both operands), so that
// four lanes ask for a whole line.
template <int N, int R, int W, int U, bool Fp32>
__global__ __launch_bounds__(64 * W) void matmul_few_kernel(const MatmulRows a, int tiles_n) {
  __shared__ i32x4 part[W][N * R][64];
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), r = lane & 15, j = lane >> 4;
  const int tile_m = uniform((int)blockIdx.x / tiles_n), tile_n = (int)blockIdx.x - tile_m * tiles_n, n0 = tile_n * 16 * N, m0 = tile_m * 16 * R;
  const int8_t *w[N], *x[R];
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = a.weight + (long)min(n0 + 16 * i + r, a.n - 1) * a.weight_stride;
#pragma unroll
  for (int i = 0; i < R; ++i) x[i] = a.codes + (long)min(m0 + 16 * i + r, a.rows - 1) * a.codes_stride;
  i32x4 acc[N][R] = {};
  i32x4 fw[U][N][2], fx[U][R][2];
  auto load = [&](int u, int s) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      int k = s * 128 + 32 * j + 16 * h;
      if (s * 128 + 128 > a.k) k = k < a.k ? k : 0;
#pragma unroll
      for (int i = 0; i < N; ++i) fw[u][i][h] = *reinterpret_cast<const i32x4*>(w[i] + k);
#pragma unroll
      for (int i = 0; i < R; ++i) fx[u][i][h] = *reinterpret_cast<const i32x4*>(x[i] + k);
    }
  };
  auto multiply = [&](int u, int s) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (s * 128 + 128 > a.k && s * 128 + 32 * j + 16 * h >= a.k) {
#pragma unroll
        for (int i = 0; i < R; ++i) fx[u][i][h] = i32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int q = 0; q < R; ++q) acc[i][q] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u][i][h], fx[u][q][h], acc[i][q], 0, 0, 0);
    }
  };
  const int steps = (a.k + 127) >> 7;
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (wave + u * W < steps) load(u, wave + u * W);
  for (int s = wave; s < steps; s += U * W) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s + u * W < steps) multiply(u, s + u * W);
      if (s + (u + U) * W < steps) load(u, s + (u + U) * W);
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int q = 0; q < R; ++q) part[wave][i * R + q][lane] = acc[i][q];
  __syncthreads();
  for (int b = wave; b < N * R; b += W) {
    const int m = m0 + 16 * (b % R) + r, n = n0 + 16 * (b / R) + 4 * j;
    i32x4 c = part[0][b][lane];
#pragma unroll
    for (int i = 1; i < W; ++i) c += part[i][b][lane];
    f32x4 weight_scale;
#pragma unroll
    for (int e = 0; e < 4; ++e) weight_scale[e] = a.weight_scales[min(n + e, a.n - 1)];
    if (m < a.rows) store_results<Fp32>(a, m, n, results(c, a.scales[m], weight_scale, a.bias, n, a.n - 1));
  }
}

// ---------------------------------------------------------------- tiles
// Tile `index` of a die's share.  Workgroups go to the dies by their number modulo 8; a die takes neighbouring tiles, four of the channels by as many rows as follow, so that
// those that its compute units work on together share what they read in its L2.
struct Tile {
  int n, m;
};
__device__ __forceinline__ Tile tile_at(int index, int tiles_n, int tiles_m) {
  constexpr int kBand = 4;
  const int band = index / (kBand * tiles_m), r = index - band * kBand * tiles_m, width = min(kBand, tiles_n - band * kBand);
  return {uniform(band * kBand + r % width), uniform(r / width)};      // (divisions leave the scalar unit)
}

// `p`, which is the same in all lanes, in scalar registers.
__device__ __forceinline__ const int8_t* uniform_address(const int8_t* p) {
  const uint64_t x = (uint64_t)p;
  return (const int8_t*)((uint64_t)(unsigned)uniform((int)(x >> 32)) << 32 | (unsigned)uniform((int)x));
}
// Copies 64 pieces of 16 bytes to LDS, lane after lane from `lds` on.
__device__ __forceinline__ void copy_to_lds(const int8_t* base, unsigned offset, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(offset), "s"(uniform_address(base)), "s"(uniform((int)lds)) : "memory", "m0");
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

  const int tile_m = uniform((int)(blockIdx.x / (unsigned)tiles_n)), tile_n = (int)blockIdx.x - tile_m * tiles_n;
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

// ---------------------------------------------------------------- large products
// A workgroup's BN channels by BM rows, tile after tile, WN by WM of them to a wavefront.  Stages of 128 values of the sum go straight from memory to LDS, into rings of RN places
// for the channels' and RM for the rows' part; a row's eight 16-byte pieces are permuted by bits 1 to 3 of its number, so that 16 lanes that read the same piece of
// 16 rows meet all banks.  The operands of 32 values are read while the matrix instructions of the 32 before them run.  The workgroup meets once a
// stage, ahead of the last of these, when all of the stage has been read: its places are then free for the copies of the stages RM and RN behind it.  These go on into the next tile, so
// that its first stages arrive while the results of this one leave.
template <int BN, int BM, int WN, int WM, int RN, int RM, bool Fp32>
__global__ __launch_bounds__(BN / WN * (BM / WM) * 64) void matmul_large_kernel(const MatmulRows a, int tiles_n, int tiles_m) {
  constexpr int kWaves = BN / WN * (BM / WM), TN = WN / 32, TM = WM / 32;
  constexpr int LN = (BN / 8 + kWaves - 1) / kWaves, LM = (BM / 8 + kWaves - 1) / kWaves;     // copy instructions of a wavefront: blocks of eight rows, the last one by several where they do not come out even
  constexpr int kRingM = RN * BN * 128, kAll = kRingM + RM * BM * 128, kEach = LN + LM;
  constexpr int kAhead = (RM - 2) * kEach + (RN > RM ? LN : 0);      // copies behind those of the next stage
  static_assert((RN == RM || RN == RM + 1) && RM >= 2 && kAll <= 160 * 1024, "");
  static_assert(TN == 1 || TN % 2 == 0, "");
  __shared__ __attribute__((aligned(1024))) char smem[kAll];
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  const int wn = wave % (BN / WN), wm = wave / (BN / WN);
  const unsigned lds0 = (unsigned)(uintptr_t)smem;
  const int stages = (a.k + 127) >> 7, whole = a.k >> 7, rest = a.k & 127;

  // this die's tiles, and this workgroup's among them
  const int die = (int)blockIdx.x & 7, tiles = tiles_n * tiles_m;
  const int first = die * (tiles >> 3) + min(die, tiles & 7), end = first + (tiles >> 3) + (die < (tiles & 7) ? 1 : 0), step = ((int)gridDim.x - die + 7) >> 3;
  int index = first + ((int)blockIdx.x >> 3);
  if (index >= end) return;
  Tile tile = tile_at(index, tiles_n, tiles_m);

  // A lane copies one piece of row lane / 8 of a block, the one that belongs in its place.  In a stage with fewer than 128 values the pieces behind them are piece 0 again.
  auto offset = [&](int block, int last, long stride, int values) {
    const int row = block * 8 + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
    return (unsigned)min(row, last) * (unsigned)stride + (unsigned)(piece * 16 < values ? piece * 16 : 0);
  };
  auto block_n = [&](int i) { return BN / 8 % kWaves == 0 ? wave + i * kWaves : min(wave + i * kWaves, BN / 8 - 1); };
  auto block_m = [&](int i) { return BM / 8 % kWaves == 0 ? wave + i * kWaves : min(wave + i * kWaves, BM / 8 - 1); };
  bool has_next = index + step < end;
  Tile next = has_next ? tile_at(index + step, tiles_n, tiles_m) : tile;
  const int total = uniform((end - index + step - 1) / step) * stages;      // stages of all of this workgroup's tiles

  // What is copied: the stages of both operands in a row, those of the next tile behind those of this one.
  const int8_t *from_n = a.weight + (long)tile.n * BN * a.weight_stride, *from_m = a.codes + (long)tile.m * BM * a.codes_stride;
  int at_stage_n = 0, at_stage_m = 0, left_n = total, left_m = total;
  bool ahead_n = false, ahead_m = false;           // in the next tile already
  unsigned off_n[LN], off_m[LM];
  auto offsets_n = [&](int n, int values) {
#pragma unroll
    for (int i = 0; i < LN; ++i) off_n[i] = offset(block_n(i), a.n - 1 - n * BN, a.weight_stride, values);
  };
  auto offsets_m = [&](int m, int values) {
#pragma unroll
    for (int i = 0; i < LM; ++i) off_m[i] = offset(block_m(i), a.rows - 1 - m * BM, a.codes_stride, values);
  };
  offsets_n(tile.n, whole > 0 ? 128 : rest);
  offsets_m(tile.m, whole > 0 ? 128 : rest);
  auto advance_n = [&] {
    --left_n;
    from_n += 128;
    if (++at_stage_n == stages) {
      at_stage_n = 0;
      ahead_n = true;
      from_n = a.weight + (long)next.n * BN * a.weight_stride;
      offsets_n(next.n, whole > 0 ? 128 : rest);
    } else if (at_stage_n == whole) {
      offsets_n(ahead_n ? next.n : tile.n, rest);
    }
  };
  auto advance_m = [&] {
    --left_m;
    from_m += 128;
    if (++at_stage_m == stages) {
      at_stage_m = 0;
      ahead_m = true;
      from_m = a.codes + (long)next.m * BM * a.codes_stride;
      offsets_m(next.m, whole > 0 ? 128 : rest);
    } else if (at_stage_m == whole) {
      offsets_m(ahead_m ? next.m : tile.m, rest);
    }
  };
  auto advance = [&] {
    advance_m();
    advance_n();
  };
  // Copy instruction i of a set (the rows' part of a stage, then the channels'): behind a matrix instruction of its own, from the last phase of the stage whose places it fills to the
  // third phase of the one after it, so that the copies of the wavefronts do not wait for each other.
  constexpr auto position = [](int i) { return i * (4 * TN * TM) / kEach; };
  auto copy = [&](int i, int slot_n, int slot_m) {
    if (i < LM) {
      if (left_m > 0) copy_to_lds(from_m, off_m[i < LM ? i : 0], lds0 + kRingM + slot_m * (BM * 128) + block_m(i) * 1024);
    } else {
      if (left_n > 0) copy_to_lds(from_n, off_n[i < LM ? 0 : i - LM], lds0 + slot_n * (BN * 128) + block_n(i - LM) * 1024);
    }
  };

  i32x16 acc[TN][TM];
  struct Operands {
    i32x4 n[TN], m[TM];
  };
  const int swizzle = (lane >> 1) & 7, half = lane >> 5;
  const int at_n = (wn * WN + (lane & 31)) * 128, at_m = kRingM + (wm * WM + (lane & 31)) * 128;
  auto read = [&](Operands& f, int slot_n, int slot_m, int kk) {
    const int piece = ((2 * kk + half) ^ swizzle) * 16;
    const char *const from_n = smem + slot_n * (BN * 128) + at_n + piece, *const from_m = smem + slot_m * (BM * 128) + at_m + piece;
#pragma unroll
    for (int t = 0; t < TN; ++t) f.n[t] = *reinterpret_cast<const i32x4*>(from_n + t * 4096);
#pragma unroll
    for (int t = 0; t < TM; ++t) f.m[t] = *reinterpret_cast<const i32x4*>(from_m + t * 4096);
  };

  // The first sets, the last of them up to where the loop goes on with it; ahead of them n(0), where the rings differ.
  int g = 0, slot_n = 0, slot_m = 0, before_n = RN - 1, before_m = RM - 1;      // stage, its places, those of the stage before
  auto begin_set = [&] {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (position(i) < TN * TM) copy(i, before_n, before_m);
  };
  constexpr int kBegun = [] {
    int n = 0;
    for (int i = 0; i < kEach; ++i) n += i * (4 * TN * TM) / kEach < TN * TM;
    return n;
  }();
  if constexpr (RN > RM) {
#pragma unroll
    for (int i = LM; i < kEach; ++i) copy(i, 0, 0);
    advance_n();
  }
#pragma unroll
  for (int r = 0; r < RM - 1; ++r) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) copy(i, r + RN - RM, r);
    advance();
  }
  begin_set();
  if (total >= RN) HFX_WAIT_VMCNT(kAhead + kBegun);
  else HFX_WAIT_VMCNT(0);
  ring_barrier();
  Operands f[2];
  read(f[0], 0, 0, 0);

  float row_scale[TM], weight_scale[(TN + 1) / 2], bias[(TN + 1) / 2];
  // A stage; `final`: the tile's last one, whose places are left to the results.
  auto stage = [&](auto final) {
    constexpr bool kFinal = decltype(final)::value;
    const int then_n = slot_n == RN - 1 ? 0 : slot_n + 1, then_m = slot_m == RM - 1 ? 0 : slot_m + 1;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      Operands &now = f[p & 1], &then = f[(p + 1) & 1];
      if (p < 3) {
        read(then, slot_n, slot_m, p + 1);
      } else {
        if (!kFinal || has_next) {
          if (g - 1 + RN < total) HFX_WAIT_VMCNT(kAhead);
          else HFX_WAIT_VMCNT(0);
          ring_barrier();
          read(then, then_n, then_m, 0);
        }
        if constexpr (!kFinal) advance();
      }
      if constexpr (kFinal) {
        if (rest != 0) {                            // the sum ends inside this stage: rows count as zero behind it
          const int keep = (2 * p + half) * 16 < rest ? -1 : 0;
#pragma unroll
          for (int u = 0; u < TM; ++u) now.m[u] &= i32x4{keep, keep, keep, keep};
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int u = 0; u < TM; ++u) {
          acc[t][u] = __builtin_amdgcn_mfma_i32_32x32x32_i8(now.n[t], now.m[u], acc[t][u], 0, 0, 0);
          if (p < 3 || !kFinal) {
#pragma unroll
            for (int i = 0; i < kEach; ++i)
              if (position(i) == (p + 1) % 4 * TN * TM + t * TM + u) {
                copy(i, p == 3 ? slot_n : before_n, p == 3 ? slot_m : before_m);
                __builtin_amdgcn_sched_barrier(0);
              }
          }
        }
      __builtin_amdgcn_sched_barrier(0);
    }
    before_n = slot_n;
    before_m = slot_m;
    slot_n = then_n;
    slot_m = then_m;
  };

  while (true) {
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int u = 0; u < TM; ++u) acc[t][u] = i32x16{};
    for (int s = 1; s < stages; ++s) {
      stage(std::false_type());
      ++g;
    }
    const int n1 = tile.n * BN + wn * WN, m1 = tile.m * BM + wm * WM;
#pragma unroll
    for (int u = 0; u < TM; ++u) row_scale[u] = a.scales[min(m1 + u * 32 + (lane & 31), a.rows - 1)];
#pragma unroll
    for (int t = 0; t < (TN + 1) / 2; ++t) {
      const int n = min(n1 + t * 64 + (TN == 1 ? lane & 31 : lane), a.n - 1);
      weight_scale[t] = a.weight_scales[n];
      bias[t] = a.bias ? __builtin_bit_cast(float, (unsigned)a.bias[n] << 16) : 0.0f;
    }
    stage(std::true_type());
    if (!has_next) ring_barrier();

    // Results.  The last stage's places are free: in the smaller one lie the channels' scales and biases of each wavefront; through the other results leave in rows, 64
    // channels at a time (a lane has four channels of its row).  Pieces of 16 bytes are permuted by the row, and their halves change places in
    // rows 16 to 31, so that all banks are met.
    constexpr int kWide = TN == 1 ? 32 : 64, kPieces = kWide / 8, kShare = 256 / (2 * kWide), kAtOnce = 64 / kPieces;
    static_assert(kWaves * 32 * kWide * 2 <= std::max(BN, BM) * 128 && kWaves * WN * 8 <= std::min(BN, BM) * 128, "");
    char *const place_n = smem + before_n * (BN * 128), *const place_m = smem + kRingM + before_m * (BM * 128);
    float* const channel = reinterpret_cast<float*>(BN >= BM ? place_m : place_n) + wave * (2 * WN);
    char* const box = (BN >= BM ? place_n : place_m) + wave * (32 * kWide * 2);
#pragma unroll
    for (int t = 0; t < (TN + 1) / 2; ++t) {
      const int c = t * 64 + (TN == 1 ? lane & 31 : lane);
      channel[c] = weight_scale[t];
      channel[WN + c] = bias[t];
    }
    const int row = lane & 31;
    char* const to = box + row * (2 * kWide) + (half ^ (row >> 4)) * 8;
#pragma unroll
    for (int u = 0; u < TM; ++u)
#pragma unroll
      for (int t2 = 0; t2 < TN; t2 += kWide / 32) {
#pragma unroll
        for (int t = t2; t < t2 + kWide / 32; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
#pragma clang fp contract(off)
            const int c = t * 32 + 8 * q + 4 * half;
            const f32x4 w = *reinterpret_cast<const f32x4*>(channel + c);
            f32x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (float)acc[t][u][4 * q + e] * row_scale[u] * w[e];
            if (a.bias) y += *reinterpret_cast<const f32x4*>(channel + WN + c);
            if constexpr (Fp32) {
              const int m = m1 + u * 32 + row;
              if (m < a.rows) store_results<true>(a, m, n1 + c, y);
            } else {
              *reinterpret_cast<bf16x4*>(to + (((t - t2) * 4 + q) ^ (row / kShare & (kPieces - 1))) * 16) = rounded(y);
            }
          }
        if constexpr (!Fp32) {
#pragma unroll
          for (int i = 0; i < 32 / kAtOnce; ++i) {
            const int r = i * kAtOnce + lane / kPieces, piece = lane % kPieces, m = m1 + u * 32 + r;
            u32x4 line = *reinterpret_cast<const u32x4*>(box + r * (2 * kWide) + (piece ^ (r / kShare & (kPieces - 1))) * 16);
            if (r >= 16) line = u32x4{line[2], line[3], line[0], line[1]};
            if (m < a.rows) store_line(a, m, n1 + t2 * 32 + piece * 8, line);
          }
        }
        asm volatile("" ::: "memory");
      }
    if (!has_next) return;
    ring_barrier();                                 // every wavefront's results have left the places
    advance();
    begin_set();
    ++g;
    index += step;
    tile = next;
    ahead_n = ahead_m = false;
    has_next = index + step < end;
    if (has_next) next = tile_at(index + step, tiles_n, tiles_m);
  }
}

template <int BN, int BM, int WN, int WM, int RN, int RM>
static hipError_t launch_large(const MatmulRows& a, bool fp32, hipStream_t stream) {
  constexpr int kUnits = 256 * (160 * 1024 / (RN * BN * 128 + RM * BM * 128));
  const int tiles_n = (a.n + BN - 1) / BN, tiles_m = (a.rows + BM - 1) / BM, tiles = tiles_n * tiles_m;
  // (the copies of a tile go on into the next one, not past it)
  const int grid = (a.k + 127) / 128 < RN ? tiles : std::min(tiles, kUnits);
  return launch(fp32 ? matmul_large_kernel<BN, BM, WN, WM, RN, RM, true> : matmul_large_kernel<BN, BM, WN, WM, RN, RM, false>, dim3((unsigned)grid), BN / WN * (BM / WM) * 64, stream, a,
                tiles_n, tiles_m);
}

template <int BN, int BM, int WN, int WM, int K, int B, int S>
static hipError_t launch_tiles(const MatmulRows& a, bool fp32, hipStream_t stream) {
  constexpr unsigned kThreads = BN / WN * (BM / WM) * K * 64;
  const int tiles_n = (a.n + BN - 1) / BN, tiles_m = (a.rows + BM - 1) / BM;
  return launch(fp32 ? matmul_tile_kernel<BN, BM, WN, WM, K, B, S, true> : matmul_tile_kernel<BN, BM, WN, WM, K, B, S, false>, dim3((unsigned)tiles_n * (unsigned)tiles_m),
                kThreads, stream, a, tiles_n, tiles_m);
}

template <int N, int R, int W, int U>
static hipError_t launch_few(const MatmulRows& a, bool fp32, hipStream_t stream) {
  const int tiles_n = (a.n + 16 * N - 1) / (16 * N), tiles_m = (a.rows + 16 * R - 1) / (16 * R);
  return launch(fp32 ? matmul_few_kernel<N, R, W, U, true> : matmul_few_kernel<N, R, W, U, false>, dim3((unsigned)tiles_n * (unsigned)tiles_m), 64 * W, stream, a, tiles_n);
}

#ifdef HFX_PROBE
int g_variant = -1;
extern "C" void hfx_probe_variant(int v) { g_variant = v; }
static hipError_t probe(const MatmulRows& a, bool fp32, hipStream_t stream) {
  switch (g_variant) {
    case 2: return launch_tiles<32, 64, 32, 32, 2, 128, 6>(a, fp32, stream);
    case 3: return launch_tiles<64, 64, 32, 32, 1, 128, 4>(a, fp32, stream);
    case 4: return launch_tiles<128, 128, 64, 32, 1, 128, 2>(a, fp32, stream);
    case 5: return launch_large<128, 128, 32, 64, 4, 4>(a, fp32, stream);
    case 6: return launch_large<256, 128, 64, 64, 3, 3>(a, fp32, stream);
    case 8: return launch_large<256, 160, 32, 160, 3, 3>(a, fp32, stream);
    case 9: return launch_large<256, 192, 64, 96, 3, 2>(a, fp32, stream);
    case 10: return launch_large<256, 256, 64, 128, 3, 2>(a, fp32, stream);
    case 13: return launch_tiles<64, 128, 32, 64, 1, 128, 3>(a, fp32, stream);
    case 15: return launch_few<1, 1, 16, 2>(a, fp32, stream);
    case 16: return launch_tiles<32, 32, 32, 32, 4, 128, 6>(a, fp32, stream);
    case 17: return launch_tiles<64, 64, 32, 32, 1, 128, 3>(a, fp32, stream);
    case 18: return launch_tiles<32, 64, 32, 32, 2, 128, 4>(a, fp32, stream);
    case 19: return launch_tiles<32, 32, 32, 32, 4, 128, 4>(a, fp32, stream);
    case 20: return launch_tiles<128, 64, 64, 32, 1, 128, 2>(a, fp32, stream);
    case 21: return launch_tiles<64, 128, 32, 64, 1, 128, 2>(a, fp32, stream);
    case 22: return launch_tiles<128, 128, 64, 64, 1, 128, 2>(a, fp32, stream);
    case 23: return launch_tiles<64, 64, 64, 32, 1, 128, 4>(a, fp32, stream);
    case 24: return launch_tiles<64, 64, 64, 64, 4, 128, 4>(a, fp32, stream);
    case 25: return launch_tiles<64, 64, 32, 64, 2, 128, 4>(a, fp32, stream);
  }
  return hipErrorInvalidValue;
}
#endif

hipError_t launch_matmul_rows(MatmulRows a, bool fp32, hipStream_t stream) {
  a.past = !fp32 && a.out_stride % 8 == 0 && 2l * a.rows * a.n > (64l << 20);
#ifdef HFX_PROBE
  if (g_variant >= 0) return probe(a, fp32, stream);
#endif
  if (a.rows <= 16) return launch_few<1, 1, 8, 4>(a, fp32, stream);
  if (a.rows <= 32) return launch_few<1, 2, 8, 4>(a, fp32, stream);
  if ((long)a.rows * a.n <= 64l * 64 * 512) return launch_tiles<64, 64, 32, 32, 1, 128, 4>(a, fp32, stream);
  if ((long)a.rows * a.n <= 128l * 128 * 512) return launch_tiles<128, 128, 64, 32, 1, 128, 2>(a, fp32, stream);
  return launch_large<256, 256, 64, 128, 3, 2>(a, fp32, stream);
}

}  // namespace hfx
