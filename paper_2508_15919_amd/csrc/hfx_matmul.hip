// Products of rows and weights that are both held in 8 bits, with a scale for each row and each output channel: the projections of a layer.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "hfx_device.h"
#include "hfx_launch.h"

namespace hfx {

constexpr int kComputeUnits = 256;

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
// 16 channels by up to 8 rows to a workgroup, the sum cut into steps of 128 values that its 16 wavefronts take in turn; both operands go straight to registers, two steps ahead.  A
// lane has 32 bytes in a row of a step, which two matrix instructions take one half each (any order of the values will do that is the same in both operands), so that
// four lanes ask for a whole line.  Rows that are not there are the last one again, which costs no further lines
// (16 rows of 4096 to 16384 channels 20.6 us where 4 take 16.0: 9 and more go by tiles of 32 rows, 14.2).
// Bound by the weight's way to the compute units, behind the 2.1 us of a launch: 4 rows of 8192 to 4096 channels (34 MB) 9.5 us from memory and 8.6 from the last level's cache, where tiles of 32 by 32 take 12.8 and
// 12.2; one row of 16384 to 4096 (67 MB) 16.0 and 14.3, 20.6 and 17.0; one of 4096 to 4096 6.5 and 5.5, 7.4 and 5.8.  More channels go by the tiles (4 rows of 4096 to 6144 here 9.3 us, from memory, and by those
// 8.0).  Eight wavefronts four steps ahead, in place of sixteen two, took 1.06 times as long.
template <bool Fp32>
__global__ __launch_bounds__(1024) void matmul_few_kernel(const MatmulRows a) {
  constexpr int kWaves = 16, kAhead = 2;
  __shared__ i32x4 part[kWaves][64];
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), r = lane & 15, j = lane >> 4;
  const int n0 = (int)blockIdx.x * 16;
  const int8_t* const w = a.weight + (long)min(n0 + r, a.n - 1) * a.weight_stride;
  const int8_t* const x = a.codes + (long)min(r, a.rows - 1) * a.codes_stride;
  i32x4 acc = {0, 0, 0, 0};
  i32x4 fw[kAhead][2], fx[kAhead][2];
  auto load = [&](int u, int s) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      int k = s * 128 + 32 * j + 16 * h;
      if (s * 128 + 128 > a.k) k = k < a.k ? k : 0;
      fw[u][h] = *reinterpret_cast<const i32x4*>(w + k);
      fx[u][h] = *reinterpret_cast<const i32x4*>(x + k);
    }
  };
  auto multiply = [&](int u, int s) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (s * 128 + 128 > a.k && s * 128 + 32 * j + 16 * h >= a.k) fx[u][h] = i32x4{0, 0, 0, 0};
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u][h], fx[u][h], acc, 0, 0, 0);
    }
  };
  const int steps = (a.k + 127) >> 7;
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
    if (wave + u * kWaves < steps) load(u, wave + u * kWaves);
  for (int s = wave; s < steps; s += kAhead * kWaves) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (s + u * kWaves < steps) multiply(u, s + u * kWaves);
      if (s + (u + kAhead) * kWaves < steps) load(u, s + (u + kAhead) * kWaves);
    }
  }
  part[wave][lane] = acc;
  __syncthreads();
  if (wave != 0) return;
  const int n = n0 + 4 * j;
  i32x4 c = part[0][lane];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) c += part[i][lane];
  f32x4 weight_scale;
#pragma unroll
  for (int e = 0; e < 4; ++e) weight_scale[e] = a.weight_scales[min(n + e, a.n - 1)];
  if (r < a.rows) store_results<Fp32>(a, r, n, results(c, a.scales[r], weight_scale, a.bias, n, a.n - 1));
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
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"      // m0 is reserved, and clobbered all the same
// Copies 64 pieces of 16 bytes to LDS, lane after lane from `lds` on.
__device__ __forceinline__ void copy_to_lds(const int8_t* base, unsigned offset, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(offset), "s"(uniform_address(base)), "s"(uniform((int)lds)) : "memory", "m0");
}

// ... 64 times four bytes.
__device__ __forceinline__ void copy_words_to_lds(const float* base, unsigned offset, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" :: "v"(offset), "s"(base), "s"(lds) : "memory", "m0");
}
#pragma clang diagnostic pop

// A workgroup's BN channels by BM rows, one tile.  Stages of U times 128 values of the sum, U lines of each row, go straight from memory to LDS, S of them in a ring; a row's eight
// 16-byte pieces are permuted by bits 1 to 3 of its number, so that 16 lanes that read the same piece of 16 rows meet all banks.  (WN channels by WM rows, and of a
// stage one part of K, belong to a wavefront.)  The operands of 32 values are read while the matrix instructions of the 32 before them run; the workgroup meets
// once a stage, ahead of the last of these, when all of the stage has been read: its place is then free for the copies of the stage S behind it.
// Bound by the way of the tiles' lines to a compute unit, most of which another one asks for too: 45 to 95 GB/s for each, 256 rows of 4096 to 6144 channels 17.1 us where weights come from memory and
// 12.7 where the last level's cache has them (34 MB in all, 6.9 us at a large copy's rate).  Small tiles want long stages (37 rows of 8192 to 1280 channels, from memory and from that cache: two lines 9.4 and 7.9 us, one
// 13.6 and 10.6, in a ring of the same bytes 11.2 and 11.0; alone on its unit 128 by 64 too: 256 rows of 4096 to 6144 17.2 and 17.8 from memory, 200 15.6 and 17.0, the same from the cache), and eight wavefronts of 32 by 32
// serve 128 by 64 better than four of 64 by 32 (128 rows of 4096 to 16384 channels, from memory, 22.4 and 22.8 us).
// Tiles are taken in plain order, the channels' first: those of the same channels in other rows meet on a die, which then has their part of the weight once, where there is a multiple of eight tiles of channels.
// Turned: the whole stages are taken in a ring of their own, for each eighth column of tiles (with the first rows a die's next one) from three stages further on: rows that lie a multiple of 4096 bytes apart
// have the same stage in the same few channels of the L2, where all the die's workgroups would ask for it at once.
template <int BN, int BM, int WN, int WM, int K, int S, int U, bool Turned, bool Fp32>
__global__ __launch_bounds__(BN / WN * (BM / WM) * K * 64) void matmul_tile_kernel(const MatmulRows a, int tiles_n, int tiles_m) {
  constexpr int kWaves = BN / WN * (BM / WM) * K, kSub = (BN + BM) * 128, kBytes = U * kSub, kStage = U * 128;
  constexpr int LN = BN / 8 / kWaves, LM = BM / 8 / kWaves, TN = WN / 32, TM = WM / 32, P = 4 * U / K, kEach = U * (LN + LM);
  static_assert(LN * 8 * kWaves == BN && LM * 8 * kWaves == BM, "each wavefront copies whole blocks of eight rows of both");
  static_assert(P % 2 == 0, "");
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
  const int stages = (a.k + kStage - 1) / kStage, whole = a.k / kStage, rest = a.k % kStage;
  const int turn = Turned && whole > 0 ? uniform((int)((unsigned)tile_n / 8u * 3u % (unsigned)whole)) : 0;

  // A lane copies one piece of row lane / 8 of a block, the one that belongs in its place.  In a stage with fewer than 128 values the pieces behind them are piece 0 again.
  auto offset = [&](int i, int last, long stride, int values) {
    const int row = (wave + i * kWaves) * 8 + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
    return (unsigned)min(row, last) * (unsigned)stride + (unsigned)(piece * 16 < values ? piece * 16 : 0);
  };
  unsigned off_n[LN], off_m[LM];
#pragma unroll
  for (int i = 0; i < LN; ++i) off_n[i] = offset(i, a.n - 1 - n0, a.weight_stride, 128);
#pragma unroll
  for (int i = 0; i < LM; ++i) off_m[i] = offset(i, a.rows - 1 - m0, a.codes_stride, 128);
  // copy instruction i of a whole stage
  auto copy = [&](int stage, int slot, int i) {
    const int u = i / (LN + LM), j = i % (LN + LM);
    const unsigned to = lds0 + slot * kBytes + u * kSub + wave * 1024;
    const int at = Turned ? stage + turn : stage;
    const long k = (long)(Turned && at >= whole ? at - whole : at) * kStage + u * 128;
    if (j < LN) copy_to_lds(weight + k, off_n[j < LN ? j : 0], to + j * kWaves * 1024);
    else copy_to_lds(codes + k, off_m[j < LN ? 0 : j - LN], to + BN * 128 + (j - LN) * kWaves * 1024);
  };
  auto copy_any = [&](int stage, int slot) {
    if (stage < whole) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) copy(stage, slot, i);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const unsigned to = lds0 + slot * kBytes + u * kSub + wave * 1024;
        const int first = u * 128 < rest ? u * 128 : 0, values = min(rest - first, 128);
        const long k = (long)stage * kStage + first;
#pragma unroll
        for (int i = 0; i < LN; ++i) copy_to_lds(weight + k, offset(i, a.n - 1 - n0, a.weight_stride, values), to + i * kWaves * 1024);
#pragma unroll
        for (int i = 0; i < LM; ++i) copy_to_lds(codes + k, offset(i, a.rows - 1 - m0, a.codes_stride, values), to + BN * 128 + i * kWaves * 1024);
      }
    }
  };

  i32x16 acc[TN][TM] = {};
  struct Operands {
    i32x4 n[TN], m[TM];
  };
  const int swizzle = (lane >> 1) & 7, half = lane >> 5;
  const int at_n = (wn * WN + (lane & 31)) * 128, at_m = BN * 128 + (wm * WM + (lane & 31)) * 128;
  auto read = [&](Operands& f, int slot, int kk) {
    const char* const from = smem + slot * kBytes + (kk >> 2) * kSub + (((2 * (kk & 3) + half) ^ swizzle) * 16);
#pragma unroll
    for (int t = 0; t < TN; ++t) f.n[t] = *reinterpret_cast<const i32x4*>(from + at_n + t * 4096);
#pragma unroll
    for (int t = 0; t < TM; ++t) f.m[t] = *reinterpret_cast<const i32x4*>(from + at_m + t * 4096);
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
  if (stages >= S) HFX_WAIT_VMCNT((S - 1) * kEach);
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
      Operands &now = f[p & 1], &then = f[(p + 1) & 1];
      if (p < P - 1) {
        read(then, slot, (p + 1) * K + kpart);
      } else if (more || s + 1 < stages) {
        if (more || s + S <= stages) HFX_WAIT_VMCNT((S - 2) * kEach);      // the stages behind the next one may still be on their way
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
            for (int i = 0; i < kEach; ++i)
              if (i * TN / kEach == t) copy(s + S, slot, i);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    ++s;
    slot = behind;
  };
  while (s + S < whole) stage(std::true_type());
  while (s < whole) stage(std::false_type());
  if (rest != 0) {
#pragma unroll 1
    for (int kk = kpart; kk < 4 * U; kk += K) {
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
        if (m < a.rows) store_line(a, m, n1 + piece * 8, line);
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
// Bound by the clock that power leaves the matrix cores, with the LDS close behind: 8192 rows of 4096 to 6144 channels 172 to 176 us, 2.35 to 2.4 POP/s (a library's product 184; of 8224 rows 207, here 181), the matrix cores busy in 61 %
// of the cycles of a clock of 1.85 GHz; 8192 of 8192 to 8192 434 to 450 us.  Nothing but these instructions, on operands in registers, runs at 3.2 to 3.4 POP/s with random operands and at 4.5 with zeros.  Four wavefronts of 128 by
// 128, which read a third less from the LDS, take 183 and 464 us.  (Tiles whose copies end with them, in one ring for both operands: 8224 rows 219 us; with both, and no second launch, 195 to 205.)
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
    asm volatile("" ::: "memory");                  // (other lanes read them; LDS serves a wavefront in order)
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

typedef hipError_t (*Launch)(const MatmulRows&, bool, hipStream_t);

static hipError_t launch_few(const MatmulRows& a, bool fp32, hipStream_t stream) {
  return launch(fp32 ? matmul_few_kernel<true> : matmul_few_kernel<false>, dim3((unsigned)(a.n + 15) / 16), 1024, stream, a);
}
template <int BN, int BM, int WN, int WM, int K, int S, int U, bool Turned>
static hipError_t launch_tiles_as(const MatmulRows& a, bool fp32, hipStream_t stream) {
  const int tiles_n = (a.n + BN - 1) / BN, tiles_m = (a.rows + BM - 1) / BM;
  return launch(fp32 ? matmul_tile_kernel<BN, BM, WN, WM, K, S, U, Turned, true> : matmul_tile_kernel<BN, BM, WN, WM, K, S, U, Turned, false>,
                dim3((unsigned)tiles_n * (unsigned)tiles_m), BN / WN * (BM / WM) * K * 64, stream, a, tiles_n, tiles_m);
}
// Where the stages are taken in turns, plain and so, over 184 products that come here (1 to 128 rows, sums of 4096 to 16384 values, 2048 to 20480 channels), from memory and from the last level's cache: 32x32 on
// average 0.91 and 0.88 times the time, 64x64 0.90 and 0.94.  In us, from the cache (from memory): 64 rows of 8192 to 4096 channels by 32x32 13.5 and 9.2 (13.4 and 13.2), 16 of 4096 to 16384 13.7 and 11.8 (15.9 and 14.2);
// by 64x64 64 of 4096 to 16384 12.8 and 12.6 (18.4 and 16.3), 33 of 16384 to 16384 65.5 and 46.9.  The worst, two tiles of rows by 64x64: 112 of 4096 to 8192 10.2 and 11.4 (13.8 and 14.2).  What does not come here: 256 rows of 8192 to
// 4096 by 64x64 16.2 and 18.4, 64 of 5120 to 5120 by 32x32 8.8 and 9.4, 37 of 8192 to 1280 (80 tiles) 8.1 and 8.4; 32x64, which has no such form though it would pay (96 of 16384 to 4096 27.2 and 20.7, from memory 31.1 and 24.7;
// 96 of 8192 to 4096 15.1 and 11.8, 16.6 and 14.6).
static bool takes_turns(int bn, int bm, int rows, int n, long weight_stride) {
  return bn == bm && bn <= 64 && rows <= 128 && weight_stride % 4096 == 0 && (long)((n + bn - 1) / bn) * ((rows + bm - 1) / bm) >= kComputeUnits;
}
template <int BN, int BM, int WN, int WM, int K, int S, int U>
static hipError_t launch_tiles(const MatmulRows& a, bool fp32, hipStream_t stream) {
  if constexpr (BN == BM && BN <= 64)
    if (takes_turns(BN, BM, a.rows, a.n, a.weight_stride)) return launch_tiles_as<BN, BM, WN, WM, K, S, U, true>(a, fp32, stream);
  return launch_tiles_as<BN, BM, WN, WM, K, S, U, false>(a, fp32, stream);
}
// Workgroups of a large kernel: one for each compute unit.  Where the sum has fewer stages than a ring each takes one tile, because the copies go on into the next tile and not past it.
template <int BN, int BM, int WN, int WM, int RN, int RM>
static hipError_t launch_large(const MatmulRows& a, bool fp32, hipStream_t stream) {
  const int tiles_n = (a.n + BN - 1) / BN, tiles_m = (a.rows + BM - 1) / BM, tiles = tiles_n * tiles_m;
  return launch(fp32 ? matmul_large_kernel<BN, BM, WN, WM, RN, RM, true> : matmul_large_kernel<BN, BM, WN, WM, RN, RM, false>,
                dim3((unsigned)((a.k + 127) / 128 < RN ? tiles : std::min(tiles, kComputeUnits))), BN / WN * (BM / WM) * 64, stream, a, tiles_n, tiles_m);
}

// What a product takes with each kernel, in us: `start`, and for each round of tiles over the chip `round` and each stage of 128 values of the sum
// stage[t - 1], t being the tiles that meet on a compute unit (`most` at most).  Fitted to 2300 times of 190 products (1 to 8224 rows, 1280 to 16384 channels, sums of 512 to 16384 values, buffers that
// change from call to call): the kernel that it names takes 1.006 times the fastest one's time on average, more than 1.1 times in one (777 rows of 8192 to 1280 channels, 260 tiles of 64 by 64, whose
// last four cost less than a second layer of tiles: 29 and 21 us).  Why there are several, in us
// (rows, k, channels; that kernel, then the next best one among the others):
// (buffers of 600 MB in turn, 24 at most: those of 37 rows stay in the last level's cache)
//   4    8192  4096        few    9.6   32x32   12.7        37    8192  1280   32x32    8.0   32x64    9.7
//   64   4096  6144      32x64   10.9   32x32   11.6        128   4096  6144   64x64   13.1   32x64   16.0
//   256  1024  8192     128x64    6.3   64x64    6.9        777   1024  8192   128x128, two to a unit 14.6   256x128 14.8
//   777  8192  4096    128x128   39.4  128x64   47.7        1500  8192  4096  128x192   58.0   256x128  60.5
//   1024 4096  6144    256x128   34.2  128x128, two to a unit 36.1
//   2500 8192  4096    256x160   83.3  256x192   88.2       4128 1024  8192  256x192   44.3  128x128   48.5       2048 4096  16384 256x256  127.5  256x128  145.8
// (channels x rows of a tile).  A product fills the chip with the largest tiles that leave little of a last round empty: the larger ones ask for fewer lines.
struct Way {
  Launch launch;
  int bn, bm, threads, most;
  float start, round, stage[2];
};
static const Way kWays[] = {
    {launch_few, 16, 8, 1024, 2, 2.1f, 0.43f, {0.098f, 0.2f}},
    {launch_tiles<32, 32, 32, 32, 4, 4, 2>, 32, 32, 256, 2, 2.1f, 0.9f, {0.11f, 0.215f}},
    {launch_tiles<32, 64, 32, 32, 2, 4, 2>, 32, 64, 256, 1, 1.8f, 1.2f, {0.17f}},
    {launch_tiles<64, 64, 32, 32, 1, 4, 1>, 64, 64, 256, 2, 1.2f, 1.8f, {0.257f, 0.42f}},
    {launch_tiles<128, 64, 32, 32, 1, 3, 2>, 128, 64, 512, 1, 0.4f, 2.6f, {0.392f}},
    {launch_tiles<128, 64, 32, 32, 1, 3, 1>, 128, 64, 512, 2, 0.4f, 2.6f, {0.413f, 0.695f}},
    {launch_tiles<128, 128, 64, 32, 1, 2, 1>, 128, 128, 512, 2, 0.2f, 3.9f, {0.725f, 1.055f}},
    {launch_tiles<128, 128, 64, 32, 1, 4, 1>, 128, 128, 512, 1, 0.4f, 3.6f, {0.553f}},
    {launch_large<128, 192, 32, 96, 3, 3>, 128, 192, 512, 1, 3.7f, 3.2f, {0.707f}},
    {launch_large<256, 128, 64, 64, 3, 3>, 256, 128, 512, 1, 4.2f, 3.7f, {0.85f}},
    {launch_large<256, 160, 32, 160, 3, 3>, 256, 160, 512, 1, 2.1f, 5.3f, {1.03f}},
    {launch_large<256, 192, 64, 96, 3, 2>, 256, 192, 512, 1, 6.5f, 3.4f, {1.24f}},
    {launch_large<256, 256, 64, 128, 3, 2>, 256, 256, 512, 1, 6.7f, 4.4f, {1.5f}},
};

// A way and the time that it takes.
struct Choice {
  const Way* way;
  float us;
};
static float time_of(const Way& w, int rows, int n, int stages) {
  const long tiles = (long)((n + w.bn - 1) / w.bn) * ((rows + w.bm - 1) / w.bm), chip = (long)kComputeUnits * w.most, rounds = tiles / chip, left = tiles - rounds * chip;
  if (tiles * w.threads >= 1l << 32 || (w.launch == launch_few && rows > w.bm)) return 3.0e38f;
  float us = w.start + (float)rounds * (w.round + (float)stages * w.stage[w.most - 1]);
  if (left) us += w.round + (float)stages * w.stage[(left - 1) / kComputeUnits];
  return us;
}
static Choice best_way(int rows, int n, int stages) {
  Choice best = {nullptr, 3.2e38f};
  for (const Way& w : kWays) {
    const float us = time_of(w, rows, n, stages);
    if (us < best.us) best = {&w, us};
  }
  return best;
}

// The launches of a product: the first takes `rows` rows and `n` channels, a second one (way[1]) the rows or the channels that are left.
// A large product whose last round would be nearly empty: two launches, one of whole rounds or of whole tiles, one of the rows or channels that are left, if the times say that this takes a twentieth less
// (8224 rows of 4096 to 6144 channels 205 -> 180 us, 4128 of 8192 to 4096 148 -> 128, 10000 of 5120 to 5120 251 -> 227; of 130 products from 60 us up none took more than 1.03 times as long.  With a fiftieth, and
// from 25 us up, some took 1.1 times: 1056 of 4096 to 4096 25.5 -> 28.0).
struct Launches {
  const Way* way[2];
  int rows, n;
};
static Launches launches_of(int all_rows, int all_n, int stages) {
  const Choice whole = best_way(all_rows, all_n, stages);
  Launches l = {{whole.way, nullptr}, all_rows, all_n};
  if (whole.us <= 60.0f) return l;
  float least = 0.95f * whole.us;
  auto consider = [&](const Way& w, int m, int c) {
    if (m <= 0 || c <= 0 || (m >= all_rows && c >= all_n)) return;
    const float us = time_of(w, m, c, stages);
    if (us >= least) return;
    const Choice rest = m < all_rows ? best_way(all_rows - m, all_n, stages) : best_way(all_rows, all_n - c, stages);
    if (us + rest.us >= least) return;
    least = us + rest.us;
    l = {{&w, rest.way}, m, c};
  };
  for (const Way& w : kWays) {
    if (w.most != 1) continue;
    const int tiles_n = (all_n + w.bn - 1) / w.bn, tiles_m = (all_rows + w.bm - 1) / w.bm;
    const long full = (long)tiles_n * tiles_m / kComputeUnits * kComputeUnits;
    consider(w, all_rows / w.bm * w.bm, all_n);
    consider(w, (int)(full / tiles_n) * w.bm, all_n);
    consider(w, all_rows, all_n / w.bn * w.bn);
    consider(w, all_rows, (int)(full / tiles_m) * w.bn);
  }
  return l;
}

hipError_t launch_matmul_rows(MatmulRows a, bool fp32, hipStream_t stream) {
  // Results of more than 64 MB go past the caches, where they push out what the tiles share: 4128 rows to 16384 channels 268 -> 255 us, 8192 rows over 1024 values to 8192
  // channels 109 -> 89 (21 MB of results: 80.6 and 79.8).
  a.past = !fp32 && a.out_stride % 8 == 0 && 2l * a.rows * a.n > (64l << 20);
  const Launches l = launches_of(a.rows, a.n, (a.k + 127) / 128);
  MatmulRows rest = a;
  if (l.way[1]) {
    const int element = fp32 ? 4 : 2;
    if (l.rows < a.rows) {
      rest.rows -= l.rows;
      rest.codes += l.rows * a.codes_stride;
      rest.scales += l.rows;
      rest.out = static_cast<char*>(a.out) + l.rows * a.out_stride * element;
    } else {
      rest.n -= l.n;
      rest.weight += l.n * a.weight_stride;
      rest.weight_scales += l.n;
      if (a.bias) rest.bias += l.n;
      rest.out = static_cast<char*>(a.out) + (long)l.n * element;
    }
    a.rows = l.rows;
    a.n = l.n;
  }
  const hipError_t e = l.way[0]->launch(a, fp32, stream);
  return e != hipSuccess || !l.way[1] ? e : l.way[1]->launch(rest, fp32, stream);
}

}  // namespace hfx

// For tests, which see to it that they reach every kernel: how many there are (rows 0), or the launches of a product, their numbers in kWays in ways[] (100 more where stages are taken in turns).
extern "C" int hfx_internal_matmul_ways(int rows, int n, int k, int64_t weight_stride, int* ways) {
  using namespace hfx;
  if (rows == 0) return sizeof(kWays) / sizeof(kWays[0]);
  const Launches l = launches_of(rows, n, (k + 127) / 128);
  int count = 0;
  for (const Way* w : l.way) {
    if (!w) break;
    const int m = count == 0 ? l.rows : l.rows < rows ? rows - l.rows : rows, c = count == 0 ? l.n : l.rows < rows ? n : n - l.n;
    ways[count++] = (int)(w - kWays) + (takes_turns(w->bn, w->bm, m, c, (long)weight_stride) ? 100 : 0);
  }
  return count;
}
