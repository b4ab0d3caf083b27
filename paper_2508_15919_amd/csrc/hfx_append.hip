// Rotary position embedding on the way into the page pool: one launch takes the step's queries, keys and values out of the projection's
// output, rotates queries and keys by their logical positions, writes the queries packed for the attention call, and keys and values into their
// pages, in bf16 or quantised to 4 bits; and the way back, from the 4-bit pages of the step's tokens to bf16 rows.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "hfx_desc.h"
#include "hfx_device.h"
#include "hfx_mx.h"
#include "hfx_launch.h"

namespace hfx {

// Rotates eight values (dimensions 8 piece .. 8 piece + 7 of a head) by the angles of their position.  A pair (a, b) turns into (a c - b s, b c + a s); every
// product and sum is rounded to fp32 by itself, so that what is quantised afterwards does not depend on how a compiler contracts them.
struct Turn {
  float c[8], s[8];
  bool on, second;       // the piece is rotated; and holds the b's of its pairs, its partner the a's
  int partner;           // lane that holds the other value of each pair
};

template <bool Interleaved>
__device__ __forceinline__ Turn turn_of(const float* __restrict__ row, int rot, int piece, int lane) {
  Turn t;
  const int pieces = rot / 8, half = pieces / 2;
  t.on = piece < pieces;
  t.second = !Interleaved && piece >= half;
  t.partner = !t.on || Interleaved ? lane : t.second ? lane - half : lane + half;
  if (t.on) {
    if constexpr (Interleaved) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 c = reinterpret_cast<const float2*>(row + 4 * piece)[i], s = reinterpret_cast<const float2*>(row + rot / 2 + 4 * piece)[i];
        t.c[2 * i] = c.x;
        t.c[2 * i + 1] = c.y;
        t.s[2 * i] = s.x;
        t.s[2 * i + 1] = s.y;
      }
    } else {
      const int at = 8 * (t.second ? piece - half : piece);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f32x4 c = reinterpret_cast<const f32x4*>(row + at)[i], s = reinterpret_cast<const f32x4*>(row + rot / 2 + at)[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          t.c[4 * i + e] = c[e];
          t.s[4 * i + e] = s[e];
        }
      }
    }
  }
  return t;
}

__device__ __forceinline__ void widen(const u32x4& v, float* x) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    x[2 * w] = __builtin_bit_cast(float, v[w] << 16);
    x[2 * w + 1] = __builtin_bit_cast(float, v[w] & 0xffff0000u);
  }
}

// All lanes of a wavefront take part (the partner's values come by a lane exchange).
template <bool Interleaved>
__device__ __forceinline__ void turn(const Turn& t, bool any, const u32x4& v, float* y) {
#pragma clang fp contract(off)
  float x[8];
  widen(v, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = x[e];
  if (!any) return;
  if constexpr (Interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = x[2 * i], b = x[2 * i + 1];
      const float ac = a * t.c[i], bs = b * t.s[i], bc = b * t.c[i], as = a * t.s[i];
      y[2 * i] = t.on ? ac - bs : a;
      y[2 * i + 1] = t.on ? bc + as : b;
    }
  } else {
    u32x4 p;
#pragma unroll
    for (int w = 0; w < 4; ++w) p[w] = (uint32_t)__shfl((int)v[w], t.partner, 64);
    float z[8];
    widen(p, z);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float xc = x[e] * t.c[e], zs = z[e] * t.s[e];
      y[e] = !t.on ? x[e] : t.second ? xc + zs : xc - zs;
    }
  }
}

__device__ __forceinline__ u32x4 narrow(const float* x) {
  u32x4 v;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const bf16x2 r = {(__bf16)x[2 * w], (__bf16)x[2 * w + 1]};
    v[w] = __builtin_bit_cast(unsigned, r);
  }
  return v;
}

// Largest magnitude, as its bits, of the 32 values that four neighbouring lanes hold (a NaN has larger bits than any number).
__device__ __forceinline__ unsigned block_top(const float* x) {
  unsigned top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __builtin_bit_cast(unsigned, x[e]) & 0x7fffffffu);
  top = max(top, (unsigned)__builtin_amdgcn_mov_dpp((int)top, 0xb1, 0xf, 0xf, true));      // lane ^ 1
  return max(top, (unsigned)__builtin_amdgcn_mov_dpp((int)top, 0x4e, 0xf, 0xf, true));     // lane ^ 2
}

// Value codes, key scales and value scales of tokens [lo, hi) of a block, which lie in LDS as they lie there: four bytes at a time where the run has all
// of their tokens, else those of its tokens.
template <int D, int T>
__device__ __forceinline__ void store_values_and_scales(char* blk, const uint8_t* s4, int tid, int lo, int hi) {
  constexpr int kG = D / 32;
  for (int i = tid; i < 9 * D / 4; i += T) {
    const int b = 4 * i;
    int first, per;              // token of the first byte; bytes that a token has in a row
    if (b < 8 * D) {
      first = b / Mx<D>::kHalf * 8 + (b & 7);
      per = 1;
    } else if (b < 8 * D + D / 2) {
      first = (b - 8 * D) / kG;
      per = kG;
    } else {
      const int r = b - 8 * D - D / 2;
      first = r / Mx<D>::kHalfScales * 8 + (r & 15) / 2;
      per = 2;
    }
    const int shift = per >> 1;  // 1, 2 or 4, and its logarithm
    if (first >= lo && first + (3 >> shift) < hi) {
      *reinterpret_cast<unsigned*>(blk + Mx<D>::kValues + b) = *reinterpret_cast<const unsigned*>(s4 + b);
    } else if (first + (3 >> shift) >= lo && first < hi) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int token = first + (e >> shift);
        if (token >= lo && token < hi) blk[Mx<D>::kValues + b + e] = (char)s4[b + e];
      }
    }
  }
}

// 16 bytes of a row that is read or written once; Past: past the caches.
template <bool Past>
__device__ __forceinline__ u32x4 load_row(const uint16_t* p) {
  const u32x4* v = reinterpret_cast<const u32x4*>(p);
  return Past ? __builtin_nontemporal_load(v) : *v;
}
template <bool Past>
__device__ __forceinline__ void store_row(uint16_t* p, const u32x4& x) {
  u32x4* v = reinterpret_cast<u32x4*>(p);
  if constexpr (Past) __builtin_nontemporal_store(x, v);
  else *v = x;
}

// Q-heads of a kv-head whose loads are in flight together.
constexpr int kQueries = 4;

// Which (run, kv-head) a workgroup takes.  Workgroups go to the dies by their index modulo 8; of 128 in a row a die takes 16 that follow each other, so
// that the heads of a run, which share its angles and rows, meet in the same L2 (8224 rows of 32 q-heads on buffers that stay, 32.4 us; 34.2 with four in a row, 39.5 with one).
__device__ __forceinline__ bool run_and_head(int n_runs, int heads, int& index, int& g) {
  constexpr unsigned kDies = HFX_QUEUE_CLASSES, kRow = 16;
  const unsigned all = (unsigned)heads * (unsigned)n_runs;
  unsigned block = (blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x;
  if (block >= all) return false;
  if (block < all / (kDies * kRow) * (kDies * kRow)) block = block / (kDies * kRow) * (kDies * kRow) + block % kDies * kRow + block / kDies % kRow;
  index = (int)(block / (unsigned)heads);
  g = (int)(block - (unsigned)index * (unsigned)heads);
  return true;
}

// One workgroup per (run, kv-head) and part, a run being the new tokens of one request in one page (at most 16): the key and value rows of the
// head are one part, the rows of the q-heads that share it the other.  A thread has one 16-byte piece of one token, of both rows or of as many q-heads as
// its loads may be in flight for.  T = 2 D threads have all 16 tokens at once, and pass the values through LDS, where a page has the tokens of a dimension
// side by side.  T = 64, for steps whose runs are of a few tokens: a wavefront goes round, values go to their bytes straight from the registers, and the
// two parts are the two wavefronts of one workgroup.
// Bound by memory where there is much to do (32 q-heads, 8 kv-heads, 128 wide, 8224 rows in long chunks: 206 MB in 38.6 us on changing buffers, 5.3 TB/s; a
// plain copy has 4.9), and by two loads that wait for each other (the run's record beside its position, then rows beside angles) and its stores where there is little (four decodes: 3.8 us, of
// which an empty kernel takes 1.5; 256 decodes into 4-bit pages 5.8).  A run of one token fills 16 of a wavefront's 64 lanes, 8 on 64-wide heads; the others do its work again and store nothing.
// With keys, values and queries in turn in one wavefront those were 6.0 and 7.5 us.
template <int D, bool Four, bool Interleaved, int T, bool Past>
__global__ __launch_bounds__(T == 64 ? 128 : T) void rope_append_kernel(const RopeAppend a) {
  constexpr bool kFew = T == 64;
  constexpr int LD = D + 8;                       // LDS row stride in elements
  constexpr int kTokens = T / (D / 8);            // at a time
  __shared__ __attribute__((aligned(16))) uint16_t sv[Four || kFew ? 1 : HFX_PAGE * LD];
  __shared__ __attribute__((aligned(16))) uint8_t s4[Four && !kFew ? 9 * D : 16];      // value codes, key scales, value scales as in the block
  const int Hkv = a.num_kv_heads, G = a.num_q_heads / Hkv, tid = threadIdx.x % T;
  const int parts = a.q ? 2 : 1;
  int index, g, part_of_head;
  if constexpr (kFew) {
    if (!run_and_head(a.n_runs, Hkv, index, g)) return;
    part_of_head = uniform((int)threadIdx.x / T);
  } else {
    if (!run_and_head(a.n_runs, parts * Hkv, index, g)) return;
    part_of_head = g & (parts - 1);
    g = parts == 2 ? g >> 1 : g;
  }
  const HfxRun run = a.runs[index];
  const bool any = a.rot > 0;
  const int position = any ? a.run_pos[index] : 0;
  const int piece = tid % (D / 8), lane = tid & 63;
  if (part_of_head == 1) {
    for (int tok = tid / (D / 8); tok < HFX_PAGE; tok += kTokens) {
      if (kTokens < HFX_PAGE && uniform(tok - tid / (D / 8)) >= run.n) break;
      const int own = min(tok, run.n - 1);         // pieces without a token read the run's last one and are not stored
      const long row = (long)run.row0 + own;
      Turn t;
      if (any) t = turn_of<Interleaved>(a.cos_sin + (long)(position + own) * a.rot, a.rot, piece, lane);
      const uint16_t* const from = a.q + row * a.q_stride + g * G * D + piece * 8;
      uint16_t* const to = a.q_out + (row * a.num_q_heads + g * G) * D + piece * 8;
      for (int h0 = 0; h0 < G; h0 += kQueries) {
        u32x4 qv[kQueries];
#pragma unroll
        for (int i = 0; i < kQueries; ++i) qv[i] = load_row<Past>(from + min(h0 + i, G - 1) * D);
#pragma unroll
        for (int i = 0; i < kQueries; ++i) {
          if (h0 + i >= G) break;
          float y[8];
          turn<Interleaved>(t, any, qv[i], y);
          if (tok < run.n) store_row<Past>(to + (h0 + i) * D, any ? narrow(y) : qv[i]);
        }
      }
    }
    return;
  }
  uint16_t* const kblk = reinterpret_cast<uint16_t*>(a.pool) + (((long)run.page * Hkv + g) * 2) * (16L * D);
  char* const blk = reinterpret_cast<char*>(a.pool) + ((long)run.page * Hkv + g) * Mx<D>::kBlock;
  for (int tok = tid / (D / 8); tok < HFX_PAGE; tok += kTokens) {
    if (kTokens < HFX_PAGE && uniform(tok - tid / (D / 8)) >= run.n) break;
    const bool live = tok < run.n;
    const int own = min(tok, run.n - 1);
    const long row = (long)run.row0 + own;
    Turn t;
    if (any) t = turn_of<Interleaved>(a.cos_sin + (long)(position + own) * a.rot, a.rot, piece, lane);
    const u32x4 kv = load_row<Past>(a.k + row * a.k_stride + g * D + piece * 8);
    const u32x4 vv = load_row<Past>(a.v + row * a.v_stride + g * D + piece * 8);
    float y[8];
    turn<Interleaved>(t, any, kv, y);
    const int slot = run.slot0 + tok;
    if constexpr (!Four) {
      if (live) {
        *reinterpret_cast<u32x4*>(kblk + ((piece >> 1) * HFX_PAGE + slot) * 16 + (piece & 1) * 8) = any ? narrow(y) : kv;
        if constexpr (kFew) {
          uint16_t* const to = kblk + 16L * D + piece * 8 * HFX_PAGE + slot;
#pragma unroll
          for (int e = 0; e < 8; ++e) to[e * HFX_PAGE] = (uint16_t)(vv[e >> 1] >> (16 * (e & 1)));
        } else {
          *reinterpret_cast<u32x4*>(sv + slot * LD + piece * 8) = vv;
        }
      }
    } else {
      constexpr int kG = D / 32;
      const int group = piece >> 2, part = piece & 3;
      const unsigned ke = scale_byte(block_top(y));
      const unsigned kc = to_fp4(y, ke);
      float x[8];
      widen(vv, x);
      const unsigned ve = scale_byte(block_top(x));
      const unsigned vc = to_fp4(x, ve);
      // a byte of value codes holds dimensions i and i + 16: lanes part and part ^ 2 join theirs, each for four of the eight
      const unsigned other = (unsigned)__builtin_amdgcn_mov_dpp((int)vc, 0x4e, 0xf, 0xf, true);
      const unsigned low = part < 2 ? vc : other >> 16, high = part < 2 ? other : vc >> 16;
      if (live) {
        *reinterpret_cast<unsigned*>(blk + (slot * kG + group) * 16 + part * 4) = kc;
        const int half = slot >> 3, at = slot & 7, tp = group >> 1, w = group & 1;
        const int i0 = 8 * (part & 1) + (part < 2 ? 0 : 4);
        uint8_t* const to = kFew ? reinterpret_cast<uint8_t*>(blk) + Mx<D>::kValues : s4;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          to[half * Mx<D>::kHalf + ((tp * 16 + i0 + i) * 2 + w) * 8 + at] = (uint8_t)((low >> (4 * i) & 15u) | (high >> (4 * i) & 15u) << 4);
        if (part == 0) {
          to[8 * D + slot * kG + group] = (uint8_t)ke;
          to[8 * D + D / 2 + half * Mx<D>::kHalfScales + (tp * 8 + at) * 2 + w] = (uint8_t)ve;
        }
      }
    }
  }
  if constexpr (!kFew) {
    __syncthreads();
    if constexpr (!Four) {
      for (int i = tid; i < 2 * D; i += T) store_value_columns<D>(kblk + 16L * D, sv, LD, i, run.slot0, run.n);
    } else {
      store_values_and_scales<D, T>(blk, s4, tid, run.slot0, run.slot0 + run.n);
    }
  }
}

// The way back: bf16 rows [T][Hkv][D] of the values that the 4-bit pages hold for the step's tokens, one workgroup of 2 D threads per (run, kv-head).  It
// writes 3.8 times what it reads and is bound by that (8224 rows of 8 heads of 128: 43 MB in 8.5 us; 256 decodes: 2.4 us).
template <int D>
__global__ __launch_bounds__(2 * D) void read_new_kv_mx_kernel(const HfxRun* __restrict__ runs, int n_runs, int Hkv, const char* __restrict__ pool,
                                                             uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out) {
  __shared__ __attribute__((aligned(16))) uint8_t s4[9 * D];
  constexpr int kG = D / 32;
  int index, g;
  if (!run_and_head(n_runs, Hkv, index, g)) return;
  const int tid = threadIdx.x;
  const HfxRun run = runs[index];
  const char* blk = pool + ((long)run.page * Hkv + g) * Mx<D>::kBlock;
  const int tok = tid / (D / 8), piece = tid % (D / 8);
  const int slot = run.slot0 + min(tok, run.n - 1), group = piece >> 2, part = piece & 3;
  const unsigned kc = *reinterpret_cast<const unsigned*>(blk + (slot * kG + group) * 16 + part * 4);
  for (int i = tid; i < 9 * D / 16; i += 2 * D) *reinterpret_cast<u32x4*>(s4 + 16 * i) = *reinterpret_cast<const u32x4*>(blk + Mx<D>::kValues + 16 * i);
  __syncthreads();
  if (tok >= run.n) return;
  const int half = slot >> 3, at = slot & 7, tp = group >> 1, w = group & 1;
  unsigned vc = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const unsigned b = s4[half * Mx<D>::kHalf + ((tp * 16 + 8 * (part & 1) + i) * 2 + w) * 8 + at];
    vc |= (part < 2 ? b & 15u : b >> 4) << (4 * i);
  }
  const unsigned ke = scale_at<0>(s4[8 * D + slot * kG + group]);
  const unsigned ve = scale_at<0>(s4[8 * D + D / 2 + half * Mx<D>::kHalfScales + (tp * 8 + at) * 2 + w]);
  const long to = (((long)run.row0 + tok) * Hkv + g) * D + piece * 8;
  *reinterpret_cast<u32x4*>(k_out + to) = u32x4{from_fp4<0>(kc, ke), from_fp4<1>(kc, ke), from_fp4<2>(kc, ke), from_fp4<3>(kc, ke)};
  *reinterpret_cast<u32x4*>(v_out + to) = u32x4{from_fp4<0>(vc, ve), from_fp4<1>(vc, ve), from_fp4<2>(vc, ve), from_fp4<3>(vc, ve)};
}

// `heads` workgroups for each run; the runs fill the two slower dimensions, the first of which holds at most 65535.
static dim3 run_grid(const HfxHeader& h, unsigned heads) {
  const unsigned per_z = (unsigned)std::min(h.n_runs, 32768);
  return dim3(heads, per_z, ((unsigned)h.n_runs + per_z - 1) / per_z);
}

hipError_t launch_rope_append(const HfxHeader& h, const void* desc, RopeAppend a, bool four, hipStream_t stream) {
  if (h.n_runs <= 0) return hipSuccess;
  a.runs = reinterpret_cast<const HfxRun*>(static_cast<const char*>(desc) + h.off_runs);
  a.run_pos = reinterpret_cast<const int*>(static_cast<const char*>(desc) + h.off_run_pos);
  a.n_runs = h.n_runs;
  a.num_q_heads = h.num_q_heads;
  a.num_kv_heads = h.num_kv_heads;
  // Runs of at most 8 tokens on average go to single wavefronts (128 chunks of n tokens, bf16 pages, then 4-bit ones, against 2 D threads: n = 2
  // 5.0 us : 7.8, 4.5 : 7.6; n = 4 5.2 : 7.8, 4.8 : 7.7; n = 8 7.4 : 8.5, 7.2 : 8.0; n = 12 10.6 : 8.4; n = 16 12.4 : 8.9; 256 decodes 5.7 : 11.8).
  const bool few = (long)h.total_q <= 8l * h.n_runs;
  // Rows of more than 64 MB in all (queries in and out, keys, values) go past the caches, where they would only be in the way: 8224 rows of 32 / 8 heads, 173 MB,
  // 43.7 -> 39.2 us on changing buffers (4-bit pages and the way back 50.9 -> 44.9).  With the attention that follows and reads the queries: 8224 rows 263.2 ->
  // 260.1 us, 4128 rows, 87 MB, 163.4 -> 162.8, but 2064 rows, 43 MB, 80.7 -> 81.6 and 520 25.1 -> 26.0.
  const int64_t row_bytes = (int64_t)((a.q ? 2 * h.num_q_heads : 0) + 2 * h.num_kv_heads) * h.head_dim * 2;
  const bool past = !few && row_bytes * h.total_q > (64ll << 20);
  auto pick = [&](auto d) {
    constexpr int D = decltype(d)::value;
    void (*const kernels[])(RopeAppend) = {
        rope_append_kernel<D, false, false, 2 * D, false>, rope_append_kernel<D, false, true, 2 * D, false>, rope_append_kernel<D, true, false, 2 * D, false>,
        rope_append_kernel<D, true, true, 2 * D, false>,   rope_append_kernel<D, false, false, 2 * D, true>, rope_append_kernel<D, false, true, 2 * D, true>,
        rope_append_kernel<D, true, false, 2 * D, true>,   rope_append_kernel<D, true, true, 2 * D, true>,   rope_append_kernel<D, false, false, 64, false>,
        rope_append_kernel<D, false, true, 64, false>,     rope_append_kernel<D, true, false, 64, false>,    rope_append_kernel<D, true, true, 64, false>};
    return launch(kernels[(few ? 8 : past ? 4 : 0) + (four ? 2 : 0) + (a.interleaved ? 1 : 0)],
                  run_grid(h, (few || !a.q ? 1u : 2u) * (unsigned)h.num_kv_heads), few ? (a.q ? 128u : 64u) : 2u * D, stream, a);
  };
  return h.head_dim == 128 ? pick(std::integral_constant<int, 128>()) : pick(std::integral_constant<int, 64>());
}

hipError_t launch_read_new_kv_mx(const HfxHeader& h, const void* desc, const void* pool, void* k_out, void* v_out, hipStream_t stream) {
  if (h.n_runs <= 0) return hipSuccess;
  const HfxRun* runs = reinterpret_cast<const HfxRun*>(static_cast<const char*>(desc) + h.off_runs);
  return launch(h.head_dim == 128 ? read_new_kv_mx_kernel<128> : read_new_kv_mx_kernel<64>, run_grid(h, (unsigned)h.num_kv_heads), 2u * (unsigned)h.head_dim, stream, runs, h.n_runs,
                h.num_kv_heads, static_cast<const char*>(pool), static_cast<uint16_t*>(k_out), static_cast<uint16_t*>(v_out));
}

}  // namespace hfx
