// Attention of a scheduled step over a page pool held in 4 bits (see hfx_mx.h for the format): the same work items, queue and split merge as over
// the bf16 pool, with kernels of their own for both kinds of items.
//
//   S^T = K . Q^T   on the scaled matrix instructions for 4 to 8 bits: the keys' codes and scale bytes go into them as they lie in the cache.  With their
//                   other operand in 6 bits they have four times the rate of a bf16 product, and a query is taken as the sum of three 6-bit numbers
//                   (split_query), each with a scale for 32 dimensions: three quarters of the matrix time, and no key is ever converted.  (Two 8-bit numbers
//                   would hold more, but with an operand of 8 bits the products take twice the time: 66 clocks a 32x32x64, not 34.)
//   O^T = V^T . P^T on the bf16 matrix instructions: a scale belongs to a token, which is the contracted index here, so the values are widened to bf16
//                   (every code times every scale is a bf16 number).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hfx_desc.h"
#include "hfx_device.h"
#include "hfx_mx.h"
#include "hfx_launch.h"

namespace hfx {

typedef int i32x8 __attribute__((ext_vector_type(8)));

typedef unsigned u32x6 __attribute__((ext_vector_type(6)));
typedef float f32x32 __attribute__((ext_vector_type(32)));
typedef __bf16 bf16x32 __attribute__((ext_vector_type(32)));

// Operand formats of the scaled matrix instructions.
constexpr int kE2M3 = 2, kE3M2 = 3, kE2M1 = 4;

// The 4-bit operand takes four registers of the eight that the builtins ask for, the 6-bit one six.
__device__ __forceinline__ i32x8 fp4_operand(const u32x4& c) { return i32x8{(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0}; }
__device__ __forceinline__ i32x8 fp6_operand(const u32x6& c) { return i32x8{(int)c[0], (int)c[1], (int)c[2], (int)c[3], (int)c[4], (int)c[5], 0, 0}; }

// 32 query values as the sum of three sets of 6-bit numbers with scales 2^(e - 127), 2^(e - 6 - 127) and 2^(e - 10 - 127).  e brings the largest magnitude into
// [3.875, 7.75), where the nearest number of E2M3 (4 significant bits, up to 7.5, steps of 1/8 below 2) is at most 1/4 away.  A bf16 value has 8 significant bits: from 1
// up the remainder is at most eight of its last places, which the 3 significant bits of E3M2 hold; a smaller value's remainder is at most 1/16 and rounds by at
// most 2^-8, which the third number, E2M3 again, takes up in steps of 2^-13 and less.  So the three are the value from 2^-6 up, 1/248 of the largest at most, and below it are at
// most 2^-14 away, 1.6e-5 of the largest.  (The first two alone, exact from about a quarter of the largest up and 0.001 of it away below, put results 0.004 off where some
// channels are 8 times the others and 0.037 where they are 100 times those; bf16 weights and result make 0.0024.)
struct Query6 {
  u32x6 n[3];
  unsigned scale;          // bytes: of each
};
constexpr unsigned kRestScale = 6, kLastScale = 10;
__device__ __forceinline__ Query6 split_query(const bf16x8* q) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u32x4 u = __builtin_bit_cast(u32x4, q[i]);
#pragma unroll
    for (int w = 0; w < 4; ++w) top = max(top, max(u[w] & 0x7fff0000u, u[w] << 16 & 0x7fff0000u));
  }
  const unsigned e = (unsigned)max((int)((top + 0x80000u) >> 23) - 2, (int)kLastScale + 1);
  auto scale = [&](unsigned lower) { return __builtin_bit_cast(float, (e - lower) << 23); };
  bf16x32 x;
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] = q[i >> 3][i & 7];
  auto rest = [&](const f32x32& taken) {                 // (exact, and a bf16 number)
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = (__bf16)((float)x[i] - taken[i]);
  };
  Query6 t;
  t.n[0] = __builtin_amdgcn_cvt_scalef32_pk32_fp6_bf16(x, scale(0));
  rest(__builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(t.n[0], scale(0)));
  t.n[1] = __builtin_amdgcn_cvt_scalef32_pk32_bf6_bf16(x, scale(kRestScale));
  rest(__builtin_amdgcn_cvt_scalef32_pk32_f32_bf6(t.n[1], scale(kRestScale)));
  t.n[2] = __builtin_amdgcn_cvt_scalef32_pk32_fp6_bf16(x, scale(kLastScale));
  t.scale = top >= 0x7f800000u ? 0xffffffu : e | (e - kRestScale) << 8 | (e - kLastScale) << 16;       // 255 makes the products NaN, which 6 bits cannot say
  return t;
}

// Values of two tokens in a row and two dimensions, i and i + 16 of 32, out of two bytes of codes (numbers Byte and Byte + 1) and the tokens' scale bytes,
// numbers At and At + 2 of `scales`: the operand registers of the two dimensions.
template <int Byte, int At>
__device__ __forceinline__ void widen_pair(unsigned codes, unsigned scales, unsigned& lo, unsigned& hi) {
  const unsigned t0 = from_fp4<Byte>(codes, scale_at<At>(scales)), t1 = from_fp4<Byte + 1>(codes, scale_at<At + 2>(scales));
  lo = __builtin_amdgcn_perm(t1, t0, 0x05040100u);
  hi = __builtin_amdgcn_perm(t1, t0, 0x07060302u);
}
// Number k of the four pairs of eight tokens with codes in a, b.
template <int At>
__device__ __forceinline__ void widen_pair(int k, unsigned a, unsigned b, const u32x4& scales, u32x4& lo, u32x4& hi) {
  unsigned l, h;
  if (k % 2 == 0) widen_pair<0, At>(k < 2 ? a : b, scales[k], l, h);
  else widen_pair<2, At>(k < 2 ? a : b, scales[k], l, h);
  lo[k] = l;
  hi[k] = h;
}
template <int At>
__device__ __forceinline__ void widen_values(unsigned a, unsigned b, const u32x4& scales, u32x4& lo, u32x4& hi) {
#pragma unroll
  for (int k = 0; k < 4; ++k) widen_pair<At>(k, a, b, scales, lo, hi);
}

// A page's block in LDS: key codes [group][16 keys][16 bytes], value codes, then the scales as in the block; the copy of the scales writes 256 bytes.
template <int D>
struct RawPage {
  static constexpr int kBytes = 16 * D + 256;
  static constexpr int kCopies = D == 128 ? 3 : 2;     // instructions that copy it
};
// Offsets, inside a block, of the lane's parts of the copy: keys change their order from [key][group] to [group][key].  Value codes, of which a unit of
// 16 bytes has eight tokens of four dimensions, keep theirs, [8 tokens][64 dimensions][16], or (InTurn) get [64 dimensions][16][8 tokens].
template <int D>
struct CopyLane {
  unsigned keys, values, scales;
};
template <int D, bool InTurn>
__device__ __forceinline__ CopyLane<D> copy_lane(int lane) {
  constexpr int kG = Mx<D>::kGroups;
  CopyLane<D> c;
  const int unit = lane & (D / 2 - 1);                 // of the value codes (D = 64: those of the lanes from 32 on)
  const unsigned values = (unsigned)(InTurn ? (unit & 1) * Mx<D>::kHalf + (unit >> 1) * 16 : unit * 16);
  c.keys = D == 128 || lane < 32 ? (unsigned)(((lane & 15) * kG + ((lane >> 4) & (kG - 1))) * 16) : Mx<D>::kValues + values;
  c.values = values;
  c.scales = (unsigned)(lane & (D / 4 - 1)) * 4;
  return c;
}
// Reads of the block table between copies that the compiler does not know of are scalar loads all the same: constant memory does not change.
typedef const __attribute__((address_space(4))) int* ConstantInts;
__device__ __forceinline__ ConstantInts constant(const int* p) { return (ConstantInts)(uintptr_t)p; }

__device__ __forceinline__ unsigned lds_offset(const void* p) {
  return (unsigned)uniform((int)(unsigned)(uintptr_t)(__attribute__((address_space(3))) const char*)p);
}

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// Direct-to-LDS copy of a page's block: base (scalar), the lane's offsets, LDS destination; Past: past the caches.  The compiler does not know of these
// loads: its own waits for vector memory become stricter by them, and those for what is copied are explicit (HFX_WAIT_VMCNT).
template <int D, bool Past>
__device__ __forceinline__ void raw_copy(const char* base, const CopyLane<D>& c, unsigned lds) {
  if constexpr (D == 128 && Past)
    asm volatile("s_mov_b32 m0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %3 nt\n\tglobal_load_lds_dwordx4 %1, %3 offset:1024 nt\n\t"
                 "global_load_lds_dword %2, %3 offset:2048 nt"
                 :: "v"(c.keys), "v"(c.values), "v"(c.scales), "s"(base), "s"(lds) : "memory", "m0");
  else if constexpr (D == 128)
    asm volatile("s_mov_b32 m0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %3\n\tglobal_load_lds_dwordx4 %1, %3 offset:1024\n\t"
                 "global_load_lds_dword %2, %3 offset:2048"
                 :: "v"(c.keys), "v"(c.values), "v"(c.scales), "s"(base), "s"(lds) : "memory", "m0");
  else if constexpr (Past)
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2 nt\n\tglobal_load_lds_dword %1, %2 offset:1024 nt"
                 :: "v"(c.keys), "v"(c.scales), "s"(base), "s"(lds) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2\n\tglobal_load_lds_dword %1, %2 offset:1024"
                 :: "v"(c.keys), "v"(c.scales), "s"(base), "s"(lds) : "memory", "m0");
}
// 64 page ids, one a lane, out of a table (scalar base) at the lane's byte offset.
__device__ __forceinline__ void ids_copy(const int* table, unsigned offset, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" :: "v"(offset), "s"(table), "s"(lds) : "memory", "m0");
}
#pragma clang diagnostic pop

// ----------------------------------------------------------------------------------------------
// Decode item: as over the bf16 pool one wavefront per kv-head (hn of them), the others interleave over page pairs.  Per pair (32 tokens) and kv-head a
// wavefront takes 4352 bytes (D = 128), by direct-to-LDS copies into a ring of its own, three pairs ahead of their use: 104 KB in flight on a CU
// without a register (pairs held in registers, three or four deep, did not fit: 793 us where this took 475).
// Bound: HBM.  256 decodes of 2048 to 16384 tokens, 32 / 8 heads of 128: 2.59 GB in 415 to 442 us by the card, 5.9 to 6.2 TB/s, merge included; through the
// caches 457 to 475, of which all but the arithmetic was 464.
//   S^T[token][head]: 16x16x128, a lane has 32 dimensions of one key (a group) with their scale; D = 64: lanes of the upper half have the
//                     same keys again, against zeros.
//   O^T[d][head]    : 16x16x32 bf16, a lane has eight tokens of dimension n of each tile.
// The softmax is that of the prefill items: weights against the maximum of the item's first pair, which is raised only when a lane's eight weights sum to
// more than 2^8, so that the common pair needs no maximum, no exchange between lanes and no rescaling.
// ----------------------------------------------------------------------------------------------
constexpr int kRingPairs = 4;
// Pages 64 bytes further apart than they are long: lanes of two pages and two groups read keys together.
template <int D>
constexpr int kDecodePage = RawPage<D>::kBytes + 64;

// Lane's parts of the LDS addresses inside a pair.
struct DecodeLane4 {
  int key, key_scale, value, value_scale;
};

__device__ __forceinline__ f32x4 decode_scores4(const u32x4& k, unsigned ks, const Query6& q) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  const i32x8 a = fp4_operand(k);
  s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, fp6_operand(q.n[0]), s, kE2M1, kE2M3, 0, (int)ks, 0, (int)q.scale);
  s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, fp6_operand(q.n[1]), s, kE2M1, kE3M2, 0, (int)ks, 1, (int)q.scale);
  s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, fp6_operand(q.n[2]), s, kE2M1, kE2M3, 0, (int)ks, 2, (int)q.scale);
  return s;
}

// State of a decode item: reference exponent and running sum of this lane's column, O^T accumulators.
template <int D>
struct DecodeState4 {
  float m, l;
  f32x4 o[D / 16];
};

// Maximum over a column: lanes n, n + 16, n + 32, n + 48.
__device__ __forceinline__ float column_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return max_xor32(x);
}

// Eight weights, rounded to bf16 for the product with the values (which with their scales fit no other 16-bit type), and their sum as they were: the roundings, 2^-9 each at
// most and as many up as down, are those of the bf16 pool's decode items.
__device__ __forceinline__ float decode_weights(const float* s, float sl2, float m, bf16x8& pb) {
  float p[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    p[e] = fast_exp2(__builtin_fmaf(s[e], sl2, -m));
    pb[e] = (__bf16)p[e];
  }
  return ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
}

template <int D>
__device__ __forceinline__ void decode_pair4(const char* ring, const DecodeLane4& a, const Query6& q, DecodeState4<D>& w, float sl2, bool first, bool tail,
                                             int nv) {
  const u32x4 ka = *reinterpret_cast<const u32x4*>(ring + a.key), kb = *reinterpret_cast<const u32x4*>(ring + a.key + 64);
  const unsigned ea = *reinterpret_cast<const uint8_t*>(ring + a.key_scale);
  const unsigned eb = *reinterpret_cast<const uint8_t*>(ring + a.key_scale + 4 * Mx<D>::kGroups);
  u32x4 v[D / 64], vs[D / 64];
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    v[i] = *reinterpret_cast<const u32x4*>(ring + a.value + i * 256);
    vs[i] = *reinterpret_cast<const u32x4*>(ring + a.value_scale + i * 16);
  }
  const f32x4 sa = decode_scores4(ka, ea, q), sb = decode_scores4(kb, eb, q);
  float s[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    s[e] = sa[e];
    s[4 + e] = sb[e];
  }
  if (tail) {              // tokens past the context
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = keep_or_neg_inf(s[e], e < nv);
  }
  auto top = [&]() {
    return column_max(fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])))) * sl2;
  };
  if (first) w.m = top();
  bf16x8 pb;
  float sum = decode_weights(s, sl2, w.m, pb);
  if (__builtin_expect(__any(sum > 256.0f), 0)) {
    const float m = fmaxf(w.m, top());
    const float alpha = fast_exp2(w.m - m);
    w.l *= alpha;
#pragma unroll
    for (int b = 0; b < D / 16; ++b) w.o[b] *= alpha;
    w.m = m;
    sum = decode_weights(s, sl2, m, pb);
  }
  w.l += sum;
#pragma unroll
  for (int t = 0; t < D / 32; ++t) {
    u32x4 lo, hi;
    if (t % 2 == 0) widen_values<0>(v[t / 2][0], v[t / 2][1], vs[t / 2], lo, hi);
    else widen_values<1>(v[t / 2][2], v[t / 2][3], vs[t / 2], lo, hi);
    bf16x8 v0 = __builtin_bit_cast(bf16x8, lo), v1 = __builtin_bit_cast(bf16x8, hi);
    if (tail) {            // unused slots hold anything
      v0 = keep_first(v0, nv);
      v1 = keep_first(v1, nv);
    }
    w.o[2 * t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pb, w.o[2 * t], 0, 0, 0);
    w.o[2 * t + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pb, w.o[2 * t + 1], 0, 0, 0);
  }
}

// Query operands of a kv-head's q-heads (column n), zero past the group: lane group j has 32 dimensions, 32j .. 32j + 31, or zeros past the head's.
template <int D>
__device__ __forceinline__ Query6 decode_query4(const __bf16* q, const HfxItem& item, int g, int Hq, int G, int n, int j) {
  const int hh = n < G ? n : G - 1;
  const __bf16* row = q + ((long)item.rq.q_start * Hq + g * G + hh) * D + (j & (Mx<D>::kGroups - 1)) * 32;
  bf16x8 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = keep_first(ld16(row + i * 8), n < G && j < Mx<D>::kGroups ? 8 : 0);
  return split_query(x);
}

// Runs the decode item t.cur and carries on for as long as the workgroup's next item is a decode item too.
template <int D, bool Past>
__device__ void decode_run4(const KArgs& a, const HfxHeader* H, const HfxItem* __restrict__ items, int n_items, Tickets& t, int* s_tk, int* ctrl,
                            char* smem) {
  constexpr int kPage = kDecodePage<D>, kRing = 2 * kRingPairs * kPage, kCopies = 2 * RawPage<D>::kCopies;
  const int tid = threadIdx.x;
  int lane = tid & 63;
  asm volatile("" : "+v"(lane));     // what follows from it is formed per run, not kept in registers through prefill runs
  const int wave = uniform(tid >> 6);
  const int Hq = H->num_q_heads, Hkv = H->num_kv_heads;
  const int G = Hq / Hkv;
  const int n = lane & 15, j = lane >> 4;
  const float sl2 = __builtin_bit_cast(float, uniform(__builtin_bit_cast(int, H->softmax_scale * 1.4426950408889634f)));
  const int* bt = reinterpret_cast<const int*>(a.desc + H->off_bt);
  const char* pool = reinterpret_cast<const char*>(a.pool);
  // Row rho of score tile A is token ((rho>>2)&1)*8 + (rho&3) of page rho>>3, of tile B the token 4 further on; so a lane holds the scores of 8
  // tokens in a row, (j&1)*8.. of page j>>1, which are the ones it takes of the values.
  constexpr int kG = Mx<D>::kGroups;
  const int token = ((n >> 2) & 1) * 8 + (n & 3), group = j & (kG - 1);
  DecodeLane4 la;
  la.key = (n >> 3) * kPage + group * 256 + token * 16;
  la.key_scale = (n >> 3) * kPage + Mx<D>::kKeyScales + token * kG + group;
  la.value = (j >> 1) * kPage + Mx<D>::kValues + (j & 1) * Mx<D>::kHalf + n * 16;
  la.value_scale = (j >> 1) * kPage + Mx<D>::kValueScales + (j & 1) * Mx<D>::kHalfScales;
  const int tok_lane = (j >> 1) * 16 + (j & 1) * 8;   // first of this lane's 8 tokens inside the pair
  const CopyLane<D> cl = copy_lane<D, false>(lane);
  char* const ring = smem + wave * kRing;
  const unsigned lds_ring = lds_offset(ring);

  HfxItem it = items[t.cur];
  DecodeWave d = decode_wave(bt, it, wave);
  for (;;) {
    // The ring holds the pairs from the one at work on; page ids are fetched one pair ahead of the copies that need them.
    int next = d.pp;                   // pair to be copied next
    int n0 = d.a0, n1 = d.a1;          // its pages
    int to = 0;                        // and its place in the ring
    auto copy_pair = [&]() {
      const unsigned long b0 = (unsigned)n0 * (unsigned)Hkv + (unsigned)d.g, b1 = (unsigned)n1 * (unsigned)Hkv + (unsigned)d.g;
      raw_copy<D, Past>(pool + b0 * Mx<D>::kBlock, cl, lds_ring + (unsigned)to);
      raw_copy<D, Past>(pool + b1 * Mx<D>::kBlock, cl, lds_ring + (unsigned)(to + kPage));
      next += d.step;
      to = to == kRing - 2 * kPage ? 0 : to + 2 * kPage;
      n0 = constant(bt)[d.bt0 + min(next, d.last_page)];
      n1 = constant(bt)[d.bt0 + min(next + 1, d.last_page)];
    };
#pragma unroll 1
    for (int i = 0; i < kRingPairs - 1 && next < d.pe; ++i) copy_pair();
    const Query6 qf = decode_query4<D>(a.q, it, d.g, Hq, G, n, j);
    // the record of the next item and, if it is a decode item, this wavefront's share of it
    const HfxItem nx = items[t.nxt < n_items ? t.nxt : t.cur];
    const bool carry_on = t.nxt < n_items && nx.type == HFX_ITEM_DECODE;
    const DecodeWave dn = decode_wave(bt, nx, wave);

    DecodeState4<D> w;
#pragma unroll
    for (int b = 0; b < D / 16; ++b) w.o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    w.m = NEG_INF;
    w.l = 0.f;
    bool reserved = false, first = true;
    int pending = 0, at = 0;
    for (int pp = d.pp; pp < d.pe; pp += d.step) {
      if (!reserved && pp + 4 * d.step >= d.pe) {   // a few pairs before the end (thread 0 sits in the first wavefront, which always has pairs)
        tickets_reserve(t, pending, ctrl);
        reserved = true;
      }
      // this pair's copies have landed: those of the pairs behind it may be on their way
      if (next < d.pe) {
        __builtin_amdgcn_s_waitcnt(0xc07f);     // lgkmcnt(0): the pair before this one, whose place is copied into, has been read
        copy_pair();
        HFX_WAIT_VMCNT((kRingPairs - 1) * kCopies);
      } else {
        const int behind = (next - pp) - d.step;
        if (behind == 2 * d.step) HFX_WAIT_VMCNT(2 * kCopies);
        else if (behind == d.step) HFX_WAIT_VMCNT(kCopies);
        else HFX_WAIT_VMCNT(0);
      }
      asm volatile("" ::: "memory");
      decode_pair4<D>(ring + at, la, qf, w, sl2, first, (pp + 2) * HFX_PAGE > d.tend, d.tend - (pp * HFX_PAGE + tok_lane));
      asm volatile("" ::: "memory");
      first = false;
      at = at == kRing - 2 * kPage ? 0 : at + 2 * kPage;
    }
    tickets_publish(t, pending, s_tk, ctrl, H);
    decode_store<D, kRing>(a, H, it, w.o, w.m, w.l, Hq, G, tid, wave, n, j, smem);
    __syncthreads();                  // frees the LDS partials; the ticket was published before the barrier in decode_store
    tickets_take(t, s_tk, n_items);
    if (!carry_on) break;
    it = nx;
    d = dn;
  }
}

// ----------------------------------------------------------------------------------------------
// Prefill item: four wavefronts, each with 32 chunk rows of one q-head, all sharing the kv-head.  Keys arrive in steps of 64 (four pages, one a
// wavefront): the wavefront copies its page's block into a ring of raw slots with direct-to-LDS loads, two steps ahead of its use at least; key codes are
// read from there as operands by all four, and the value codes are widened to bf16 by the wavefront that copied them, a step ahead of
// their use, into one of two slots in operand order.  So each value is widened once a workgroup, not once a wavefront.
// Bound: on long chunks the matrix cores are busy for 58 % of the cycles, and vector instructions, of which a third widen values, take about as many without overlapping
// them well; and the clock that power leaves, 1.77 GHz.  Four chunks of 2048 rows behind 0 to 12288 tokens and 32 decodes, 32 / 8 heads of 128: 780 to 788 us, 1222 to 1235 TFLOP/s
// (over the bf16 pool 828 on the same card; a library product of 16384^3 has 1485); on zeros, which take less power, 619 us.
//   S^T[key][row]  = K . Q^T     32x32x64 scaled, keys' codes against the three numbers of the queries
//   O^T[d][row]   += V^T . P^T   32x32x16 bf16, as over the bf16 pool
// ----------------------------------------------------------------------------------------------
template <int D>
struct Smem4 {
  static constexpr int kRawPage = RawPage<D>::kBytes;
  static constexpr int kRawStep = 4 * kRawPage;
  static constexpr int kRawSteps = 3;
  static constexpr int kValuePage = 32 * D;            // [D / 32][32 dimensions][2 halves of 8 tokens] bf16, halves of rows 8-15 and 24-31 swapped
  static constexpr int kValueStep = 4 * kValuePage;
  static constexpr int kRing = kRawSteps * kRawStep;
  static constexpr int kOut = kRing + 2 * kValueStep;  // result rows on their way out (prefill_store), 2 KB a wavefront
  static constexpr int kPrefill = kOut + 4 * 2048, kDecode = 4 * 2 * kRingPairs * kDecodePage<D>;
  static constexpr int kBytes = kPrefill > kDecode ? kPrefill : kDecode;
};
constexpr int kStepKeys = 64;

template <int D>
struct PrefillWave4 {
  f32x16 o[D / 32];            // O^T accumulators per 32-dimension block
  Query6 q[D / 64];            // of 64 dimensions
  float m, l;                  // reference exponent (base-2 domain); running sum (when the item is done)
  f32x4 sum;                   // running sum of this lane's weights, four times
};

// Operand registers of a stage's 32 keys.
template <int D>
struct Keys4 {
  u32x4 k[D / 64];
  unsigned scale;              // the key's scales; shifted by 8 j (keys_ready), byte 2i is that of k[i]
};

template <int D>
__device__ __forceinline__ void keys_ready(Keys4<D>& k, int j) { k.scale >>= 8 * j; }

template <int D>
__device__ __forceinline__ Keys4<D> read_keys4(const char* stage, int k_lane, int s_lane) {
  Keys4<D> r;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) r.k[i] = *reinterpret_cast<const u32x4*>(stage + k_lane + i * 512);
  if constexpr (D == 128) r.scale = *reinterpret_cast<const unsigned*>(stage + s_lane);
  else r.scale = (unsigned)*reinterpret_cast<const uint16_t*>(stage + s_lane);
  return r;
}

// Matrix instructions of a stage's scores.
template <int D>
constexpr int kScoreProducts = 3 * (D / 64);
// Number i of them: 64 dimensions i / 3, number i % 3 of the queries.  (The empty asm holds it where it is: the
// compiler takes it for an ordinary function of its operands and moves it down to where the result is used, out of the softmax it is meant to run beside.)
template <int D>
__device__ __forceinline__ void score_product(const PrefillWave4<D>& w, const Keys4<D>& k, int i, f32x16& s) {
  const Query6& q = w.q[i / 3];
  const i32x8 a = fp4_operand(k.k[i / 3]), b = fp6_operand(q.n[i % 3]);
  const int ks = (int)k.scale, qs = (int)q.scale;
  if (i == 0) s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, s, kE2M1, kE2M3, 0, ks, 0, qs);
  if (i == 1) s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, s, kE2M1, kE3M2, 0, ks, 1, qs);
  if (i == 2) s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, s, kE2M1, kE2M3, 0, ks, 2, qs);
  if (i == 3) s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, s, kE2M1, kE2M3, 2, ks, 0, qs);
  if (i == 4) s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, s, kE2M1, kE3M2, 2, ks, 1, qs);
  if (i == 5) s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, s, kE2M1, kE2M3, 2, ks, 2, qs);
  asm volatile("" : "+v"(s));
}

template <int D>
__device__ __forceinline__ bf16x8 value_fragment4(const char* values, int i, int v_lane) {
  constexpr int B = D / 32;
  return *reinterpret_cast<const bf16x8*>(values + (i / B) * Smem4<D>::kValuePage + (i % B) * 1024 + v_lane);
}

struct Nothing {
  __device__ __forceinline__ void operator()(int) const {}
};

// Which weights are formed where (see Share): of a stage's 16 the value phase takes 12 (64-wide heads: 10), the score phase, three quarters as long here, the others
// at its beginning, so that the rounded weights are known well before it ends.  It has its portions spread over its instructions, one or two behind each.  (8, 10, 12 and
// 14 in the value phase: four chunks of 2048 rows 780.0, 781.1, 780.5 and 780.9 us.)
template <int D>
struct Share4;
template <>
struct Share4<128> {
  static constexpr int values[9] = {0, 0, 2, 4, 6, 8, 10, 11, 12}, scores[9] = {12, 14, 16, 16, 16, 16, 16, 16, 16};
};
template <>
struct Share4<64> {
  static constexpr int values[5] = {0, 2, 5, 7, 10}, scores[5] = {10, 13, 16, 16, 16};
};

// The weights of a stage on their way, rounded to bf16 like the result that they make (the other operand, values with their scales, fits no other 16-bit type), as
// over the bf16 pool, but summed, as rounded, by the matrix cores (values_phase4): an instruction of 16 clocks for eight
// weights of each lane, against 40 of the vector unit, which is what bounds a step.  What has to be known beforehand, whether the reference exponent is still
// in place, is in the rounded weights' top exponent bit: it is set from 2 up, which kHeadroom = 7 below the maximum is a growth of 2^8.
constexpr float kHeadroom = 7.0f;
struct Weighing4 {
  float p[16];
  unsigned pw[8];            // rounded pairs

  __device__ __forceinline__ void finish(int i) {
    const bf16x2 r = {(__bf16)p[2 * i], (__bf16)p[2 * i + 1]};
    pw[i] = __builtin_bit_cast(unsigned, r);
    asm volatile("" : "+v"(pw[i]));
  }
  // weights of scores [e0, e1), and the pairs that were completed in [before, e0)
  __device__ __forceinline__ void portion(int before, int e0, int e1, const f32x16& s, float sl2, float m) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (e >= e0 && e < e1) {
        p[e] = fast_exp2(__builtin_fmaf(s[e], sl2, -m));
        asm volatile("" : "+v"(p[e]));
      }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (2 * i + 1 >= before && 2 * i + 1 < e0) finish(i);
  }
  __device__ __forceinline__ bf16x8 fragment(int sp) const {
    return __builtin_bit_cast(bf16x8, u32x4{pw[4 * sp], pw[4 * sp + 1], pw[4 * sp + 2], pw[4 * sp + 3]});
  }
  __device__ __forceinline__ bool large() const {
    const unsigned any = (pw[0] | pw[1] | pw[2]) | (pw[3] | pw[4] | pw[5]) | (pw[6] | pw[7]);
    return (any & 0x40004000u) != 0;
  }
};

// Whether x holds in either lane of a row, n or n + 32.
__device__ __forceinline__ bool in_row(bool x) {
  const Pair32 p = swap32(x ? 1.0f : 0.0f);
  return p.lo + p.hi > 0.0f;
}

// The weights of a stage, all known, as operands; taken again in the rows whose scores have outgrown the reference exponent.  So does a weight that is
// not finite look, which the product that sums the weights (summing_operand) would multiply by zero into the sums of other rows: where
// one is left, by a query that is not finite or a score that overflows, the row's accumulators become NaN for good and its weights zero.  (By integer operations:
// the file is compiled with -fno-honor-nans.)
template <int D>
__device__ __forceinline__ void settle_weights4(PrefillWave4<D>& w, const f32x16& s, bf16x8* pb, const Weighing4& wt, float sl2) {
  pb[0] = wt.fragment(0);
  pb[1] = wt.fragment(1);
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(wt.large()) != 0, 0)) {
    const float raised = fmaxf(w.m, row_max(s, sl2) + kHeadroom);
    const float m = in_row(wt.large()) ? raised : w.m;
    unsigned alpha = __builtin_bit_cast(unsigned, fast_exp2(w.m - m));
    w.m = m;
    weights(s, sl2, m, pb);
    u32x4 p[2] = {__builtin_bit_cast(u32x4, pb[0]), __builtin_bit_cast(u32x4, pb[1])};
    bool lost = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned u = p[i / 4][i % 4];
      lost |= (u & 0x7f80u) == 0x7f80u || (u & 0x7f800000u) == 0x7f800000u;
    }
    const unsigned keep = in_row(lost) ? 0u : ~0u;
#pragma unroll
    for (int i = 0; i < 2; ++i) pb[i] = __builtin_bit_cast(bf16x8, p[i] & keep);
    alpha = (alpha & keep) | (0x7fc00000u & ~keep);
    asm volatile("" : "+v"(alpha));
    const float a = __builtin_bit_cast(float, alpha);
    w.sum *= a;
#pragma unroll
    for (int b = 0; b < D / 32; ++b) w.o[b] *= a;
  }
}

// Operand that sums eight weights of each lane: a 16x16x32 product takes the lane's weights as those of k-group lane >> 4 and column lane & 15, and gives it
// rows 4 (lane >> 4) .. + 3 of that column; so rows 4 g .. 4 g + 3 have ones in k-group g and zeros elsewhere.
__device__ __forceinline__ bf16x8 summing_operand(int lane) {
  const unsigned one = (lane & 15) >> 2 == lane >> 4 ? 0x3f803f80u : 0u;
  return __builtin_bit_cast(bf16x8, u32x4{one, one, one, one});
}

// First phase of a stage: scores of the next one, the second half of the weights of the present one (scores cur) between them, and the present
// stage's value fragments.  between(i) goes behind instruction i.
template <int D, class Between>
__device__ __forceinline__ f32x16 scores_phase4(const PrefillWave4<D>& w, Keys4<D>& k, int j, bf16x8* frag, const f32x16& cur, Weighing4& wt, float sl2,
                                                const char* values, int v_lane, Between between) {
  constexpr int S = D / 16, P = kScoreProducts<D>;
  keys_ready<D>(k, j);
  f32x16 acc;
#pragma unroll
  for (int v = 0; v < 16; ++v) acc[v] = 0.f;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    score_product<D>(w, k, i, acc);
    between(i);
#pragma unroll
    for (int h = i * S / P; h < (i + 1) * S / P; ++h) {
      frag[h] = value_fragment4<D>(values, h, v_lane);
      wt.portion(h == 0 ? Share4<D>::values[S - 1] : Share4<D>::scores[h - 1], Share4<D>::scores[h], Share4<D>::scores[h + 1], cur, sl2, w.m);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  wt.portion(Share4<D>::scores[S - 1], 16, 16, cur, sl2, w.m);
  return acc;
}

// Second phase: weighted values of the present stage, the first half of the weights of the next one (scores next) between them.
template <int D, class Between>
__device__ __forceinline__ void values_phase4(PrefillWave4<D>& w, const bf16x8* frag, const bf16x8* pb, const f32x16& next, Weighing4& wt, float sl2,
                                              const bf16x8& ones, Between between) {
  constexpr int B = D / 32, S = 2 * B;
#pragma unroll
  for (int i = 0; i < S; ++i) {
    w.o[i % B] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i], pb[i / B], w.o[i % B], 0, 0, 0);
    if (i % B == B - 1) w.sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[i / B], w.sum, 0, 0, 0);
    between(i);
    wt.portion(i == 0 ? 0 : Share4<D>::values[i - 1], Share4<D>::values[i], Share4<D>::values[i + 1], next, sl2, w.m);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Query operands of this lane's row (rows past the chunk read the last row and are never stored): of each 64 dimensions lane group j has 32j .. 32j + 31.
template <int D>
__device__ __forceinline__ void query_load4(bf16x8 (*x)[4], const __bf16* q, int row0, int last, int Hq, int n, int j) {
  const __bf16* qp = q + (long)min(row0 + n, last) * Hq * D + j * 32;
#pragma unroll
  for (int i = 0; i < D / 64; ++i)
#pragma unroll
    for (int p = 0; p < 4; ++p) x[i][p] = ld16(qp + i * 64 + p * 8);
}

template <int D>
__device__ __forceinline__ void query_rows4(PrefillWave4<D>& w, const bf16x8 (*x)[4]) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i) w.q[i] = split_query(x[i]);
}

__device__ __forceinline__ int item_steps(const HfxItem& it) { return (int)((unsigned)(it.ke - it.kb + kStepKeys - 1) / kStepKeys); }

// What the loop over an item's steps needs to know of the item after it: how to copy its steps and where its query rows are.
struct NextItem4 {
  int left, bt, last, head;
  int q_row0, q_last;
  const __bf16* q;
};

// A wavefront's part of widening a step's values, spread over the step.
template <int D>
struct Widening {
  u32x4 codes, scales;
  u32x4 lo, hi;

  __device__ __forceinline__ void read(const char* from, const char* from_scales, int lane) {
    scales = *reinterpret_cast<const u32x4*>(from_scales);
    if constexpr (D == 128) {
      codes = *reinterpret_cast<const u32x4*>(from);
    } else {
      const uint2 c = *reinterpret_cast<const uint2*>(from);
      codes[0] = c.x;
      codes[1] = c.y;
#pragma unroll
      for (int k = 0; k < 4; ++k) scales[k] >>= 8 * (lane >> 5);         // which 32 dimensions of 64
    }
  }
  // piece i of D / 16; every fourth completes two operands
  __device__ __forceinline__ void piece(int i, char* to) {
    const int k = i & 3;
    if (i < 4) widen_pair<0>(k, codes[0], codes[1], scales, lo, hi);
    else widen_pair<1>(k, codes[2], codes[3], scales, lo, hi);
    if (k == 3) {
      *reinterpret_cast<u32x4*>(to + i / 4 * 1024) = lo;
      *reinterpret_cast<u32x4*>(to + i / 4 * 1024 + 512) = hi;
    }
  }
};

// What the second half of an item (prefill_run4) hands to the first: a wavefront's accumulators, reference exponents and sums, where its ring was.
template <int D>
struct Joined {
  static constexpr int kWave = (D / 32 * 16 + 2) * 64 * 4;
  static_assert(4 * kWave <= Smem4<D>::kPrefill, "in the place of the second half's rings");
};
template <int D>
__device__ __forceinline__ void join_halves(PrefillWave4<D>& w, int part, int lane, char* place) {
  f32x4* const o = reinterpret_cast<f32x4*>(place) + lane;
  float* const ml = reinterpret_cast<float*>(place + D / 32 * 16 * 256) + lane;
  ring_barrier();          // the rings are not read any more, and nothing is on its way to them
  if (part == 1) {
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) o[(b * 4 + q4) * 64] = f32x4{w.o[b][q4 * 4], w.o[b][q4 * 4 + 1], w.o[b][q4 * 4 + 2], w.o[b][q4 * 4 + 3]};
    ml[0] = w.m;
    ml[64] = w.l;
  }
  ring_barrier();
  if (part == 0) {
    const float m = fmaxf(w.m, ml[0]), own = fast_exp2(w.m - m), other = fast_exp2(ml[0] - m);
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const f32x4 x = o[(b * 4 + q4) * 64];
#pragma unroll
        for (int e = 0; e < 4; ++e) w.o[b][q4 * 4 + e] = __builtin_fmaf(x[e], other, w.o[b][q4 * 4 + e] * own);
      }
    w.l = __builtin_fmaf(ml[64], other, w.l * own);
    w.m = m;
  }
}

// Runs the prefill item t.cur and, for as long as the workgroup's next item is a prefill item as well, carries straight on into it: the stream of
// page copies does not stop between items, only the per-row state is swapped.  Returns with t.cur at the first item it did not process.
//
// A wavefront's work on a step of two stages, behind the step's synchronisation point (scores of its first stage are there):
//   scores of the second stage  | second half of the first's softmax, reads of its value fragments, the copies of the page two steps further on
//   values of the first stage   | first half of the second's softmax, half of the next step's widening, key operands of the next step's first stage
//   scores of the next step's first stage, values of the second stage likewise.
//
// Halves: a workgroup of eight wavefronts has one item, the first four the first half of its steps and the others the second, and the first join what both
// have (prompts_attention_mx_kernel).  Both take the same number of steps, and so cross the same barriers: the second one's last may have no keys left.
template <int D, bool Halves>
__device__ void prefill_run4(const KArgs& a, const HfxHeader* H, const HfxItem* __restrict__ items, int n_items, Tickets& t, int* s_tk, int* ctrl,
                             char* smem, int* s_ids) {
  typedef Smem4<D> L;
  constexpr int SK = HFX_STAGE_KEYS, S = D / 16;
  const int part = Halves ? uniform((int)threadIdx.x / HFX_WG_THREADS) : 0;
  const int tid = Halves ? (int)threadIdx.x % HFX_WG_THREADS : (int)threadIdx.x;
  int lane = tid & 63;
  asm volatile("" : "+v"(lane));     // what follows from it is formed per run, not kept in registers through decode runs
  const int wave = uniform(tid >> 6);
  const int Hq = H->num_q_heads, Hkv = H->num_kv_heads;
  const int G = Hq / Hkv;
  const int n = lane & 31, j = lane >> 5;
  char* stage = smem + Smem4<D>::kOut + wave * 2048;
  const float sl2 = __builtin_bit_cast(float, uniform(__builtin_bit_cast(int, H->softmax_scale * 1.4426950408889634f)));
  const int* __restrict__ bt = reinterpret_cast<const int*>(a.desc + H->off_bt);
  const char* pool = reinterpret_cast<const char*>(a.pool);
  // row of this lane's key inside a stage's 32 keys (as over the bf16 pool)
  const int krow = (n >> 4) * 16 + ((n >> 2) & 1) * 8 + ((n >> 3) & 1) * 4 + (n & 3);
  const int k_lane = (krow >> 4) * L::kRawPage + j * 256 + (krow & 15) * 16;
  const int s_lane = (krow >> 4) * L::kRawPage + Mx<D>::kKeyScales + (krow & 15) * Mx<D>::kGroups;
  const int v_lane = (n * 2 + (j ^ ((n >> 3) & 1))) * 16;   // V^T rows 32b + n, keys 8j.. of a page
  char* const values = smem + L::kRing;
  const bf16x8 ones = summing_operand(lane);
  const CopyLane<D> cl = copy_lane<D, true>(lane);
  const unsigned lds_raw = lds_offset(smem + wave * L::kRawPage);
  // widening: this lane's value codes in the raw page (tokens half, unit w_i; D = 128: of 64 dimensions w_of, D = 64: of 32), their scales, and where its
  // dimensions go.  Eight lanes in a row write 128 bytes in a row, which is what a write of 16 bytes a lane takes to do without bank conflicts (with the
  // dimension in the low bits of the lane it took 16 cycles instead of 8; with the keys' reads, 12 % of a long step's cycles went to conflicts, 1 % now).
  const int half = lane & 1, w_i = (lane >> 1) & 15, w_of = lane >> 5;
  const int w_codes = wave * L::kRawPage + Mx<D>::kValues, w_lane = D == 128 ? lane * 16 : (lane & 31) * 16 + w_of * 8;
  const int w_scales = wave * L::kRawPage + Mx<D>::kValueScales + half * Mx<D>::kHalfScales + (D == 128 ? w_of * 16 : 0);
  const int w_to = wave * L::kValuePage + w_of * (D == 128 ? 2048 : 1024) + w_i * 32 + (half ^ (w_i >> 3)) * 16;

  HfxItem item0 = items[t.cur];
  const HfxItem item1 = items[t.nxt < n_items ? t.nxt : t.cur];
  int half_steps = 0;
  if constexpr (Halves) {
    half_steps = (item_steps(item0) + 1) / 2;
    const int cut = item0.kb + half_steps * kStepKeys;
    if (part == 0) item0.ke = min(item0.ke, cut);
    else item0.kb = cut;
  }
  auto steps_of = [&](const HfxItem& item) { return Halves ? half_steps : item_steps(item); };
  bool next_ok = t.nxt < n_items && item1.type == HFX_ITEM_PREFILL;
  const unsigned inv_g = 0xffffffffu / (unsigned)G + 1u;      // h / G by a multiplication (0 for G = 1)
  auto q_rows = [&](const HfxItem& item, const WaveRows& r) { return a.q + ((long)item.rq.q_start * Hq + r.head) * D; };
  auto next_item = [&](const HfxItem& item) {
    const WaveRows r = wave_rows(item, wave);
    NextItem4 x;
    x.left = steps_of(item);
    x.bt = item.rq.bt_start + (int)((unsigned)item.kb / HFX_PAGE) + wave;
    x.last = item.rq.bt_start + item.rq.n_pages - 1;
    x.head = G == 1 ? item.h0 : (int)__umulhi((unsigned)item.h0, inv_g);
    x.q_row0 = r.row0;
    x.q_last = item.rq.q_len - 1;
    x.q = q_rows(item, r);
    return x;
  };
  // The stream of page copies: the steps of the current item and then those of the next.  Page ids come in lots of up to 64 steps, into LDS by the same
  // kind of load as the pages (with a lot in a register the compiler waited for it, and with it for every copy in flight, wherever the paths of
  // the step loop meet: a 4096-row chunk behind 61440 tokens took 862 us, 795 without, with queries of two numbers); the next lot is asked for as soon as one is begun.
  NextItem4 nx = next_item(item1);
  int left_to_ask, ask_bt, ask_last, ask_head;
  auto ask_start = [&](const NextItem4& x) {
    left_to_ask = x.left;
    ask_bt = x.bt;
    ask_last = x.last;
    ask_head = x.head;
  };
  bool in_next = false;
  const int* const lots = s_ids + wave * 128;
  const unsigned lds_lots = lds_offset(lots);
  int lot = 1, at = 0, end = 0, head = 0;              // the lot at hand: which half of the lots, next entry, end, kv-head
  int have2 = 0, head2 = 0;                            // entries and kv-head of the one behind it
  bool asked = false;                                  // since the last wait for everything
  int ahead = 0;                       // steps whose copies have been issued, counted from the one at work
  int wide = 0;                        // steps whose values have been widened, likewise
  int raw_g = 0, value_g = 0;          // ring offsets of the step at work
  auto ask = [&]() {
    if (left_to_ask <= 0 && !in_next && next_ok) {
      in_next = true;
      ask_start(nx);
    }
    if (have2 == 0 && left_to_ask > 0) {
      ids_copy(bt, (unsigned)min(ask_bt + 4 * lane, ask_last) * 4u, lds_lots + (unsigned)(lot ^ 1) * 256u);
      have2 = min(left_to_ask, 64);
      head2 = ask_head;
      left_to_ask -= have2;
      ask_bt += 4 * 64;
      asked = true;
    }
  };
  auto raw_slot = [&](int steps) {     // of the step so many behind the one at work
    const int to = raw_g + steps * L::kRawStep;
    return to < L::kRing ? to : to - L::kRing;
  };
  // copies the next step, whose entry of the lot at hand is `page`, to ring offset `to`
  auto copy_one = [&](int page, int to) {
    const unsigned block = (unsigned)page * (unsigned)Hkv + (unsigned)head;
    raw_copy<D, false>(pool + (unsigned long)block * Mx<D>::kBlock, cl, lds_raw + (unsigned)to);
    ++at;
  };
  // copies steps until `limit` are on their way, as far as they are known; lots that have been asked for have landed, unless `asked`
  auto feed = [&](int limit) {
    while (ahead < limit) {
      if (at == end) {
        if (have2 == 0 || asked) break;
        lot ^= 1;
        at = lot * 64;
        end = at + have2;
        head = head2;
        have2 = 0;
        ask();
      }
      copy_one(uniform(lots[at]), raw_slot(ahead));
      ++ahead;
    }
  };
  // Workgroups b and b + 256 share a CU, and where both have something to issue the older one goes first: left to that, the older half of a long step's
  // workgroups ended at 710 us and the younger at 895.  So the younger one has the higher priority in two of three of its steps (that step
  // 869 us; in one of two, three of four and all: 875, 875 and 896; none: 904).  Where prefill items do not fill two rounds, the older workgroups have the
  // largest ones and rightly go first (a prompt of 2500 tokens 56.4 us, 60.8 with turns; two chunks of 2048 on 64-wide heads, and steps of a few hundred rows beside decodes, either way).
  const bool turns = gridDim.x == HFX_PLAN_WGS && blockIdx.x >= HFX_PLAN_WGS / 2 && H->n_prefill_items >= 2 * HFX_PLAN_WGS;
  int turn = 0;
  PrefillWave4<D> w;
  HfxItem it;
  int kt, left, ctx_len;
  WaveRows wr;
  auto item_start = [&](const HfxItem& item) {
    it = item;
    kt = item.kb;
    left = steps_of(item);
    ctx_len = item.rq.ctx_len;
    wr = wave_rows(item, wave);
  };
  item_start(item0);
  {
    bf16x8 qx[D / 64][4];
    const NextItem4 first = next_item(item0);
    ask_start(first);
    query_load4<D>(qx, first.q, first.q_row0, first.q_last, Hq, n, j);
    ask();
    query_rows4<D>(w, qx);
  }

  for (;;) {
    // Start of an item: its first step's keys have landed for everybody and its values are widened, or that is done now.
    ask();
    if (wide < 1) {
      HFX_WAIT_VMCNT(0);
      asm volatile("" ::: "memory");
      asked = false;
      feed(L::kRawSteps);
      HFX_WAIT_VMCNT(0);
      asked = false;
      ring_barrier();
      Widening<D> wd;
      wd.read(smem + raw_g + w_codes + w_lane, smem + raw_g + w_scales, lane);
#pragma unroll
      for (int i = 0; i < S; ++i) wd.piece(i, values + value_g + w_to);
      wide = 1;
    }
    w.sum = f32x4{0.f, 0.f, 0.f, 0.f};
    const int wave_end = wr.wave_kend, unmasked_upto = wr.wave_pmin;
    auto mask_stage = [&](f32x16& s, int key0) {     // keys past this lane's row's horizon (rows past the chunk: its last row's)
      if (key0 + SK - 1 > unmasked_upto) mask_scores(s, min(unmasked_upto + n, ctx_len - 1), key0 + j * 8);
    };
    f32x16 s0;
    Weighing4 wt;
    Keys4<D> keys = read_keys4<D>(smem + raw_g, k_lane, s_lane);
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) w.o[b][v] = 0.f;
    keys_ready<D>(keys, j);
#pragma unroll
    for (int v = 0; v < 16; ++v) s0[v] = 0.f;
#pragma unroll
    for (int i = 0; i < kScoreProducts<D>; ++i) score_product<D>(w, keys, i, s0);
    keys = read_keys4<D>(smem + raw_g + 2 * L::kRawPage, k_lane, s_lane);
    mask_stage(s0, kt);
    w.m = fmaxf(HFX_M_NONE, row_max(s0, sl2)) + kHeadroom;
    wt.portion(0, 0, 4, s0, sl2, w.m);
    wt.portion(0, 4, Share4<D>::values[S], s0, sl2, w.m);
    wt.portion(4, Share4<D>::values[S - 1], Share4<D>::values[S - 1], s0, sl2, w.m);
    auto mask_values = [&](bf16x8* frag, int key0) {               // unused slots may hold anything
      if (key0 + SK > ctx_len) {
#pragma unroll
        for (int i = 0; i < S; ++i) frag[i] = keep_first(frag[i], ctx_len - (key0 + i / (D / 32) * 16 + j * 8));
      }
    };
    int plain = 0;        // steps ahead that every row of the wavefront sees whole and whose copies are in the lot at hand and in time
    bool whole = false;   // the present step is one
    for (; left > 0; --left) {
      const char* const slot = values + value_g;
      value_g ^= L::kValueStep;
      char* const to = values + value_g + w_to;
      const int raw_next = raw_slot(1);
      const char* const raw = smem + raw_next;
      // Synchronisation point: the values of this step are widened, the next one's raw pages have landed, and nobody reads the slots any more that are
      // filled next.
      if (plain == 0) {
        whole = false;
        if (ahead == L::kRawSteps && !asked && wave_end > 0 && kt + 3 * SK - 1 <= unmasked_upto) {
          plain = uniform(min(min(left - 1, end - at), (int)((unsigned)(unmasked_upto - kt - 3 * SK + 1) / kStepKeys) + 1));
          whole = plain > 0;
        }
      }
      if (__builtin_expect(whole, 1)) {
        --plain;
        const int page = lots[at];           // (read ahead of the waits)
        HFX_WAIT_VMCNT(RawPage<D>::kCopies);
        ring_barrier();
        copy_one(uniform(page), raw_g);
        if (turns) {
          if (turn == 0) __builtin_amdgcn_s_setprio(0);
          if (turn == 1) __builtin_amdgcn_s_setprio(1);
          turn = turn == 2 ? 0 : turn + 1;
        }
      } else {
        if (left == 1) {                     // the next ticket is asked for and published (and what comes after the item is multiplied for nothing)
          int reply = 0;
          tickets_reserve(t, reply, ctrl);
          HFX_WAIT_VMCNT(0);
          asked = false;
          tickets_publish(t, reply, s_tk, ctrl, H);
        } else if (ahead == L::kRawSteps && !asked) {
          HFX_WAIT_VMCNT(RawPage<D>::kCopies);
        } else {
          HFX_WAIT_VMCNT(0);
          asked = false;
        }
        ring_barrier();
        wide = ahead > 1 ? 1 : 0;            // whether the next step's pages have landed (copies issued now have not); if not, what is widened below is nothing yet
        feed(1 + L::kRawSteps);
        ask();
        --ahead;
      }
      raw_g = raw_next;
      Widening<D> wd;
      if (whole || kt < wave_end) {
        bf16x8 frag[S], pb[2];
        f32x16 s1 = scores_phase4<D>(w, keys, j, frag, s0, wt, sl2, slot, v_lane, [&](int i) {
          if (i == 1) wd.read(raw + w_codes + w_lane, raw + w_scales, lane);
        });
        settle_weights4<D>(w, s0, pb, wt, sl2);
        if (!whole) {
          mask_stage(s1, kt + SK);
          mask_values(frag, kt);
        }
        __builtin_amdgcn_sched_barrier(0);
        values_phase4<D>(w, frag, pb, s1, wt, sl2, ones, [&](int i) {
          if (i == 0) keys = read_keys4<D>(raw, k_lane, s_lane);
          if (i % 2 == 1) wd.piece(i / 2, to);
        });
        s0 = scores_phase4<D>(w, keys, j, frag, s1, wt, sl2, slot + 2 * L::kValuePage, v_lane, Nothing());
        settle_weights4<D>(w, s1, pb, wt, sl2);
        if (!whole) {
          mask_stage(s0, kt + 2 * SK);
          mask_values(frag, kt + SK);
        }
        __builtin_amdgcn_sched_barrier(0);
        values_phase4<D>(w, frag, pb, s0, wt, sl2, ones, [&](int i) {
          if (i == 0) keys = read_keys4<D>(raw + 2 * L::kRawPage, k_lane, s_lane);
          if (i < S / 2) wd.piece(S / 2 + i, to);          // (early, so that the synchronisation point does not wait for the writes)
        });
      } else {
        wd.read(raw + w_codes + w_lane, raw + w_scales, lane);
#pragma unroll
        for (int i = 0; i < S; ++i) wd.piece(i, to);
      }
      kt += kStepKeys;
    }
    w.l = w.sum[0];
    // hand-over
    tickets_take(t, s_tk, n_items);
    if constexpr (Halves) {
      join_halves<D>(w, part, lane, smem + (part == 0 ? L::kPrefill : 0) + wave * Joined<D>::kWave);
      if (part == 0) prefill_store<D>(a, H, it, wr, w, Hq, wave, lane, stage);
      break;
    }
    if (!next_ok) {
      prefill_store<D>(a, H, it, wr, w, Hq, wave, lane, stage);
      break;
    }
    const HfxItem item_c = items[t.cur];
    const HfxItem item_n = items[t.nxt < n_items ? t.nxt : t.cur];
    bf16x8 qx[D / 64][4];
    query_load4<D>(qx, nx.q, nx.q_row0, nx.q_last, Hq, n, j);
    if (!in_next) ask_start(nx);
    in_next = false;
    nx = next_item(item_n);
    next_ok = t.nxt < n_items && item_n.type == HFX_ITEM_PREFILL;
    prefill_store<D>(a, H, it, wr, w, Hq, wave, lane, stage);
    query_rows4<D>(w, qx);
    item_start(item_c);
  }
  __builtin_amdgcn_s_setprio(0);
  __syncthreads();     // every wavefront is done with the ring before the LDS is used for anything else
}

// Steps whose decode work outweighs their prefill work have a queue that keeps the two on different CUs, for the sake of the decodes' stream of a bf16 pool.
// Here that stream is a quarter as long, and where every item is dealt (two a workgroup) what counts is that the workgroups end together: prefill
// items go first, the largest at the front, and the decode items behind them.  (us, the queue's own order and this one: 21 decodes and a 300-token prompt 19.9,
// 18.5; 32 decodes and 777 tokens 38.3, 30.8; 64-wide heads, 48 decodes and three chunks 40.9, 38.3; 32 decodes of 8k to 64k tokens and 1024
// rows behind 8192 on 8 / 1 heads 149, 80.  Queues that go on behind the dealt items keep their order: with queries of two numbers 200 decodes and two chunks took 296, 327.)
//
// Place in the queue of item number `rank` in that order.  The queue gives the prefill items the workgroups of the first `pair` CUs, in both rounds, the
// decode items the others, and what is left over follows.  Any two ranks have different places, whatever the queue is.
__device__ __forceinline__ int place_by_kind(int rank, int n_prefill, int n_decode) {
  constexpr int kHalf = HFX_PLAN_WGS / 2;
  const int pair = min((n_prefill + 3) / 4, kHalf / 2);
  const bool prefill = rank < n_prefill;
  const int own = prefill ? rank : rank - n_prefill, others = prefill ? n_decode : n_prefill, width = prefill ? pair : kHalf - pair;
  int i = own, at = prefill ? 0 : pair;
  if (i >= 2 * width) {
    i -= 2 * width;
    at += HFX_PLAN_WGS;
  }
  if (i >= width) {
    i -= width;
    at += kHalf;
  }
  // (past the two rounds, or where the others have run out before: behind all of them)
  return own < 4 * width && at + i - own <= others ? at + i : others + own;
}

// Past: the pages of decode items go past the caches (the planner's stream_mx).
template <int D, bool Past>
__global__ __launch_bounds__(HFX_WG_THREADS, 2) void mixed_attention_mx_kernel(const HfxHeader hdr, const int by_kind, const char* __restrict__ desc,
                                                                                int* __restrict__ ctrl,
                                                                                const __bf16* __restrict__ q, const __bf16* __restrict__ pool,
                                                                                float* __restrict__ ws, __bf16* __restrict__ out) {
  KArgs a;
  a.desc = desc;
  a.q = q;
  a.pool = pool;
  a.ws = ws;
  a.out = out;
  __shared__ __attribute__((aligned(1024))) char smem[Smem4<D>::kBytes];
  __shared__ int s_tk[2];
  __shared__ __attribute__((aligned(16))) int s_ids[4 * 128];            // page ids of steps to come (prefill_run4)
  const HfxHeader* H = &hdr;
  const HfxItem* items = reinterpret_cast<const HfxItem*>(a.desc + H->off_items);
  const int n_items = H->n_items;
  Tickets t = tickets_start(H, a.desc);
  if (by_kind) {
    if (t.cur < n_items) t.cur = place_by_kind(t.cur, H->n_prefill_items, H->n_decode_items);
    if (t.nxt < n_items) t.nxt = place_by_kind(t.nxt, H->n_prefill_items, H->n_decode_items);
  }
  while (t.cur < n_items) {
    if (items[t.cur].type == HFX_ITEM_DECODE) decode_run4<D, Past>(a, H, items, n_items, t, s_tk, ctrl, smem);
    else prefill_run4<D, false>(a, H, items, n_items, t, s_tk, ctrl, smem, s_ids);
  }
  queue_done(H, ctrl);
}

// Steps of prompts alone that have fewer items than the chip has CUs: a workgroup an item, of twice the wavefronts.
template <int D>
__global__ __launch_bounds__(2 * HFX_WG_THREADS, 2) void prompts_attention_mx_kernel(const HfxHeader hdr, const char* __restrict__ desc, const __bf16* __restrict__ q,
                                                                                    const __bf16* __restrict__ pool, float* __restrict__ ws,
                                                                                    __bf16* __restrict__ out) {
  KArgs a;
  a.desc = desc;
  a.q = q;
  a.pool = pool;
  a.ws = ws;
  a.out = out;
  __shared__ __attribute__((aligned(1024))) char smem[2 * Smem4<D>::kPrefill];
  __shared__ __attribute__((aligned(16))) int s_ids[2 * 4 * 128];
  const HfxHeader* H = &hdr;
  Tickets t;
  t.cur = (int)blockIdx.x;
  t.nxt = 0x7fffffff;
  t.parity = 0;
  t.queue = t.own = false;
  t.order = nullptr;
  const int part = uniform((int)threadIdx.x / HFX_WG_THREADS);
  prefill_run4<D, true>(a, H, reinterpret_cast<const HfxItem*>(a.desc + H->off_items), H->n_items, t, nullptr, nullptr, smem + part * Smem4<D>::kPrefill,
                        s_ids + part * 4 * 128);
}

hipError_t max_resident_workgroups_mx(int head_dim, int* per_cu) {
  if (head_dim == 128) return hipOccupancyMaxActiveBlocksPerMultiprocessor(per_cu, mixed_attention_mx_kernel<128, false>, HFX_WG_THREADS, 0);
  return hipOccupancyMaxActiveBlocksPerMultiprocessor(per_cu, mixed_attention_mx_kernel<64, false>, HFX_WG_THREADS, 0);
}

hipError_t launch_mixed_attention_mx(const HfxHeader& h, int grid, void* desc, const void* q, const void* pool, void* ws, void* out, hipStream_t stream) {
  HfxHeader hb = h;
  const bool by_kind = !h.deal_balanced && h.n_prefill_items > 0 && h.n_items <= kDealtTickets * grid;
  if (by_kind) hb.deal_balanced = 1;
  const HfxHeader hk = launch_header(hb, grid);
  const char* d = static_cast<const char*>(desc);
  int* ctrl = reinterpret_cast<int*>(static_cast<char*>(desc) + h.off_ctrl);
  const __bf16* qp = static_cast<const __bf16*>(q);
  const __bf16* pp = static_cast<const __bf16*>(pool);
  float* wp = static_cast<float*>(ws);
  __bf16* op = static_cast<__bf16*>(out);
  // Prompts alone whose items leave half of the CUs' wavefronts idle: an item goes to eight wavefronts where there are keys enough to share (32 / 8 heads, us, with four
  // and with eight: 777 tokens 20.5, 18.6; 400 14.6, 14.1; 64 behind 500 16.5, 15.9; 200 11.4, 11.3; but 100 9.4, 9.8 and 40 8.3, 9.5; 64-wide heads, 700 behind
  // 300 18.9, 15.7).
  if (h.n_decode_items == 0 && h.n_items <= HFX_PLAN_WGS / 2 && h.max_ctx_len > 4 * kStepKeys) {
    const hipError_t e = launch(h.head_dim == 128 ? prompts_attention_mx_kernel<128> : prompts_attention_mx_kernel<64>, dim3((unsigned)h.n_items),
                                2 * HFX_WG_THREADS, stream, hk, d, qp, pp, wp, op);
    return e != hipSuccess ? e : launch_merge(h, desc, ws, out, stream);
  }
  void (*const kernels[])(HfxHeader, int, const char*, int*, const __bf16*, const __bf16*, float*, __bf16*) = {
      mixed_attention_mx_kernel<64, false>, mixed_attention_mx_kernel<64, true>, mixed_attention_mx_kernel<128, false>, mixed_attention_mx_kernel<128, true>};
  const hipError_t e = launch(kernels[(h.head_dim == 128 ? 2 : 0) + (h.stream_mx ? 1 : 0)], dim3(grid), HFX_WG_THREADS, stream, hk, (int)by_kind, d, ctrl, qp, pp, wp, op);
  return e != hipSuccess ? e : launch_merge(h, desc, ws, out, stream);
}

}  // namespace hfx
