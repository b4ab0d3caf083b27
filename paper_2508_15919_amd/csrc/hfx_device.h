// Device code shared by the kernels over the bf16 page pool and over the 4-bit one: the work queue's tickets, lane exchanges, the
// masks and the softmax of a prefill stage, result stores, and how kernels are launched.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hfx_desc.h"

namespace hfx {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

#define NEG_INF (-__builtin_inff())

struct KArgs {
  const char* desc;      // device descriptor blob (read-only here; the control words go through `ctrl`)
  const __bf16* q;       // [T][Hq][D]
  const __bf16* pool;    // [pages][Hkv][2][16*D]
  float* ws;             // split partials
  __bf16* out;           // [T][Hq][D]
};

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ bf16x8 ld16(const __bf16* p) { return *reinterpret_cast<const bf16x8*>(p); }

// `x` where keep, -inf elsewhere, as a select on the bit pattern: the scores of masked keys may be
// NaN (unused slots hold anything), and attention is compiled with -fno-honor-nans, under which a
// floating-point select of a NaN is not defined.
__device__ __forceinline__ float keep_or_neg_inf(float x, bool keep) {
  const unsigned u = keep ? __builtin_bit_cast(unsigned, x) : 0xff800000u;
  return __builtin_bit_cast(float, u);
}

// Exchange between lane n and lane n ^ 32 with the swap instruction gfx950 has for it (the upper half
// of one register against the lower half of another); a shuffle would go through LDS and put
// its latency, and a wait for every LDS read in flight, into the softmax of every stage.
// swap32(x): {x of the lower-half lane of the pair, x of its upper-half lane}, in both lanes.
// The copies in and out are hidden from the optimizer, which otherwise folds the swap of a value
// with itself, and whatever combines its two results, into the value.
struct Pair32 {
  float lo, hi;
};
__device__ __forceinline__ Pair32 swap32(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  unsigned u2 = u;
  asm volatile("" : "+v"(u2));
  const auto r = __builtin_amdgcn_permlane32_swap(u, u2, false, false);
  unsigned a = r[0], b = r[1];
  asm volatile("" : "+v"(a), "+v"(b));
  Pair32 p;
  p.lo = __builtin_bit_cast(float, a);
  p.hi = __builtin_bit_cast(float, b);
  return p;
}
__device__ __forceinline__ float max_xor32(float x) {
  const Pair32 p = swap32(x);
  return fmaxf(p.lo, p.hi);
}
__device__ __forceinline__ float sum_xor32(float x) {
  const Pair32 p = swap32(x);
  return p.lo + p.hi;
}

// zero the elements e >= nv of an 8-element bf16 vector (nv may be <= 0 or >= 8)
__device__ __forceinline__ bf16x8 keep_first(bf16x8 v, int nv) {
  const unsigned bits = (1u << min(max(nv, 0), 8)) - 1u;
  u32x4 u = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int lo = (int)(bits << (31 - 2 * w)) >> 31, hi = (int)(bits << (30 - 2 * w)) >> 31;   // all ones where kept
    u[w] &= __builtin_amdgcn_perm((unsigned)hi, (unsigned)lo, 0x05040100u);
  }
  return __builtin_bit_cast(bf16x8, u);
}

// s_waitcnt vmcnt(N) alone (gfx9 encoding: vmcnt in bits 3:0 and 15:14, the other counters left at their maxima)
#define HFX_WAIT_VMCNT(N) __builtin_amdgcn_s_waitcnt(((N) & 15) | (((N) >> 4) << 14) | (7 << 4) | (15 << 8))

// Work-queue tickets of a workgroup.  It holds the item it is processing and the item after it
// (whose record is therefore known while the current item runs, so that a prefill item can
// request the first tiles of its successor before it ends).  The ticket after those is asked
// for by thread 0 shortly before the current item ends, published through LDS ahead of a
// barrier the item crosses anyway, and taken at the hand-over.  Asking late matters: a
// workgroup that asks at the start of a long item reserves work it will not touch for a long
// time, and in a step with about three items per workgroup that left half the chip idle while
// the other half worked through its reservations.  The first two tickets of a workgroup are its
// index plus 0 and 1 grids (the queue is in descending cost, so this deals the largest items
// out evenly, and a workgroup starts without a round trip to a counter).  Where that deals all items, no counter
// is touched: atomics on one address from all over the chip take about 14 ns each, one after the other, and 256 workgroups that
// ask for a ticket and report their end spend 7 us on them (4 decodes of 100 to 2000 tokens 13.7 us, 12.7 without; a prompt of 777
// tokens 17.5 and 16.7; 300 rows behind 3000 on 64-wide heads 25.7 and 23.5; 512 workgroups of one short decode piece each 21.2
// and 12.2).
constexpr int kDealtTickets = 2;
struct Tickets {
  int cur, nxt;
  int parity;
  bool queue;        // there may be items behind the next one
  bool own;          // ... and among them some for this die (first wavefront)
  const int* order;  // queue position -> item, if the queue does not hold the items in their order
};

// The dealt tickets of a step whose queue is in descending cost.  Workgroups b and b + 256 share a CU, so
// dealt straight the largest item meets the 256th largest on one CU, the smallest two of the round
// meet on another, and the second round gives the workgroups with the largest items one more.  Here the
// first round runs up and then down the queue -- with fewer items than workgroups, the CUs that stay with
// one workgroup get the largest -- and the second runs down, both within the positions that are equal
// modulo the number of classes.  (2500 tokens on 32/8 heads 66 -> 57 us, 4096 tokens 134 -> 126 us; nothing on queues of
// many items.)
// `mode` is set by the launch: the grid is HFX_PLAN_WGS (1), or more than half of that, one item each (2).
__device__ __forceinline__ void deal_balanced(Tickets& t, int mode, int n_items) {
  constexpr int kHalf = HFX_PLAN_WGS / 2, kLow = HFX_QUEUE_CLASSES - 1;
  const int b = (int)blockIdx.x;
  if (mode == 1) {
    if (b >= kHalf) t.cur = kHalf + (((HFX_PLAN_WGS - 1 - b) & ~kLow) | (b & kLow));
    t.nxt = HFX_PLAN_WGS + (((HFX_PLAN_WGS - 1 - t.cur) & ~kLow) | (b & kLow));
  } else {
    const int paired = n_items - kHalf;           // CUs with two workgroups
    if (b >= kHalf) t.cur = n_items - 1 - (b - kHalf);
    else t.cur = b < paired ? kHalf - paired + b : b - paired;
  }
}

// Queue positions past the dealt ones, up to die_items, fall into HFX_QUEUE_CLASSES classes, position p into class
// p % HFX_QUEUE_CLASSES, each with a counter of its own; those behind are shared.  A workgroup asks the counter of the class of its index and, once that class
// is empty, the shared one.  Workgroups are placed on the chip's dies round-robin by index, so a class is served by the workgroups of
// one die, and the planner puts items that read the same keys into one class: they then share
// that die's L2.  The shared end of the queue, the smallest items, is what lets the dies end together.  Without die_items all positions are shared.
//
// What bounds the counters: atomics and atomic loads on one line from all over the chip are served one after the other, 14 ns
// each.  With all counters on one line, and every workgroup whose class was empty reading the eight of them one by one to find work elsewhere, the end
// of a step with classes took 40 to 90 us, whatever the step (17 short prompts of each of six tasks 87 us from one queue and 185 with classes);
// with a line each, and one load for all eight, still 4 to 6 us, which the shared end does not cost (31 short prompts on 8/1 heads 46 us and 40).
// A workgroup that knows the queue to be empty asks no more, and workgroups report their end by class.  The prefill-heavy mixed step, which has classes,
// took 858 us before and 818 after.
//
// Thread 0 asks for one more ticket; the reply, an offset from the dealt tickets or from the shared positions, goes to
// tickets_publish.  The other lanes keep what `pending` held: a select on it would
// wait for the reply, and with it for everything in flight, wherever the compiler places it.
__device__ __forceinline__ void tickets_reserve(const Tickets& t, int& pending, int* ctrl) {
  if (!t.queue) return;
  int word = t.own ? HFX_CTRL_TICKETS((int)blockIdx.x & (HFX_QUEUE_CLASSES - 1)) : HFX_CTRL_SHARED;
  asm volatile("" : "+s"(word));      // (the address is formed here and not kept in vector registers)
  if (threadIdx.x == 0) pending = atomicAdd(ctrl + word, 1);
}
// The first wavefront turns the reply into an item and thread 0 puts it into LDS (two slots alternate, so one barrier per hand-over is
// enough).
__device__ __forceinline__ void tickets_publish(Tickets& t, int pending, int* s_tk, int* ctrl, const HfxHeader* H) {
  if (!t.queue || uniform((int)threadIdx.x >> 6) != 0) return;
  const int dealt = kDealtTickets * (int)gridDim.x, die_items = (int)H->die_items, shared = max(dealt, die_items);
  int pos = uniform(pending);
  if (t.own) {
    pos = dealt + pos * HFX_QUEUE_CLASSES + ((int)blockIdx.x & (HFX_QUEUE_CLASSES - 1));
    if (pos >= die_items) {
      t.own = false;
      int word = HFX_CTRL_SHARED, reply = 0;
      asm volatile("" : "+s"(word));
      if (threadIdx.x == 0) reply = atomicAdd(ctrl + word, 1);
      pos = shared + uniform(reply);
    }
  } else {
    pos += shared;
  }
  if (t.order && pos < H->n_items) pos = t.order[pos];
  if (threadIdx.x == 0) s_tk[t.parity] = pos;
}
// ... after a workgroup barrier that follows tickets_publish.  Counters only grow: once a ticket is past the end, so are all later ones.
__device__ __forceinline__ void tickets_take(Tickets& t, int* s_tk, int n_items) {
  t.cur = t.nxt;
  t.nxt = 0x7fffffff;
  if (t.queue) t.nxt = uniform(s_tk[t.parity]);
  t.queue = t.nxt < n_items;
  t.parity ^= 1;
}

// The first tickets of a workgroup.
__device__ __forceinline__ Tickets tickets_start(const HfxHeader* H, const char* desc) {
  const int n_items = H->n_items;
  Tickets t;
  t.cur = (int)blockIdx.x;
  t.nxt = (int)(blockIdx.x + gridDim.x);
  if (H->deal_balanced) deal_balanced(t, (int)H->deal_balanced, n_items);
  t.order = nullptr;
  if (H->off_queue) {
    t.order = reinterpret_cast<const int*>(desc + H->off_queue);
    if (t.cur < n_items) t.cur = t.order[t.cur];
    if (t.nxt < n_items) t.nxt = t.order[t.nxt];
  }
  t.own = (int)H->die_items > kDealtTickets * (int)gridDim.x;
  t.parity = 0;
  t.queue = n_items > kDealtTickets * (int)gridDim.x;
  return t;
}

// The end of a workgroup: the last one of a launch that used the queue's counters restores them.
__device__ __forceinline__ void queue_done(const HfxHeader* H, int* ctrl) {
  const int n_items = H->n_items;
  // the ticket fetched last is never used; it must have reached the counter before this
  // workgroup reports itself finished, or it could land after the reset below
  HFX_WAIT_VMCNT(0);
  asm volatile("" ::: "memory");
  if (n_items > kDealtTickets * (int)gridDim.x && threadIdx.x == 0) {
    // the workgroups of a class count themselves, and its last one the classes
    const int cls = (int)blockIdx.x & (HFX_QUEUE_CLASSES - 1);
    if (atomicAdd(ctrl + HFX_CTRL_DONE(cls), 1) == ((int)gridDim.x - cls + HFX_QUEUE_CLASSES - 1) / HFX_QUEUE_CLASSES - 1 &&
        atomicAdd(ctrl + HFX_CTRL_DONE(HFX_QUEUE_CLASSES), 1) == min((int)gridDim.x, HFX_QUEUE_CLASSES) - 1) {
      for (int c = 0; c < HFX_QUEUE_CLASSES; ++c) {
        atomicExch(ctrl + HFX_CTRL_TICKETS(c), 0);
        atomicExch(ctrl + HFX_CTRL_DONE(c), 0);
      }
      atomicExch(ctrl + HFX_CTRL_SHARED, 0);
      atomicExch(ctrl + HFX_CTRL_DONE(HFX_QUEUE_CLASSES), 0);
    }
  }
}

// What a wavefront derives from a decode item: its kv-head, its share of the page pairs, and the
// pages of its first two pairs.
struct DecodeWave {
  int g;          // kv-head
  int step;       // pages between two pairs of this wavefront
  int pp, pe;     // next page (pair-aligned) and end of the item's page range
  int tend;       // tokens of the context that the item may see (end of its range or of the context)
  int bt0, last_page;
  int a0, a1, b0, b1;   // page ids of the pair at pp and of the one after it
};

__device__ __forceinline__ int decode_page(const int* __restrict__ bt, const DecodeWave& d, int i) {
  return bt[d.bt0 + (i < d.last_page ? i : d.last_page)];
}

__device__ __forceinline__ DecodeWave decode_wave(const int* __restrict__ bt, const HfxItem& it, int wave) {
  DecodeWave d;
  const int HW = it.hn, sh = HW >> 1;      // 1, 2 or 4, and its logarithm
  d.g = it.h0 + (wave & (HW - 1));
  d.step = 8 >> sh;
  d.pp = it.kb + 2 * (wave >> sh);
  d.pe = it.ke;
  d.tend = min(it.ke * HFX_PAGE, it.rq.ctx_len);
  d.bt0 = it.rq.bt_start;
  d.last_page = it.rq.n_pages - 1;
  d.a0 = decode_page(bt, d, d.pp);
  d.a1 = decode_page(bt, d, d.pp + 1);
  d.b0 = decode_page(bt, d, d.pp + d.step);
  d.b1 = decode_page(bt, d, d.pp + d.step + 1);
  return d;
}

// Combines a decode item's wavefronts and stores the result: wavefront partials (o[b][v] is dimension 16b + 4j + v of q-head n of the
// wavefront's kv-head, m and l its reference exponent and running sum) go through LDS, and the token partitions of each head are joined into
// normalised bf16 rows or, where the item is one split of a group, into (m, l, acc) partial rows.  A wavefront's 16 rows of D + 4 floats lie Stride bytes
// behind those of the one before it, or (0) directly.
constexpr int decode_part_bytes(int D) { return 4 * 16 * (D + 4) * 4; }     // LDS that they take without gaps
template <int D, int Stride = 0>
__device__ __forceinline__ void decode_store(const KArgs& a, const HfxHeader* H, const HfxItem& it, const f32x4* o, float m, float l, int Hq, int G,
                                             int tid, int wave, int n, int j, char* smem) {
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);

  constexpr int PS = D + 4;
  auto part = [&](int w, int head) {
    if constexpr (Stride == 0) return reinterpret_cast<float*>(smem) + (w * 16 + head) * PS;
    else return reinterpret_cast<float*>(smem + w * Stride) + head * PS;
  };
  if (n < G) {
    float* dst = part(wave, n);
#pragma unroll
    for (int b = 0; b < D / 16; ++b) *reinterpret_cast<f32x4*>(dst + b * 16 + 4 * j) = o[b];
    if (j == 0) {
      dst[D] = m;
      dst[D + 1] = l;
    }
  }
  __syncthreads();

  // combine the TW token partitions of each head; row = hwi * G + hh
  const int HW = it.hn, TW = 4 >> (HW >> 1);
  const int rows = HW * G;
  float* ws_acc = a.ws;
  float* ws_ml = reinterpret_cast<float*>(reinterpret_cast<char*>(a.ws) + H->ws_off_ml);
  constexpr int C4 = D / 4;
  for (int idx = tid; idx < rows * C4; idx += HFX_WG_THREADS) {
    const int row = idx / C4, d4 = (idx % C4) * 4;
    const int hwi = row / G, hh = row % G;
    float mm = NEG_INF;
    for (int tt = 0; tt < TW; ++tt) mm = fmaxf(mm, part(tt * HW + hwi, hh)[D]);
    float ll = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int tt = 0; tt < TW; ++tt) {
      const float* src = part(tt * HW + hwi, hh);
      const float wgt = fast_exp2(src[D] - mm);
      ll += src[D + 1] * wgt;
      acc += *reinterpret_cast<const f32x4*>(src + d4) * wgt;
    }
    if (it.group < 0) {
      const float inv = 1.0f / ll;
      bf16x4 ob;
#pragma unroll
      for (int e = 0; e < 4; ++e) ob[e] = (__bf16)(acc[e] * inv);
      *reinterpret_cast<bf16x4*>(a.out + ((long)it.rq.q_start * Hq + it.h0 * G + row) * D + d4) = ob;
    } else {
      const long pr = (long)it.slot_row + row;
      *reinterpret_cast<f32x4*>(ws_acc + pr * D + d4) = acc;
      if (d4 == 0) {
        ws_ml[pr * 2] = mm;
        ws_ml[pr * 2 + 1] = ll;
      }
    }
  }
}

// Workgroup barrier of the ring: this wavefront's LDS reads are done.  The compiler may move loads across
// the barrier builtin, which claims no memory effect, so the empty asm on both sides holds them.
__device__ __forceinline__ void ring_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

#define HFX_M_NONE (-3.402823466e38f)   // reference exponent before the first stage: lower than any score

// Weights of 16 scores against reference exponent m, and their sum (fp32, four partial sums; plain
// adds, because the two-element dot-product instruction does not issue while a matrix instruction
// executes).
__device__ __forceinline__ float weights(const f32x16& s, float sl2, float m, bf16x8* pb) {
  float ps[4];
#pragma unroll
  for (int v = 0; v < 16; v += 2) {
    const float p0 = fast_exp2(__builtin_fmaf(s[v], sl2, -m));
    const float p1 = fast_exp2(__builtin_fmaf(s[v + 1], sl2, -m));
    if (v < 8) ps[v >> 1] = p0 + p1;
    else ps[(v >> 1) & 3] += p0 + p1;
    pb[v >> 3][v & 7] = (__bf16)p0;
    pb[v >> 3][(v & 7) + 1] = (__bf16)p1;
  }
  return (ps[0] + ps[1]) + (ps[2] + ps[3]);
}

// Masks the scores of keys that this lane's row must not see (those past `pos`): s[v] is key
// key0 + (v>>3)*16 + (v&7)   (key0 already includes the lane's 8j).  The visible ones are the first few
// of the 16, so one bit mask says which; selects on compares would hold 16 condition masks at once.  Masked
// scores may be NaN (unused slots hold anything), hence integer operations.
__device__ __forceinline__ void mask_scores(f32x16& s, int pos, int key0) {
  const int d = pos - key0;
  const int visible = min(max(d + 1, 0), 8) + min(max(d - 15, 0), 8);
  const int bits = (1 << visible) - 1;
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const unsigned keep = (unsigned)((int)((unsigned)bits << (31 - v)) >> 31);     // all ones where visible
    const float x = s[v];            // (a bit cast of the vector element itself would read element 0)
    s[v] = __builtin_bit_cast(float, (__builtin_bit_cast(unsigned, x) & keep) | (0xff800000u & ~keep));
  }
}

// Maximum over the 32 scores of this lane's row (16 here, 16 in lane ^ 32), in the base-2 domain.
__device__ __forceinline__ float row_max(const f32x16& s, float sl2) {
  float mx = fmaxf(s[0], s[1]);
#pragma unroll
  for (int v = 2; v < 16; v += 2) mx = fmaxf(fmaxf(mx, s[v]), s[v + 1]);   // v_max3_f32
  return max_xor32(mx) * sl2;
}

// m is the reference exponent of an item's running sums: the maximum of its first stage to begin
// with.  A stage's weights are taken against the m at hand; only when some lane's 16 weights sum to
// more than 2^8 -- its maximum has grown well over m -- is m raised to the maximum, O and l rescaled,
// and the weights taken again.  So the common stage needs neither the maximum nor the exchange
// between the lanes of a row, and no weight exceeds 2^8.
template <int D, class Wave>
__device__ __forceinline__ void settle_weights(Wave& w, const f32x16& s, bf16x8* pb, float sum, float sl2) {
  if (__builtin_expect(__any(sum > 256.0f), 0)) {
    const float mx = fmaxf(w.m, row_max(s, sl2));
    const float alpha = fast_exp2(w.m - mx);
    w.l *= alpha;
#pragma unroll
    for (int b = 0; b < D / 32; ++b) w.o[b] *= alpha;
    w.m = mx;
    sum = weights(s, sl2, w.m, pb);
  }
  w.l += sum;
}

// Which scores have their weights formed behind which matrix instruction: number i of the value phase takes scores
// [values[i], values[i + 1]) of the next stage, number i of the score phase [scores[i], scores[i + 1]) of the present one.
// The first value instruction takes none, because the scores of the next stage come out of the matrix instruction just before it,
// and the last score instruction none, so that the sum of the weights is known by the end of its phase.
template <int D>
struct Share;
template <>
struct Share<128> {
  static constexpr int values[9] = {0, 0, 1, 2, 3, 5, 6, 7, 8}, scores[9] = {8, 9, 10, 11, 13, 14, 15, 16, 16};
};
template <>
struct Share<64> {
  static constexpr int values[5] = {0, 2, 4, 6, 8}, scores[5] = {8, 10, 12, 14, 16};
};

// The weights of a stage on their way.  A pair is summed and rounded one portion after its exponentials, so that nothing
// waits for an exponential just issued.  The empty asm statements hold the results where they are formed: left to itself
// the compiler puts the sums and roundings of all portions behind the last one.
struct Weighing {
  float p[16], ps[4];
  unsigned pw[8];            // rounded pairs

  __device__ __forceinline__ void finish(int i) {
    const float t = p[2 * i] + p[2 * i + 1];
    if (i < 4) ps[i] = t;
    else ps[i & 3] += t;
    const bf16x2 r = {(__bf16)p[2 * i], (__bf16)p[2 * i + 1]};
    pw[i] = __builtin_bit_cast(unsigned, r);
    asm volatile("" : "+v"(pw[i]), "+v"(ps[i & 3]));
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
  __device__ __forceinline__ float sum() const { return (ps[0] + ps[1]) + (ps[2] + ps[3]); }
};

struct NoCopy {
  __device__ __forceinline__ void operator()(int) const {}
};

// What a wavefront derives from a prefill item: its q-head and rows, and the key ranges that
// decide whether a stage is worked on and whether it needs masks.
struct WaveRows {
  int head, row0;             // q-head and first chunk row
  int wave_kend, wave_pmin;
};

__device__ __forceinline__ WaveRows wave_rows(const HfxItem& it, int wave) {
  WaveRows r;
  // hn is 1, 2 or 4 (a division would take the vector unit, and with it all that follows from its result)
  r.head = it.h0 + (wave & (it.hn - 1));
  r.row0 = it.row0 + (wave >> (it.hn >> 1)) * HFX_WAVE_ROWS;
  const int p = it.rq.ctx_len - it.rq.q_len;
  r.wave_kend = r.row0 < it.rq.q_len ? min(it.ke, p + min(r.row0 + HFX_WAVE_ROWS, it.rq.q_len)) : 0;   // keys >= this: nothing to do
  r.wave_pmin = p + r.row0;                                                            // keys <= this are visible to every row
  return r;
}

// Result of a finished prefill item (accumulators w.o, reference exponent w.m, sum w.l): normalised bf16 rows, or (m, l, acc) partial rows when the item is one split of a group.
// A lane holds 4-dimension pieces of its own row, so stored straight from the registers every
// instruction would touch 32 rows with 16 bytes each, and the write path takes one request per
// (instruction, line).  The bf16 rows therefore go through `stage` (2 KB of LDS owned by this
// wavefront, 32 dimensions of its 32 rows at a time) and leave in 64-byte pieces, 16 rows per
// instruction.  The 16-byte units of a row are permuted by the row number, and the two 8-byte halves of a unit
// change places in rows 16-31, so that writes and reads spread over all LDS banks.
template <int D, class Wave>
__device__ __forceinline__ void prefill_store(const KArgs& a, const HfxHeader* H, const HfxItem& it, const WaveRows& r,
                                              const Wave& w, int Hq, int wave, int lane, char* stage) {
  // o[b][v] is dimension 32b + (v>>2)*8 + 4j + (v&3) of chunk row row0 + (lane & 31)
  const float lsum = sum_xor32(w.l);
  // The lane's parts of the destination addresses are formed here, per call: left visible, the
  // compiler hoists them out of the item loop, runs out of registers and parks them in scratch
  // memory, and the reload at every hand-over waits for every load the stage ring has in flight.
  asm volatile("" : "+v"(lane));
  const int n = lane & 31, j = lane >> 5;
  if (it.group < 0) {
    const float inv = 1.0f / lsum;
    const int row0 = r.row0;
    const int rr = lane >> 2, u = lane & 3;      // read-back: row rr + 16i, 16-byte unit u
    __bf16* dst = a.out + (((long)it.rq.q_start + row0 + rr) * Hq + r.head) * D + u * 8;
    char* wr = stage + n * 64 + (j ^ (n >> 4)) * 8;
    const char* rd = stage + rr * 64 + ((u ^ ((rr >> 2) & 3)) * 16);
    // LDS serves a wavefront's accesses in order, so the next 32 dimensions are written while the lines of these are on
    // their way back
    u32x4 line[D / 32][2];
#pragma unroll
    for (int b = 0; b < D / 32; ++b) {
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        bf16x4 ob;
#pragma unroll
        for (int e = 0; e < 4; ++e) ob[e] = (__bf16)(w.o[b][q4 * 4 + e] * inv);
        *reinterpret_cast<bf16x4*>(wr + ((q4 ^ ((n >> 2) & 3)) * 16)) = ob;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) line[b][i] = *reinterpret_cast<const u32x4*>(rd + i * 1024);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (row0 + rr + 16 * i < it.rq.q_len) {
#pragma unroll
        for (int b = 0; b < D / 32; ++b) {
          const u32x4 t = line[b][i];
          *reinterpret_cast<u32x4*>(dst + (long)i * 16 * Hq * D + b * 32) = i == 1 ? u32x4{t[2], t[3], t[0], t[1]} : t;
        }
      }
  } else {
    float* ws_acc = a.ws;
    float* ws_ml = reinterpret_cast<float*>(reinterpret_cast<char*>(a.ws) + H->ws_off_ml);
    const long pr = (long)it.slot_row + wave * HFX_WAVE_ROWS + n;
    float* dst = ws_acc + pr * D + 4 * j;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        f32x4 t = {w.o[b][q4 * 4], w.o[b][q4 * 4 + 1], w.o[b][q4 * 4 + 2], w.o[b][q4 * 4 + 3]};
        *reinterpret_cast<f32x4*>(dst + b * 32 + q4 * 8) = t;
      }
    if (j == 0) {
      ws_ml[pr * 2] = w.m;
      ws_ml[pr * 2 + 1] = lsum;
    }
  }
}

__device__ __forceinline__ int item_stages(const HfxItem& it) { return (int)((unsigned)(it.ke - it.kb + HFX_STAGE_KEYS - 1) / HFX_STAGE_KEYS); }

// Slots [slot0, slot0 + n) of a bf16 value block [D][16 slots] out of token rows in LDS (row stride ld): a thread of 2 D has 8 slots of dimension
// tid / 2; slots outside the run hold what was in LDS and are not stored.
template <int D>
__device__ __forceinline__ void store_value_columns(uint16_t* vblk, const uint16_t* sv, int ld, int tid, int slot0, int n) {
  const int d = tid >> 1, s0 = (tid & 1) * 8;
  uint16_t* dst = vblk + tid * 8;
  const int lo = slot0 - s0, hi = lo + n;     // the run, relative to the thread's slots
  if (lo >= 8 || hi <= 0) return;
  uint16_t x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = sv[(s0 + e) * ld + d];
  if (lo <= 0 && hi >= 8) {
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (uint32_t)x[2 * e] | ((uint32_t)x[2 * e + 1] << 16);
    *reinterpret_cast<u32x4*>(dst) = v;
  } else {
    // part of them: two at a time where both belong to the run
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int a = 2 * w, b = 2 * w + 1;
      const bool in_a = a >= lo && a < hi, in_b = b >= lo && b < hi;
      if (in_a && in_b) *reinterpret_cast<uint32_t*>(dst + a) = (uint32_t)x[a] | ((uint32_t)x[b] << 16);
      else if (in_a) dst[a] = x[a];
      else if (in_b) dst[b] = x[b];
    }
  }
}

// Launches a kernel without dynamic LDS and answers for this launch alone.  (hipGetLastError() names the last error of any
// earlier call of the thread: with one that the caller had not read yet, work was enqueued and HFX_ERR_DEVICE returned.)  The error
// of a launch that fails is read here, because the caller learns of it; an older one stays the caller's to read.
template <typename... P, typename... A>
static hipError_t launch(void (*kernel)(P...), dim3 grid, unsigned threads, hipStream_t stream, const A&... args) {
  static_assert(sizeof...(P) == sizeof...(A), "one value for each parameter");
  auto call = [&](P... values) {
    void* address[] = {(void*)&values...};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), address, 0, stream);
  };
  const hipError_t e = call(args...);
  if (e != hipSuccess) (void)hipGetLastError();
  return e;
}
}  // namespace hfx
