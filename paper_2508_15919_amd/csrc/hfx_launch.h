// Host-callable launch helpers implemented next to the kernels (internal).
#pragma once
#include <hip/hip_runtime_api.h>

#include "hfx_desc.h"

namespace hfx {

hipError_t max_resident_workgroups(int head_dim, int* per_cu);
hipError_t launch_mixed_attention(const HfxHeader& header, int grid, void* desc, const void* q, const void* pool,
                                  void* ws, void* out, hipStream_t stream);
// Device address, on the current device, of the library's fixed workspace of HFX_STATIC_WS_BYTES
// (looked up once per device, then cached).
hipError_t static_workspace(void** ptr);
hipError_t launch_gather_kv(const HfxHeader& h, int n_tokens, const void* desc, const void* pool, int request,
                            void* k_out, void* v_out, hipStream_t stream);

hipError_t launch_append_kv(const HfxHeader& h, const void* desc, const void* k_new, const void* v_new, void* pool,
                            hipStream_t stream);

// What the rotating append takes; rows are apart by the strides, in elements.  q, cos_sin: may be null (rot 0).
struct RopeAppend {
  const HfxRun* runs;        // filled in by launch_rope_append, as the next four
  const int* run_pos;
  int n_runs, num_q_heads, num_kv_heads;
  int rot, interleaved;
  const float* cos_sin;      // [position][rot]: cosines, sines
  const uint16_t *q, *k, *v;
  long q_stride, k_stride, v_stride;
  uint16_t* q_out;           // [T][Hq][D]
  void* pool;
};
// Rotates and appends to a bf16 page pool or (four) to a 4-bit one.
hipError_t launch_rope_append(const HfxHeader& h, const void* desc, RopeAppend a, bool four, hipStream_t stream);
hipError_t launch_read_new_kv_mx(const HfxHeader& h, const void* desc, const void* pool, void* k_out, void* v_out, hipStream_t stream);

// What the norm takes.  residual (and with it sum), out and codes (with scales) may be null.
struct RmsNorm {
  const uint16_t *x, *residual, *weight;
  uint16_t *sum, *out;       // [rows][cols]
  int8_t* codes;             // [rows][cols]
  float* scales;
  long x_stride, residual_stride;
  int cols;
  float eps;
  double part;               // 1 / cols; filled in by launch_rms_norm
};
hipError_t launch_rms_norm(RmsNorm a, int rows, hipStream_t stream);

// What the rows' way to 8 bits takes.  times, out and codes (with scales) may be null.
struct QuantiseRows {
  const uint16_t *x, *times;
  uint16_t* out;             // [rows][cols]
  int8_t* codes;             // [rows][cols]
  float* scales;
  long x_stride, times_stride;
  int cols, activation;
};
hipError_t launch_quantise_rows(const QuantiseRows& a, int rows, hipStream_t stream);

// What a product takes: codes [rows][k] and [n][k], their scales, results [rows][n].  bias may be null.
struct MatmulRows {
  const int8_t *codes, *weight;
  const float *scales, *weight_scales;
  const uint16_t* bias;
  void* out;
  long codes_stride, weight_stride, out_stride;
  int rows, n, k;
  bool past;                 // results go past the caches; filled in by launch_matmul_rows
};
hipError_t launch_matmul_rows(MatmulRows a, bool fp32, hipStream_t stream);

// The header as an attention kernel gets it.
HfxHeader launch_header(const HfxHeader& header, int grid);
// The attention launch over a 4-bit page pool; arguments as launch_mixed_attention.
hipError_t max_resident_workgroups_mx(int head_dim, int* per_cu);
hipError_t launch_mixed_attention_mx(const HfxHeader& header, int grid, void* desc, const void* q, const void* pool, void* ws, void* out,
                                      hipStream_t stream);
// The launch that merges what the attention launch split, if it split anything.
hipError_t launch_merge(const HfxHeader& header, const void* desc, const void* ws, void* out, hipStream_t stream);

// Copies a host staging buffer to the device on `stream`: by a kernel from pinned memory to memory of the
// stream's GPU, by the runtime otherwise.  Either way the buffer is read when the stream gets there.
hipError_t upload(const void* host, void* device, size_t bytes, hipStream_t stream);

// Copies pages by (source, destination) id pairs: `n_pairs` of them in `host`, with room for as many in `device`.
hipError_t copy_pages(const void* host, void* device, long n_pairs, unsigned units_per_page, const void* src, void* dst, hipStream_t stream);

}  // namespace hfx
