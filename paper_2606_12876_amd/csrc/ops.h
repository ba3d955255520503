// Arguments and launchers of the operators between the layers (rms norm, 4-bit weights, paged
// attention, cache pages). Arguments are already validated.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/aqmb.h"

namespace aqmb {

struct NormArgs {
  const void* x;
  const void* residual;   // or null, with residual_out
  void* residual_out;
  const void* weight;
  void* y;
  float* scales;          // F8 and I8 outputs only
  int64_t x_stride, residual_stride, y_stride;
  float weight_offset, eps;
  int rows, cols, y_dtype, scale_group;
};
hipError_t launch_rms_norm(const NormArgs& a, aqmb_dtype dtype, hipStream_t st);

// A layer of 4-bit weights. Tiles of 16 rows x 128 inputs (1 KiB): lane l of a wave owns the 16 bytes
// 16 l.. of a tile, row l % 16; its dword s holds inputs 32 s + 8 (l / 16) + {0, 2, 4, 6, 1, 3, 5, 7}
// in nibbles 0..7, the order in which the kernel's masks take the nibbles out.
constexpr int kW4Rows = 16, kW4Cols = 128;
struct W4 {
  uint32_t magic;
  aqmb_w4_desc d;
  int device, n_cu;
  int n_rt, n_kt;          // row tiles, input tiles
  unsigned char* tiles;    // [n_rt][n_kt][1024]
  uint16_t* scales;        // [n_rt][n_kt][4 rows / 4][128 / g][4] fp16, 0 in the padding
  unsigned char* zeros;    // the same shape, or one tile's (all 8) if not asymmetric
  bool asymmetric;
};
constexpr uint32_t kW4Magic = 0x41513457u;
hipError_t launch_w4_pack(const W4& L, const uint8_t* weights, const uint16_t* scales, const uint8_t* zeros,
                          hipStream_t st);
hipError_t launch_w4_gemv(const W4& L, const void* x, aqmb_dtype x_dtype, int64_t x_stride, const float* x_scales,
                          int x_scale_group, int batch, void* y, aqmb_dtype y_dtype, int64_t y_stride, hipStream_t st);

struct AttnArgs {
  const void* k;
  const void* v;
  const float* k_scale;
  const float* v_scale;
  int64_t page_stride, head_stride, slot_stride;   // elements of k and v
  int64_t sc_page, sc_head, sc_slot;               // elements of the scales
  int n_pages, page_size;
  const void* q;
  int64_t q_stride;
  const int* table;
  int64_t table_stride;
  const int* lengths;
  int n_seqs, max_length, window;
  float scale;
  void* out;
  int64_t out_stride;
  float* lse;
  int n_heads, n_kv, head_dim;
  int chunk, n_splits;     // positions per workgroup, workgroups along a sequence
  int waves;               // per workgroup
  float* part;             // n_splits > 1: partial sums and (max, sum) pairs
};
// How attention splits a sequence of up to max_length positions (window: as the call).
struct AttnPlan { int chunk, n_splits, waves; size_t bytes; };
AttnPlan attn_plan(int n_heads, int n_kv, int head_dim, int n_seqs, int max_length, int window, int n_cu);
hipError_t launch_attention(const AttnArgs& a, aqmb_dtype dtype, bool f8, hipStream_t st);

hipError_t launch_kv_append(const aqmb_kv_cache& c, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                            aqmb_dtype dtype, const int64_t* slots, int n_tokens, hipStream_t st);
hipError_t launch_kv_copy(const aqmb_kv_cache* caches, int n_caches, const int32_t* src, const int32_t* dst, int n_pairs,
                          hipStream_t st);

}  // namespace aqmb
