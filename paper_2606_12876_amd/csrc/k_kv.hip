// Upkeep of a paged key-value cache: writing new tokens (scaled to e4m3 where the cache is 8-bit) and
// copying pages. Pure movement: every byte is read once and written once, so HBM (or, for a decode
// step's few tokens, the launch) bounds both.
#include "device.h"
#include "ops.h"
#include "wave.h"

namespace aqmb {

struct AppendArgs {
  aqmb_kv_cache c;
  int64_t head_stride, slot_stride, sc_head, sc_slot;
  const uint16_t* k;
  const uint16_t* v;
  int64_t k_stride, v_stride;
  const int64_t* slots;
  int64_t pairs;            // tokens * heads
};

struct __attribute__((packed, aligned(2))) Raw16 { uint32_t w[4]; };

// Half a wave per (token, head) and per k or v: lane l owns values 8 l .. 8 l + 7 (head_dim <= 256).
template <int DT, bool F8>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
  const int64_t pair = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (pair >= a.pairs) return;
  const int lane = threadIdx.x % 32;
  const bool is_v = threadIdx.x % 64 >= 32;
  const int64_t token = pair / a.c.n_kv_heads, head = pair % a.c.n_kv_heads;
  const int64_t at = a.slots[token];
  if (at < 0 || at >= (int64_t)a.c.n_pages * a.c.page_size) return;
  const int64_t page = at / a.c.page_size, slot = at % a.c.page_size;
  const bool on = 8 * lane < a.c.head_dim;
  const uint16_t* src = (is_v ? a.v + token * a.v_stride : a.k + token * a.k_stride) + head * a.c.head_dim + 8 * lane;
  const int64_t dst = page * a.c.page_stride + head * a.head_stride + slot * a.slot_stride + 8 * lane;
  void* out = is_v ? a.c.v : a.c.k;
  Raw16 r = {{0, 0, 0, 0}};
  if (on) r = *(const Raw16*)src;
  if constexpr (!F8) {
    if (on) *(u32x4_t*)((uint16_t*)out + dst) = u32x4_t{r.w[0], r.w[1], r.w[2], r.w[3]};
  } else {
    float f[8];
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = DT == AQMB_F16 ? f16lo(r.w[i]) : bf16lo(r.w[i]);
      f[2 * i + 1] = DT == AQMB_F16 ? f16hi(r.w[i]) : bf16hi(r.w[i]);
    }
    // The largest magnitude as bits: infinity and NaN come out above every finite value.
#pragma unroll
    for (int i = 0; i < 8; ++i) big = max(big, __builtin_bit_cast(uint32_t, f[i]) & 0x7FFFFFFFu);
    big = over_lanes<32>(big, max_bits);
    const Scaling scaling = scaling_of(big, 448.f);
    const float mul = scaling.mul;
    uint2 b;
    uint32_t w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * k] * mul, f[4 * k + 1] * mul, 0, false);
      w[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * k + 2] * mul, f[4 * k + 3] * mul, lo, true);
    }
    b = scaling.finite ? make_uint2(w[0], w[1]) : make_uint2(0, 0);
    if (on) *(uint2*)((uint8_t*)out + dst) = b;
    if (lane == 0) {
      float* sc = is_v ? a.c.v_scale : a.c.k_scale;
      sc[page * a.c.n_kv_heads * a.c.page_size + head * a.sc_head + slot * a.sc_slot] = scaling.scale;
    }
  }
}

hipError_t launch_kv_append(const aqmb_kv_cache& c, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                            aqmb_dtype dtype, const int64_t* slots, int n_tokens, hipStream_t st) {
  AppendArgs a;
  a.c = c;
  const bool hm = c.layout == AQMB_KV_HEAD_MAJOR;
  a.sc_head = hm ? c.page_size : 1;
  a.sc_slot = hm ? 1 : c.n_kv_heads;
  a.head_stride = a.sc_head * c.head_dim;
  a.slot_stride = a.sc_slot * c.head_dim;
  a.k = (const uint16_t*)k;
  a.v = (const uint16_t*)v;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.slots = slots;
  a.pairs = (int64_t)n_tokens * c.n_kv_heads;
  const unsigned blocks = (unsigned)((a.pairs + 3) / 4);
  if (c.dtype != AQMB_F8) append_kernel<AQMB_F16, false><<<blocks, 256, 0, st>>>(a);   // bits only: either type
  else if (dtype == AQMB_F16) append_kernel<AQMB_F16, true><<<blocks, 256, 0, st>>>(a);
  else append_kernel<AQMB_BF16, true><<<blocks, 256, 0, st>>>(a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------- page copies
struct CopyArgs {
  void* data[2 * AQMB_MAX_CACHES];        // keys and values of every cache
  float* scale[2 * AQMB_MAX_CACHES];
  const int* src;
  const int* dst;
  int64_t page_stride;                    // bytes
  int64_t page_bytes, scale_bytes;
  int n_pages, n_pairs;
};
// 8 KiB per workgroup: 200 pages of 4 layers (365 MB) 69 us, 16 KiB 71, 32 KiB 109; streaming stores (76 without), cached
// loads (a page may be copied several times; 74 with streaming ones).
constexpr int kCopyThreads = 256, kCopyUnits = 2;

// blockIdx: x part of a page, y pair (folded above 32768), z buffer.
__global__ __launch_bounds__(kCopyThreads) void copy_kernel(CopyArgs a, int pair0) {
  const int pair = pair0 + blockIdx.y;
  const int s = a.src[pair], d = a.dst[pair];
  if (s < 0 || s >= a.n_pages || d < 0 || d >= a.n_pages || s == d) return;
  const char* from = (const char*)a.data[blockIdx.z] + (int64_t)s * a.page_stride;
  char* to = (char*)a.data[blockIdx.z] + (int64_t)d * a.page_stride;
  const int64_t at = ((int64_t)blockIdx.x * kCopyUnits * kCopyThreads + threadIdx.x) * 16;
  u32x4_t v[kCopyUnits];
#pragma unroll
  for (int i = 0; i < kCopyUnits; ++i) {
    const int64_t o = at + (int64_t)i * kCopyThreads * 16;
    if (o + 16 <= a.page_bytes) v[i] = *(const u32x4_t*)(from + o);
  }
#pragma unroll
  for (int i = 0; i < kCopyUnits; ++i) {
    const int64_t o = at + (int64_t)i * kCopyThreads * 16;
    if (o + 16 <= a.page_bytes) __builtin_nontemporal_store(v[i], (u32x4_t*)(to + o));
    // An 8-bit page may end 8 bytes into a unit.
    else if (o < a.page_bytes) *(uint2*)(to + o) = *(const uint2*)(from + o);
  }
  if (blockIdx.x == 0 && a.scale_bytes) {
    float* sc = a.scale[blockIdx.z];
    const int64_t n = a.scale_bytes / 4;
    for (int64_t i = threadIdx.x; i < n; i += kCopyThreads) sc[(int64_t)d * n + i] = sc[(int64_t)s * n + i];
  }
}

hipError_t launch_kv_copy(const aqmb_kv_cache* caches, int n_caches, const int32_t* src, const int32_t* dst, int n_pairs,
                          hipStream_t st) {
  CopyArgs a = {};
  const aqmb_kv_cache& c = caches[0];
  const bool f8 = c.dtype == AQMB_F8;
  for (int i = 0; i < n_caches; ++i) {
    a.data[2 * i] = caches[i].k;
    a.data[2 * i + 1] = caches[i].v;
    a.scale[2 * i] = caches[i].k_scale;
    a.scale[2 * i + 1] = caches[i].v_scale;
  }
  a.src = src;
  a.dst = dst;
  const int64_t tokens = (int64_t)c.n_kv_heads * c.page_size;
  a.page_stride = c.page_stride * (f8 ? 1 : 2);
  a.page_bytes = tokens * c.head_dim * (f8 ? 1 : 2);
  a.scale_bytes = f8 ? tokens * 4 : 0;
  a.n_pages = c.n_pages;
  a.n_pairs = n_pairs;
  const int64_t unit = (int64_t)kCopyThreads * kCopyUnits * 16;
  const unsigned parts = (unsigned)((a.page_bytes + unit - 1) / unit);
  for (int p = 0; p < n_pairs; p += 32768) {
    const int n = n_pairs - p < 32768 ? n_pairs - p : 32768;
    copy_kernel<<<dim3(parts, n, 2 * n_caches), kCopyThreads, 0, st>>>(a, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace aqmb
