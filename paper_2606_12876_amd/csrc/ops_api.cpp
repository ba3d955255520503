// The C-ABI entry points of the operators between the layers: validation, layer registry, dispatch.
// Arguments are checked before anything touches the GPU.
#include <hip/hip_runtime.h>

#include <cmath>
#include <mutex>
#include <new>
#include <unordered_set>

#include "ops.h"

namespace aqmb {
aqmb_status fail(aqmb_status s, const char* fmt, ...);
void clear_error();

static std::mutex g_w4_mu;
static std::unordered_set<W4*> g_w4;

static bool is_live(W4* L) {
  std::lock_guard<std::mutex> lk(g_w4_mu);
  return L && g_w4.count(L) && L->magic == kW4Magic;
}

static aqmb_status hip_status(hipError_t e, const char* what) {
  return e == hipSuccess ? AQMB_OK : fail(AQMB_EHIP, "%s: %s", what, hipGetErrorString(e));
}

static void free_w4(W4* L) {
  if (L->tiles) (void)hipFree(L->tiles);
  if (L->scales) (void)hipFree(L->scales);
  if (L->zeros) (void)hipFree(L->zeros);
  L->magic = 0;
  delete L;
}

static bool is16(int t) { return t == AQMB_F16 || t == AQMB_BF16; }
static bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }
static int elem(int t) { return t == AQMB_F32 ? 4 : t == AQMB_F8 || t == AQMB_I8 ? 1 : 2; }

static aqmb_status check_cache(const aqmb_kv_cache* c, const char* where) {
  if (!c) return fail(AQMB_EINVAL, "%s: cache is NULL", where);
  if (c->dtype != AQMB_F8 && !is16(c->dtype))
    return fail(AQMB_EUNSUPPORTED, "%s: cache dtype %d is not F16, BF16 or F8", where, c->dtype);
  if (c->layout != AQMB_KV_HEAD_MAJOR && c->layout != AQMB_KV_SLOT_MAJOR)
    return fail(AQMB_EINVAL, "%s: unknown layout %d", where, c->layout);
  if (c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1 || c->head_dim < 1)
    return fail(AQMB_EINVAL, "%s: n_pages, page_size, n_kv_heads and head_dim must be >= 1", where);
  if (c->page_size > 32768) return fail(AQMB_EUNSUPPORTED, "%s: page_size = %d above 32768", where, c->page_size);
  if (c->n_kv_heads > 32768) return fail(AQMB_EUNSUPPORTED, "%s: n_kv_heads = %d above 32768", where, c->n_kv_heads);
  if (c->head_dim % 8 || c->head_dim > 256)
    return fail(AQMB_EUNSUPPORTED, "%s: head_dim = %d is not a multiple of 8 up to 256", where, c->head_dim);
  if (c->page_stride < (int64_t)c->n_kv_heads * c->page_size * c->head_dim || c->page_stride % 8)
    return fail(AQMB_EINVAL, "%s: page_stride = %lld is shorter than a page or no multiple of 8", where,
                (long long)c->page_stride);
  if (c->page_stride > (int64_t)1 << 40) return fail(AQMB_EINVAL, "%s: page_stride above 2^40", where);
  if (!c->k || !c->v) return fail(AQMB_EINVAL, "%s: k or v of the cache is NULL", where);
  const size_t al = c->dtype == AQMB_F8 ? 8 : 16;
  if (!aligned(c->k, al) || !aligned(c->v, al))
    return fail(AQMB_EINVAL, "%s: k and v of the cache must be %zu-byte aligned", where, al);
  if (c->dtype == AQMB_F8) {
    if (!c->k_scale || !c->v_scale) return fail(AQMB_EINVAL, "%s: an F8 cache needs k_scale and v_scale", where);
    if (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return fail(AQMB_EINVAL, "%s: misaligned scales", where);
  } else if (c->k_scale || c->v_scale) {
    return fail(AQMB_EINVAL, "%s: scales belong to an F8 cache only", where);
  }
  return AQMB_OK;
}

// The type of q, k and v beside a cache: the cache's own, or either 16-bit one for an 8-bit cache.
static aqmb_status check_beside(const aqmb_kv_cache* c, int dtype, const char* where) {
  if (!is16(dtype)) return fail(AQMB_EUNSUPPORTED, "%s: dtype %d is not F16 or BF16", where, dtype);
  if (c->dtype != AQMB_F8 && dtype != c->dtype)
    return fail(AQMB_EUNSUPPORTED, "%s: dtype %d differs from the cache's %d", where, dtype, c->dtype);
  return AQMB_OK;
}

static aqmb_status check_attention(const aqmb_kv_cache* c, int n_heads, int n_seqs, int max_length, int window,
                                   const char* where) {
  const aqmb_status s = check_cache(c, where);
  if (s != AQMB_OK) return s;
  if (n_heads < 1 || n_heads % c->n_kv_heads)
    return fail(AQMB_EINVAL, "%s: n_heads = %d is not a multiple of n_kv_heads = %d", where, n_heads, c->n_kv_heads);
  if (n_heads > 65535 || n_seqs > 65535) return fail(AQMB_EUNSUPPORTED, "%s: more than 65535 heads or sequences", where);
  if (n_seqs < 1) return fail(AQMB_EINVAL, "%s: n_seqs = %d must be >= 1", where, n_seqs);
  if (max_length < 0 || max_length > 1 << 27) return fail(AQMB_EINVAL, "%s: max_length = %d outside [0, 2^27]", where, max_length);
  if (window < 0) return fail(AQMB_EINVAL, "%s: window = %d is negative", where, window);
  return AQMB_OK;
}

// Compute units of the current device, asked of the runtime once per device.
static hipError_t compute_units(int* n) {
  static std::mutex mu;
  static int known[64];
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  std::lock_guard<std::mutex> lk(mu);
  if (dev < 64 && known[dev]) {
    *n = known[dev];
    return hipSuccess;
  }
  e = hipDeviceGetAttribute(n, hipDeviceAttributeMultiprocessorCount, dev);
  if (e == hipSuccess && dev < 64) known[dev] = *n;
  return e;
}

}  // namespace aqmb

using namespace aqmb;

extern "C" {

aqmb_status aqmb_rms_norm(const void* x, aqmb_dtype dtype, int64_t x_stride, const void* residual, void* residual_out,
                          int64_t residual_stride, const void* weight, float weight_offset, float eps, int rows,
                          int cols, void* y, aqmb_dtype y_dtype, int64_t y_stride, float* scales, int scale_group,
                          aqmb_stream_t stream) {
  clear_error();
  const bool q8 = y_dtype == AQMB_F8 || y_dtype == AQMB_I8;
  if (!is16(dtype)) return fail(AQMB_EUNSUPPORTED, "rms_norm: dtype %d is not F16 or BF16", (int)dtype);
  if (!q8 && !is16(y_dtype) && y_dtype != AQMB_F32) return fail(AQMB_EUNSUPPORTED, "rms_norm: unknown y dtype %d", (int)y_dtype);
  if (!x || !weight || !y) return fail(AQMB_EINVAL, "rms_norm: x, weight or y is NULL");
  if (!residual != !residual_out) return fail(AQMB_EINVAL, "rms_norm: residual and residual_out go together");
  if (rows < 1 || cols < 1) return fail(AQMB_EINVAL, "rms_norm: rows = %d and cols = %d must be >= 1", rows, cols);
  if (cols > AQMB_MAX_NORM_COLS) return fail(AQMB_EUNSUPPORTED, "rms_norm: cols = %d above %d", cols, AQMB_MAX_NORM_COLS);
  // A launch has fewer than 2^32 threads; a row takes at most two for every 8 columns, and 16 if it is short (then
  // 16 rows share a workgroup).
  const int64_t threads = cols <= 64 ? ((int64_t)rows + 15) / 16 * 256 : (int64_t)rows * ((cols + 7) / 8 * 2);
  if (threads >= (int64_t)1 << 32)
    return fail(AQMB_EUNSUPPORTED, "rms_norm: rows = %d of %d columns are more than one launch takes", rows, cols);
  if (x_stride < cols || y_stride < cols || (residual && residual_stride < cols))
    return fail(AQMB_EINVAL, "rms_norm: a row stride is below cols = %d", cols);
  if (!(eps >= 0.f) || std::isinf(eps)) return fail(AQMB_EINVAL, "rms_norm: eps must be finite and >= 0");
  if (q8 != (scales != nullptr)) return fail(AQMB_EINVAL, "rms_norm: scales belong to an 8-bit y, and only there");
  if (q8 && scale_group != 0 && scale_group != 32 && scale_group != 64 && scale_group != 128)
    return fail(AQMB_EUNSUPPORTED, "rms_norm: scale_group = %d is not 0, 32, 64 or 128", scale_group);
  if (!aligned(x, 2) || !aligned(residual, 2) || !aligned(residual_out, 2) || !aligned(weight, 2) ||
      !aligned(y, elem(y_dtype)) || !aligned(scales, 4))
    return fail(AQMB_EINVAL, "rms_norm: a pointer is not aligned to its elements");
  const NormArgs a = {x, residual, residual_out, weight, y, scales, x_stride, residual_stride, y_stride,
                      weight_offset, eps, rows, cols, (int)y_dtype, scale_group};
  return hip_status(launch_rms_norm(a, dtype, (hipStream_t)stream), "rms_norm: launch");
}

aqmb_status aqmb_w4_create(aqmb_w4_t* out, const aqmb_w4_desc* desc, const uint8_t* weights, const uint16_t* scales,
                           const uint8_t* zeros, aqmb_stream_t stream) {
  clear_error();
  if (!out) return fail(AQMB_EINVAL, "w4_create: out is NULL");
  *out = nullptr;
  if (!desc) return fail(AQMB_EINVAL, "w4_create: descriptor is NULL");
  if (desc->d_out < 1 || desc->d_in < 1)
    return fail(AQMB_EINVAL, "w4_create: d_out = %d and d_in = %d must be >= 1", desc->d_out, desc->d_in);
  if (desc->d_out > 1 << 30 || desc->d_in > 1 << 30 || (uint64_t)desc->d_out * (uint64_t)desc->d_in >= (1ull << 32))
    return fail(AQMB_EINVAL, "w4_create: d_out and d_in must be at most 2^30, their product below 2^32");
  if (desc->group_size != 32 && desc->group_size != 64 && desc->group_size != 128)
    return fail(AQMB_EUNSUPPORTED, "w4_create: group_size = %d is not 32, 64 or 128", desc->group_size);
  // Laid out by one launch, a thread for every dword of the tiles (256 of each): fewer than 2^32.
  const int n_rt = (desc->d_out - 1) / kW4Rows + 1, n_kt = (desc->d_in - 1) / kW4Cols + 1;
  if ((int64_t)n_rt * n_kt >= 1 << 24)
    return fail(AQMB_EINVAL, "w4_create: %d x %d weights are 2^24 tiles of %d x %d or more", desc->d_out, desc->d_in,
                kW4Rows, kW4Cols);
  if (!weights || !scales) return fail(AQMB_EINVAL, "w4_create: weights or scales is NULL");
  if (!aligned(scales, 2)) return fail(AQMB_EINVAL, "w4_create: scales must be 2-byte aligned");

  W4* L = new (std::nothrow) W4();
  if (!L) return fail(AQMB_ENOMEM, "w4_create: host allocation failed");
  L->magic = kW4Magic;
  L->d = *desc;
  hipError_t e = hipGetDevice(&L->device);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&L->n_cu, hipDeviceAttributeMultiprocessorCount, L->device);
  if (e != hipSuccess) { free_w4(L); return hip_status(e, "w4_create: device"); }
  L->n_rt = n_rt;
  L->n_kt = n_kt;
  const size_t tiles = (size_t)L->n_rt * L->n_kt, n_scales = tiles * (kW4Cols / desc->group_size) * kW4Rows;
  L->asymmetric = zeros != nullptr;
  struct { void** p; size_t n; } allocs[] = {{(void**)&L->tiles, tiles * 1024}, {(void**)&L->scales, n_scales * 2},
                                             {(void**)&L->zeros, zeros ? n_scales : n_scales / tiles}};
  for (auto& a : allocs) {
    e = hipMalloc(a.p, a.n);
    if (e != hipSuccess) {
      *a.p = nullptr;
      (void)hipGetLastError();
      free_w4(L);
      return fail(AQMB_ENOMEM, "w4_create: hipMalloc(%zu) failed: %s", a.n, hipGetErrorString(e));
    }
  }
  const hipStream_t st = (hipStream_t)stream;
  if ((e = launch_w4_pack(*L, weights, scales, zeros, st)) != hipSuccess || (e = hipStreamSynchronize(st)) != hipSuccess) {
    free_w4(L);
    return hip_status(e, "w4_create: layout");
  }
  try {
    std::lock_guard<std::mutex> lk(g_w4_mu);
    g_w4.insert(L);
  } catch (...) {
    free_w4(L);
    return fail(AQMB_ENOMEM, "w4_create: host allocation failed");
  }
  *out = (aqmb_w4_t)L;
  return AQMB_OK;
}

aqmb_status aqmb_w4_destroy(aqmb_w4_t layer) {
  clear_error();
  if (!layer) return AQMB_OK;
  W4* L = (W4*)layer;
  {
    std::lock_guard<std::mutex> lk(g_w4_mu);
    if (!g_w4.erase(L)) return fail(AQMB_EINVAL, "w4_destroy: not a live layer");
  }
  int cur = -1;
  (void)hipGetDevice(&cur);
  if (cur != L->device) (void)hipSetDevice(L->device);
  const bool moved = cur >= 0 && cur != L->device;
  const hipError_t e = hipDeviceSynchronize();
  free_w4(L);
  if (moved) (void)hipSetDevice(cur);
  return hip_status(e, "w4_destroy");
}

aqmb_status aqmb_w4_get_desc(aqmb_w4_t layer, aqmb_w4_desc* out) {
  clear_error();
  if (!is_live((W4*)layer)) return fail(AQMB_EINVAL, "w4_get_desc: not a live layer");
  if (!out) return fail(AQMB_EINVAL, "w4_get_desc: out is NULL");
  *out = ((W4*)layer)->d;
  return AQMB_OK;
}

aqmb_status aqmb_w4_gemv(aqmb_w4_t layer, const void* x, aqmb_dtype x_dtype, int64_t x_stride, const float* x_scales,
                         int x_scale_group, int batch, void* y, aqmb_dtype y_dtype, int64_t y_stride,
                         aqmb_stream_t stream) {
  clear_error();
  W4* L = (W4*)layer;
  if (!is_live(L)) return fail(AQMB_EINVAL, "w4_gemv: not a live layer");
  const bool q8 = x_dtype == AQMB_F8 || x_dtype == AQMB_I8;
  if (!q8 && !is16(x_dtype)) return fail(AQMB_EUNSUPPORTED, "w4_gemv: x dtype %d is not F16, BF16, F8 or I8", (int)x_dtype);
  if (!is16(y_dtype) && y_dtype != AQMB_F32) return fail(AQMB_EUNSUPPORTED, "w4_gemv: y dtype %d is not F16, BF16 or F32", (int)y_dtype);
  if (!x || !y) return fail(AQMB_EINVAL, "w4_gemv: x or y is NULL");
  if (batch < 1) return fail(AQMB_EINVAL, "w4_gemv: batch = %d must be >= 1", batch);
  if (batch > AQMB_MAX_BATCH) return fail(AQMB_EUNSUPPORTED, "w4_gemv: batch = %d above %d", batch, AQMB_MAX_BATCH);
  if (x_stride < L->d.d_in || y_stride < L->d.d_out) return fail(AQMB_EINVAL, "w4_gemv: a row stride is below the row");
  if (q8 != (x_scales != nullptr)) return fail(AQMB_EINVAL, "w4_gemv: x_scales belong to an 8-bit x, and only there");
  if (q8 && x_scale_group != 0 && x_scale_group != L->d.group_size)
    return fail(AQMB_EUNSUPPORTED, "w4_gemv: x_scale_group = %d is not 0 or the layer's %d", x_scale_group, L->d.group_size);
  if (!aligned(x, elem(x_dtype)) || !aligned(y, elem(y_dtype)) || !aligned(x_scales, 4))
    return fail(AQMB_EINVAL, "w4_gemv: a pointer is not aligned to its elements");
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_status(e, "w4_gemv: hipGetDevice");
  if (dev != L->device) return fail(AQMB_EINVAL, "layer lives on device %d but device %d is current", L->device, dev);
  e = launch_w4_gemv(*L, x, x_dtype, x_stride, x_scales, q8 ? x_scale_group : 0, batch, y, y_dtype, y_stride, (hipStream_t)stream);
  return hip_status(e, "w4_gemv: launch");
}

aqmb_status aqmb_paged_attention_workspace_bytes(const aqmb_kv_cache* cache, int n_heads, int n_seqs, int max_length,
                                                 int window, size_t* bytes) {
  clear_error();
  if (!bytes) return fail(AQMB_EINVAL, "paged_attention_workspace_bytes: bytes is NULL");
  const aqmb_status s = check_attention(cache, n_heads, n_seqs, max_length, window, "paged_attention_workspace_bytes");
  if (s != AQMB_OK) return s;
  int n_cu = 0;
  const hipError_t e = compute_units(&n_cu);
  if (e != hipSuccess) return hip_status(e, "paged_attention_workspace_bytes");
  *bytes = attn_plan(n_heads, cache->n_kv_heads, cache->head_dim, n_seqs, max_length, window, n_cu).bytes;
  return AQMB_OK;
}

aqmb_status aqmb_paged_attention(const aqmb_kv_cache* cache, const void* q, aqmb_dtype dtype, int64_t q_stride,
                                 int n_heads, const int32_t* page_table, int64_t table_stride, const int32_t* lengths,
                                 int n_seqs, int max_length, float scale, int window, void* out, int64_t out_stride,
                                 float* lse, void* workspace, size_t workspace_bytes, aqmb_stream_t stream) {
  clear_error();
  const char* where = "paged_attention";
  aqmb_status s = check_attention(cache, n_heads, n_seqs, max_length, window, where);
  if (s != AQMB_OK || (s = check_beside(cache, dtype, where)) != AQMB_OK) return s;
  const aqmb_kv_cache& c = *cache;
  if (!q || !page_table || !lengths || !out) return fail(AQMB_EINVAL, "%s: q, page_table, lengths or out is NULL", where);
  const int64_t row = (int64_t)n_heads * c.head_dim;
  if (q_stride < row || out_stride < row || q_stride % 8 || out_stride % 8)
    return fail(AQMB_EINVAL, "%s: q_stride and out_stride must be multiples of 8 of at least n_heads * head_dim", where);
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(page_table, 4) || !aligned(lengths, 4) || !aligned(lse, 4))
    return fail(AQMB_EINVAL, "%s: a misaligned pointer", where);
  if (table_stride < 1 || max_length > table_stride * (int64_t)c.page_size)
    return fail(AQMB_EINVAL, "%s: max_length = %d needs more pages than table_stride = %lld", where, max_length,
                (long long)table_stride);
  if (!std::isfinite(scale)) return fail(AQMB_EINVAL, "%s: scale is not finite", where);
  int n_cu = 0;
  hipError_t e = compute_units(&n_cu);
  if (e != hipSuccess) return hip_status(e, where);
  const AttnPlan plan = attn_plan(n_heads, c.n_kv_heads, c.head_dim, n_seqs, max_length, window, n_cu);
  if (plan.bytes && (!workspace || workspace_bytes < plan.bytes))
    return fail(AQMB_EINVAL, "%s: workspace of %zu bytes, %zu needed", where, workspace ? workspace_bytes : (size_t)0, plan.bytes);
  if (plan.bytes && !aligned(workspace, 16)) return fail(AQMB_EINVAL, "%s: workspace must be 16-byte aligned", where);
  const bool hm = c.layout == AQMB_KV_HEAD_MAJOR;
  AttnArgs a;
  a.k = c.k;
  a.v = c.v;
  a.k_scale = c.k_scale;
  a.v_scale = c.v_scale;
  a.page_stride = c.page_stride;
  a.sc_page = (int64_t)c.n_kv_heads * c.page_size;
  a.sc_head = hm ? c.page_size : 1;
  a.sc_slot = hm ? 1 : c.n_kv_heads;
  a.head_stride = a.sc_head * c.head_dim;
  a.slot_stride = a.sc_slot * c.head_dim;
  a.n_pages = c.n_pages;
  a.page_size = c.page_size;
  a.q = q;
  a.q_stride = q_stride;
  a.table = page_table;
  a.table_stride = table_stride;
  a.lengths = lengths;
  a.n_seqs = n_seqs;
  a.max_length = max_length;
  a.window = window;
  a.scale = scale;
  a.out = out;
  a.out_stride = out_stride;
  a.lse = lse;
  a.n_heads = n_heads;
  a.n_kv = c.n_kv_heads;
  a.head_dim = c.head_dim;
  a.chunk = plan.chunk;
  a.n_splits = plan.n_splits;
  a.waves = plan.waves;
  a.part = (float*)workspace;
  return hip_status(launch_attention(a, dtype, c.dtype == AQMB_F8, (hipStream_t)stream), "paged_attention: launch");
}

aqmb_status aqmb_kv_append(const aqmb_kv_cache* cache, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                           aqmb_dtype dtype, const int64_t* slots, int n_tokens, aqmb_stream_t stream) {
  clear_error();
  aqmb_status s = check_cache(cache, "kv_append");
  if (s != AQMB_OK || (s = check_beside(cache, dtype, "kv_append")) != AQMB_OK) return s;
  if (!k || !v || !slots) return fail(AQMB_EINVAL, "kv_append: k, v or slots is NULL");
  if (n_tokens < 1) return fail(AQMB_EINVAL, "kv_append: n_tokens = %d must be >= 1", n_tokens);
  const int64_t row = (int64_t)cache->n_kv_heads * cache->head_dim;
  if (k_stride < row || v_stride < row) return fail(AQMB_EINVAL, "kv_append: a stride is below a token");
  if (!aligned(k, 2) || !aligned(v, 2) || !aligned(slots, 8)) return fail(AQMB_EINVAL, "kv_append: a misaligned pointer");
  // 64 threads each, in workgroups of four, fewer than 2^32 a launch
  if (((int64_t)n_tokens * cache->n_kv_heads + 3) / 4 >= (int64_t)1 << 24)
    return fail(AQMB_EUNSUPPORTED, "kv_append: n_tokens * n_kv_heads above 2^26 - 4");
  return hip_status(launch_kv_append(*cache, k, k_stride, v, v_stride, dtype, slots, n_tokens, (hipStream_t)stream),
                    "kv_append: launch");
}

aqmb_status aqmb_kv_copy_pages(const aqmb_kv_cache* caches, int n_caches, const int32_t* src, const int32_t* dst,
                               int n_pairs, aqmb_stream_t stream) {
  clear_error();
  if (!caches || !src || !dst) return fail(AQMB_EINVAL, "kv_copy_pages: caches, src or dst is NULL");
  if (n_caches < 1 || n_pairs < 1)
    return fail(AQMB_EINVAL, "kv_copy_pages: n_caches = %d and n_pairs = %d must be >= 1", n_caches, n_pairs);
  if (n_caches > AQMB_MAX_CACHES) return fail(AQMB_EUNSUPPORTED, "kv_copy_pages: n_caches = %d above %d", n_caches, AQMB_MAX_CACHES);
  for (int i = 0; i < n_caches; ++i) {
    const aqmb_status s = check_cache(caches + i, "kv_copy_pages");
    if (s != AQMB_OK) return s;
    const aqmb_kv_cache &c = caches[i], &d = caches[0];
    if (c.dtype != d.dtype || c.layout != d.layout || c.n_pages != d.n_pages || c.page_size != d.page_size ||
        c.n_kv_heads != d.n_kv_heads || c.head_dim != d.head_dim || c.page_stride != d.page_stride)
      return fail(AQMB_EINVAL, "kv_copy_pages: cache %d differs from cache 0", i);
  }
  if (!aligned(src, 4) || !aligned(dst, 4)) return fail(AQMB_EINVAL, "kv_copy_pages: a misaligned pointer");
  return hip_status(launch_kv_copy(caches, n_caches, src, dst, n_pairs, (hipStream_t)stream), "kv_copy_pages: launch");
}

}  // extern "C"
