// Rotary positions of a step's or a prompt's queries and keys, and the same on the way into a paged cache.
//
//   a' = amplitude (a cos - b sin),  b' = amplitude (b cos + a sin),  angle = position * frequency
//
// A workgroup turns heads of one token. Its threads first compute the token's cosines and sines, one for each value
// of a head, into LDS; then L lanes own a head, 8 neighbouring values each, with their partners: neighbours in the
// same registers (interleaved), or a second load of the same head (halves), which the first one's cache lines serve.
// Every value is read from HBM once and written once, and that bounds a prompt; a decode step is bound by latency.
#include "device.h"
#include "ops.h"
#include "wave.h"

namespace aqmb {

namespace {

struct __attribute__((packed, aligned(2))) Raw8 { uint32_t w[4]; };

enum Pairs { kNeighbours = 0, kHalves8 = 1, kHalves = 2 };    // kHalves8: rotary_dim / 2 is a multiple of 8

struct Args {
  RotaryArgs r;
  int64_t head_stride, slot_stride, sc_head, sc_slot;         // of the cache
  int pairs, half, heads_per_block, n_total;
};

template <int DT>
__device__ __forceinline__ void widen8(const Raw8& r, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = DT == AQMB_F16 ? f16lo(r.w[i]) : bf16lo(r.w[i]);
    f[2 * i + 1] = DT == AQMB_F16 ? f16hi(r.w[i]) : bf16hi(r.w[i]);
  }
}
template <int DT>
__device__ __forceinline__ Raw8 narrow8(const float* f) {
  Raw8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.w[i] = DT == AQMB_F16 ? pack_f16x2(f[2 * i], f[2 * i + 1]) : pack_bf16x2(f[2 * i], f[2 * i + 1]);
  return r;
}

// (cos, sin) of an angle in turns, within half a turn: reduced to an eighth of a turn around the nearest quarter, then
// the Taylor polynomials, whose first left out terms are below 2^-28 there.
__device__ __forceinline__ float2 cos_sin(double turns) {
  const double q = rint(4.0 * turns);
  const float x = (float)((turns - 0.25 * q) * 6.283185307179586), x2 = x * x;
  float s = fmaf(x2, 2.755731922398589e-6f, -1.984126984126984e-4f);
  s = fmaf(x2, s, 8.333333333333333e-3f);
  s = fmaf(x2, s, -1.666666666666667e-1f);
  s = fmaf(x * x2, s, x);
  float c = fmaf(x2, -2.755731922398589e-7f, 2.480158730158730e-5f);
  c = fmaf(x2, c, -1.388888888888889e-3f);
  c = fmaf(x2, c, 4.166666666666667e-2f);
  c = fmaf(x2, c, -0.5f);
  c = fmaf(x2, c, 1.f);
  const int n = (int)q;
  const float a = n & 1 ? s : c, b = n & 1 ? c : s;
  return make_float2((n + 1) & 2 ? -a : a, n & 2 ? -b : b);
}

// A head's values 8 lane .. 8 lane + 7 and their partners.
struct Piece { Raw8 x, p; };
__device__ __forceinline__ Piece load(const Args& a, const uint16_t* head, int e, bool turned) {
  Piece v;
  v.x = *(const Raw8*)(head + e);
  v.p = v.x;
  if (turned && e < a.r.rot.rotary_dim) {
    if (a.pairs == kHalves8) {
      v.p = *(const Raw8*)(head + (e < a.half ? e + a.half : e - a.half));
    } else if (a.pairs == kHalves) {
      uint32_t u[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = e + j;
        u[j] = head[i < a.half ? i + a.half : i < 2 * a.half ? i - a.half : i];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) v.p.w[j] = u[2 * j] | u[2 * j + 1] << 16;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) v.p.w[j] = __builtin_amdgcn_alignbit(v.x.w[j], v.x.w[j], 16);
    }
  }
  return v;
}

// kCache: 0 none, 1 of 16 bits, 2 of 8 bits. L lanes per head.
template <int DT, int kCache, int L>
__global__ __launch_bounds__(256) void rotary_kernel(Args a) {
  __shared__ __align__(16) float2 table[256];
  const int64_t token = blockIdx.x;
  const int e = threadIdx.x % L * 8, dim = a.r.head_dim, rot = a.r.rot.rotary_dim;
  const bool on = e < dim;
  const int end = min((int)(blockIdx.y + 1) * a.heads_per_block, a.n_total);
  int h = blockIdx.y * a.heads_per_block + threadIdx.x / L;
  int64_t at = -1;
  if constexpr (kCache) at = a.r.slots[token];

  const auto source = [&](int head) {
    const int k = head - a.r.n_heads, v = k - a.r.n_kv;
    return k < 0 ? (const uint16_t*)a.r.q + token * a.r.q_stride + (int64_t)head * dim
                 : v < 0 ? (const uint16_t*)a.r.k + token * a.r.k_stride + (int64_t)k * dim
                         : (const uint16_t*)a.r.v + token * a.r.v_stride + (int64_t)v * dim;
  };
  Piece next = {};
  if (h < end && on) next = load(a, source(h), e, h < a.r.n_heads + a.r.n_kv);
  if (threadIdx.x < (unsigned)dim) {
    const int i = threadIdx.x;
    float2 cs = make_float2(1.f, 0.f);
    if (i < rot) {
      const bool first = a.pairs == kNeighbours ? i % 2 == 0 : i < a.half;
      const int pair = a.pairs == kNeighbours ? i / 2 : first ? i : i - a.half;
      const double turns = (double)a.r.positions[token] * (a.r.rot.frequencies[pair] * 0.15915494309189535);
      cs = cos_sin(turns - rint(turns));
      if (first != (a.r.rot.inverse != 0)) cs.y = -cs.y;
      cs.x *= a.r.rot.amplitude;
      cs.y *= a.r.rot.amplitude;
    }
    table[i] = cs;
  }
  __syncthreads();
  float c[8], s[8];
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const float4 t = *(const float4*)(table + e + j);      // past the head's end: not used
    c[j] = t.x, s[j] = t.y, c[j + 1] = t.z, s[j + 1] = t.w;
  }

  for (; h < end; h += 256 / L) {
    const Piece now = next;
    const int more = h + 256 / L;
    if (more < end && on) next = load(a, source(more), e, more < a.r.n_heads + a.r.n_kv);
    const int k = h - a.r.n_heads, v = k - a.r.n_kv;
    float f[8];
    widen8<DT>(now.x, f);
    if (v < 0 && e < rot) {
      float p[8];
      widen8<DT>(now.p, p);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = e + j < rot ? fmaf(f[j], c[j], p[j] * s[j]) : f[j];
    }
    if (kCache == 0 || k < 0) {
      if (!on) continue;
      uint16_t* out = k < 0 ? (uint16_t*)a.r.q_out + token * a.r.q_out_stride + (int64_t)h * dim
                            : (uint16_t*)a.r.k_out + token * a.r.k_out_stride + (int64_t)k * dim;
      *(Raw8*)(out + e) = e < rot ? narrow8<DT>(f) : now.x;
      continue;
    }
    if constexpr (kCache != 0) {
      if (at < 0 || at >= (int64_t)a.r.cache.n_pages * a.r.cache.page_size) continue;
      const int64_t page = at / a.r.cache.page_size, slot = at % a.r.cache.page_size, head = v < 0 ? k : v;
      const int64_t dst = page * a.r.cache.page_stride + head * a.head_stride + slot * a.slot_stride + e;
      void* out = v < 0 ? a.r.cache.k : a.r.cache.v;
      if constexpr (kCache == 1) {
        const Raw8 y = v < 0 && e < rot ? narrow8<DT>(f) : now.x;
        if (on) *(u32x4_t*)((uint16_t*)out + dst) = u32x4_t{y.w[0], y.w[1], y.w[2], y.w[3]};
      } else {
        uint32_t big = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) big = max(big, on ? __builtin_bit_cast(uint32_t, f[j]) & 0x7FFFFFFFu : 0);
        big = over_lanes<L>(big, max_bits);
        const Scaling sc = scaling_of(big, 448.f);
        uint32_t w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j] * sc.mul, f[4 * j + 1] * sc.mul, 0, false);
          w[j] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j + 2] * sc.mul, f[4 * j + 3] * sc.mul, lo, true);
        }
        if (on) *(uint2*)((uint8_t*)out + dst) = sc.finite ? make_uint2(w[0], w[1]) : make_uint2(0, 0);
        if (e == 0) {
          float* scales = v < 0 ? a.r.cache.k_scale : a.r.cache.v_scale;
          scales[page * a.r.cache.n_kv_heads * a.r.cache.page_size + head * a.sc_head + slot * a.sc_slot] = sc.scale;
        }
      }
    }
  }
}

template <int DT, int kCache>
hipError_t go(const Args& a, dim3 grid, int lanes, hipStream_t st) {
  if (lanes == 8) rotary_kernel<DT, kCache, 8><<<grid, 256, 0, st>>>(a);
  else if (lanes == 16) rotary_kernel<DT, kCache, 16><<<grid, 256, 0, st>>>(a);
  else rotary_kernel<DT, kCache, 32><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

// Workgroups: one for every token and as many heads as 256 threads own at once, at least 8 values a lane.
hipError_t launch_rotary(const RotaryArgs& r, aqmb_dtype dtype, hipStream_t st) {
  Args a;
  a.r = r;
  const bool cached = r.slots != nullptr;
  if (cached) {
    const bool hm = r.cache.layout == AQMB_KV_HEAD_MAJOR;
    a.sc_head = hm ? r.cache.page_size : 1;
    a.sc_slot = hm ? 1 : r.cache.n_kv_heads;
    a.head_stride = a.sc_head * r.cache.head_dim;
    a.slot_stride = a.sc_slot * r.cache.head_dim;
  }
  a.half = r.rot.rotary_dim / 2;
  a.pairs = r.rot.layout == AQMB_ROTARY_INTERLEAVED ? kNeighbours : a.half % 8 == 0 ? kHalves8 : kHalves;
  a.n_total = r.n_heads + r.n_kv * (cached ? 2 : 1);
  const int lanes = r.head_dim <= 64 ? 8 : r.head_dim <= 128 ? 16 : 32, at_once = 256 / lanes;
  a.heads_per_block = at_once;
  const dim3 grid(r.n_tokens, (a.n_total + a.heads_per_block - 1) / a.heads_per_block);
  const bool f16 = dtype == AQMB_F16;
  if (!cached) return f16 ? go<AQMB_F16, 0>(a, grid, lanes, st) : go<AQMB_BF16, 0>(a, grid, lanes, st);
  if (r.cache.dtype != AQMB_F8) return f16 ? go<AQMB_F16, 1>(a, grid, lanes, st) : go<AQMB_BF16, 1>(a, grid, lanes, st);
  return f16 ? go<AQMB_F16, 2>(a, grid, lanes, st) : go<AQMB_BF16, 2>(a, grid, lanes, st);
}

}  // namespace aqmb
