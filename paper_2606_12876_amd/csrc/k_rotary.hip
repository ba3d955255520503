// Rotary positions of a step's or a prompt's queries and keys, and the same on the way into a paged cache.
//
//   a' = amplitude (a cos - b sin),  b' = amplitude (b cos + a sin),  angle = position * frequency
//
// A workgroup turns the heads of a few tokens. Its threads first load, then compute the tokens' cosines and sines into LDS, one pair's
// each; L lanes own a head, 16 of its values each, two 16-byte loads and two stores (halves: 8 neighbours of either
// half, so 8 pairs). Every value is read once and written once, and that bounds a prompt; a decode step is bound by latency.
#include "device.h"
#include "ops.h"
#include "wave.h"

namespace aqmb {

namespace {

struct __attribute__((packed, aligned(2))) Raw8 { uint32_t w[4]; };

// kHalves8: rotary_dim / 2 is a multiple of 8.
enum Pairs { kNeighbours = 0, kHalves8 = 1, kHalves = 2 };

constexpr int kMany = 4;           // heads that a lane loads before it turns them, of many tokens; 1 of few
constexpr int kTokens = 16;        // of a workgroup, at most

struct Args {
  RotaryArgs r;
  int64_t head_stride, slot_stride, sc_head, sc_slot;         // of the cache
  int half, n_total, tokens, heads;                           // tokens and heads per workgroup
  bool stream;                                                // streaming stores
  uint32_t by_heads;                                          // 2^32 / heads, rounded up (heads > 1)
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

// An angle in turns, less whole ones. 1 / (2 pi) in two parts, and what the first one's product rounds off: an angle of one
// part only would be off by 2^-53 of itself, more than sine and cosine are from 2^30 on.
__device__ __forceinline__ double turns_of(double angle) {
#pragma clang fp contract(off)               // t is the rounded product everywhere
  constexpr double kHi = 0x1.45f306dc9c883p-3, kLo = -0x1.6b01ec5417056p-57;
  const double t = angle * kHi, rest = fma(angle, kLo, fma(angle, kHi, -t));
  const double f = (t - rint(t)) + rest;       // rest is above a half where t's steps are whole turns
  return f - rint(f);
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

// kCache: 0 none, 1 of 16 bits, 2 of 8 bits. L lanes per head.
template <int DT, int kCache, int L, int kPairs, int kBatch>
__global__ __launch_bounds__(256) void rotary_kernel(Args a) {
  extern __shared__ __align__(16) float2 table[];      // [tokens][half] (cos, sin)
  const int lane = threadIdx.x % L, dim = a.r.head_dim, rot = a.r.rot.rotary_dim, half = a.half;
  // A lane's two pieces of 8 values, each beside its neighbours' so that a store writes a run. Halves: the same 8 pairs'
  // first and second values, or two pieces behind the pairs.
  const int rest = kPairs == kHalves8 ? (dim - rot + 15) / 16 : (dim + 15) / 16;
  const bool paired = kPairs == kHalves8 && 8 * lane < half;
  const int e0 = kPairs == kHalves8 && !paired ? rot + 8 * (lane - half / 8) : 8 * lane;
  const int e1 = paired ? e0 + half : e0 + 8 * rest;
  const bool on0 = paired || lane - (kPairs == kHalves8 ? half / 8 : 0) < rest, on1 = on0 && e1 < dim;
  const bool turns = kPairs == kHalves8 ? paired : on0 && e0 < rot;
  const int64_t token0 = (int64_t)blockIdx.x * a.tokens;
  const int head0 = blockIdx.y * a.heads, n_heads = min(a.heads, a.n_total - head0);
  const int n_tokens = (int)min((int64_t)a.tokens, a.r.n_tokens - token0), units = n_tokens * a.heads;

  struct Unit { int token, head; bool on; };
  const auto unit = [&](int u) {
    const int t = a.heads == 1 ? u : (int)__umulhi((uint32_t)u, a.by_heads), h = u - t * a.heads;
    return Unit{t, head0 + h, u < units && h < n_heads};
  };
  const auto source = [&](const Unit& u) {
    const int64_t token = token0 + u.token;
    const int k = u.head - a.r.n_heads, v = k - a.r.n_kv;
    return k < 0 ? (const uint16_t*)a.r.q + token * a.r.q_stride + (int64_t)u.head * dim
                 : v < 0 ? (const uint16_t*)a.r.k + token * a.r.k_stride + (int64_t)k * dim
                         : (const uint16_t*)a.r.v + token * a.r.v_stride + (int64_t)v * dim;
  };

  for (int first = threadIdx.x / L; first - (int)(threadIdx.x / L) < units; first += kBatch * (256 / L)) {
    Raw8 x0[kBatch], x1[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const Unit u = unit(first + b * (256 / L));
      x0[b] = x1[b] = Raw8{{0, 0, 0, 0}};
      if (u.on) {
        const uint16_t* src = source(u);
        if (on0) x0[b] = *(const Raw8*)(src + e0);
        if (on1) x1[b] = *(const Raw8*)(src + e1);
      }
    }
    if (first == (int)(threadIdx.x / L)) {               // the first time: the whole workgroup
      for (int i = threadIdx.x; i < n_tokens * half; i += 256) {
        const int t = i / half, pair = i - t * half;
        float2 cs = cos_sin(turns_of((double)a.r.positions[token0 + t] * a.r.rot.frequencies[pair]));
        if (a.r.rot.inverse) cs.y = -cs.y;
        table[i] = make_float2(cs.x * a.r.rot.amplitude, cs.y * a.r.rot.amplitude);
      }
      __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const Unit u = unit(first + b * (256 / L));
      if (!u.on) continue;                               // all lanes of the head
      const int k = u.head - a.r.n_heads, v = k - a.r.n_kv;
      const bool turned = v < 0 && turns;
      float f0[8], f1[8];
      if (turned || kCache == 2) {
        widen8<DT>(x0[b], f0);
        widen8<DT>(x1[b], f1);
      }
      if (turned) {
        const float2* cs = table + u.token * half;
        if constexpr (kPairs == kHalves) {
          // The partners, one by one, out of the head's cache lines.
          const uint16_t* src = source(u);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int e = j < 8 ? e0 + j : e1 + j - 8;
            if (e >= rot) continue;
            const bool low = e < half;
            const uint32_t w = src[low ? e + half : e - half];
            const float p = DT == AQMB_F16 ? f16lo(w) : bf16lo(w);
            const float2 t = cs[low ? e : e - half];
            float& f = j < 8 ? f0[j % 8] : f1[j % 8];
            f = fmaf(f, t.x, low ? -p * t.y : p * t.y);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int pair = kPairs == kHalves8 ? e0 + j : (j < 4 ? e0 : e1) / 2 + j % 4;
            const float2 t = cs[min(pair, half - 1)];
            float& x = kPairs == kHalves8 ? f0[j] : j < 4 ? f0[2 * (j % 4)] : f1[2 * (j % 4)];
            float& y = kPairs == kHalves8 ? f1[j] : j < 4 ? f0[2 * (j % 4) + 1] : f1[2 * (j % 4) + 1];
            const float tx = fmaf(x, t.x, -y * t.y), ty = fmaf(y, t.x, x * t.y);
            // Behind the pairs: 16 bits take the words that were loaded, below.
            const bool in = kPairs == kHalves8 || kCache != 2 || pair < half;
            x = in ? tx : x;
            y = in ? ty : y;
          }
        }
      }
      Raw8 y0 = turned ? narrow8<DT>(f0) : x0[b], y1 = turned ? narrow8<DT>(f1) : x1[b];
      if constexpr (kPairs != kHalves8) {                // values behind the pairs, in words of two: their own bits, also a NaN's
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y0.w[j] = e0 + 2 * j < rot ? y0.w[j] : x0[b].w[j];
          y1.w[j] = e1 + 2 * j < rot ? y1.w[j] : x1[b].w[j];
        }
      }
      const int64_t token = token0 + u.token;
      if (kCache == 0 || k < 0) {
        uint16_t* out = k < 0 ? (uint16_t*)a.r.q_out + token * a.r.q_out_stride + (int64_t)u.head * dim
                              : (uint16_t*)a.r.k_out + token * a.r.k_out_stride + (int64_t)k * dim;
        if (kBatch > 1 && a.stream) {
          typedef u32x4_t __attribute__((aligned(2))) U;
          if (on0) __builtin_nontemporal_store(u32x4_t{y0.w[0], y0.w[1], y0.w[2], y0.w[3]}, (U*)(out + e0));
          if (on1) __builtin_nontemporal_store(u32x4_t{y1.w[0], y1.w[1], y1.w[2], y1.w[3]}, (U*)(out + e1));
        } else {
          if (on0) *(Raw8*)(out + e0) = y0;
          if (on1) *(Raw8*)(out + e1) = y1;
        }
        continue;
      }
      if constexpr (kCache != 0) {
        const int64_t at = a.r.slots[token];
        if (at < 0 || at >= (int64_t)a.r.cache.n_pages * a.r.cache.page_size) continue;
        const int64_t page = at / a.r.cache.page_size, slot = at % a.r.cache.page_size, head = v < 0 ? k : v;
        const int64_t dst = page * a.r.cache.page_stride + head * a.head_stride + slot * a.slot_stride;
        void* out = v < 0 ? a.r.cache.k : a.r.cache.v;
        if constexpr (kCache == 1) {
          if (on0) *(u32x4_t*)((uint16_t*)out + dst + e0) = u32x4_t{y0.w[0], y0.w[1], y0.w[2], y0.w[3]};
          if (on1) *(u32x4_t*)((uint16_t*)out + dst + e1) = u32x4_t{y1.w[0], y1.w[1], y1.w[2], y1.w[3]};
        } else {
          uint32_t big = 0;                              // what is off holds zeros
#pragma unroll
          for (int j = 0; j < 8; ++j)
            big = max(big, max(__builtin_bit_cast(uint32_t, f0[j]) & 0x7FFFFFFFu, __builtin_bit_cast(uint32_t, f1[j]) & 0x7FFFFFFFu));
          big = over_lanes<L>(big, max_bits);
          const Scaling sc = scaling_of(big, 448.f);
          const auto write = [&](const float* f, int e) {
            uint32_t w[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j] * sc.mul, f[4 * j + 1] * sc.mul, 0, false);
              w[j] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j + 2] * sc.mul, f[4 * j + 3] * sc.mul, lo, true);
            }
            *(uint2*)((uint8_t*)out + dst + e) = sc.finite ? make_uint2(w[0], w[1]) : make_uint2(0, 0);
          };
          if (on0) write(f0, e0);
          if (on1) write(f1, e1);
          if (lane == 0) {
            float* scales = v < 0 ? a.r.cache.k_scale : a.r.cache.v_scale;
            scales[page * a.r.cache.n_kv_heads * a.r.cache.page_size + head * a.sc_head + slot * a.sc_slot] = sc.scale;
          }
        }
      }
    }
  }
}

template <int DT, int kCache, int L, int kBatch>
hipError_t go(const Args& a, dim3 grid, hipStream_t st) {
  const size_t lds = (size_t)a.tokens * a.half * sizeof(float2);
  if (a.r.rot.layout == AQMB_ROTARY_INTERLEAVED) rotary_kernel<DT, kCache, L, kNeighbours, kBatch><<<grid, 256, lds, st>>>(a);
  else if (a.half % 8 == 0) rotary_kernel<DT, kCache, L, kHalves8, kBatch><<<grid, 256, lds, st>>>(a);
  else rotary_kernel<DT, kCache, L, kHalves, kBatch><<<grid, 256, lds, st>>>(a);
  return hipGetLastError();
}
template <int DT, int kCache, int L>
hipError_t go(const Args& a, dim3 grid, bool few, hipStream_t st) {
  return few ? go<DT, kCache, L, 1>(a, grid, st) : go<DT, kCache, L, kMany>(a, grid, st);
}
template <int DT, int kCache>
hipError_t go(const Args& a, dim3 grid, int lanes, bool few, hipStream_t st) {
  return lanes == 4 ? go<DT, kCache, 4>(a, grid, few, st) : lanes == 8 ? go<DT, kCache, 8>(a, grid, few, st)
                                                                        : go<DT, kCache, 16>(a, grid, few, st);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& r, aqmb_dtype dtype, hipStream_t st) {
  Args a = {};
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
  a.n_total = r.n_heads + r.n_kv * (cached ? 2 : 1);
  const int lanes = r.head_dim <= 64 ? 4 : r.head_dim <= 128 ? 8 : 16, at_once = 256 / lanes;
  // Few tokens: a head per lane group and workgroups over the heads, short code. Many: all heads of some tokens in a
  // workgroup, about kMany per lane group. 40 heads of 128: 1 token 2.3 us against 2.9, 512 tokens 3.6 and 4.8, 4096 14.9 and
  // 15.4, 8192 the same; 16 heads of 64: 2048 tokens 3.8 and 4.9, 4096 6.3 and 5.8, 32768 35.4 and 32.8. More heads of a token than a workgroup
  // takes at once go the way of few at any number of tokens: 136 heads of 128, 1024 tokens 13.9 and 13.3, 4096 48.5 and 52; 68 of 256
  // 14.2 and 13.6, 48.5 and 52.
  const bool few = (int64_t)r.n_tokens * a.n_total < (int64_t)512 * kMany * at_once || a.n_total > kMany * at_once;
  a.tokens = few ? 1 : kMany * at_once / a.n_total < kTokens ? kMany * at_once / a.n_total : kTokens;
  a.heads = few && a.n_total > at_once ? at_once : a.n_total;
  // Streaming stores where a head's runs are whole pieces of 64 bytes (8192 tokens of 40 heads of 128: 33.7 us against
  // 37.9; runs of 96 bytes: 11.8 and 9.9).
  a.stream = r.rot.layout == AQMB_ROTARY_INTERLEAVED || a.half % 8 ? r.head_dim % 64 == 0 : a.half % 32 == 0 && (r.head_dim - r.rot.rotary_dim) % 64 == 0;
  a.by_heads = (uint32_t)((0xFFFFFFFFull + a.heads) / a.heads);
  const dim3 grid((r.n_tokens + a.tokens - 1) / a.tokens, (a.n_total + a.heads - 1) / a.heads);
  const bool f16 = dtype == AQMB_F16;
  if (!cached) return f16 ? go<AQMB_F16, 0>(a, grid, lanes, few, st) : go<AQMB_BF16, 0>(a, grid, lanes, few, st);
  if (r.cache.dtype != AQMB_F8) return f16 ? go<AQMB_F16, 1>(a, grid, lanes, few, st) : go<AQMB_BF16, 1>(a, grid, lanes, few, st);
  return f16 ? go<AQMB_F16, 2>(a, grid, lanes, few, st) : go<AQMB_BF16, 2>(a, grid, lanes, few, st);
}

}  // namespace aqmb
