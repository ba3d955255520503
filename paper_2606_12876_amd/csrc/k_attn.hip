// Attention of one new token per sequence over a paged key-value cache.
//
//   score_t = scale <q, K_t>,  out = sum_t exp(score_t - m) V_t / sum_t exp(score_t - m)
//
// K and V are read once and nothing else is large, so HBM bounds it; everything below serves loads in
// flight. A workgroup takes a chunk of one sequence's positions for the (up to 16) query heads of one
// key-value head, its waves take turns at tiles of 32 positions, each with a running maximum and sum
// of its own. Both products run on the matrix cores without LDS:
//   S^T = K Q^T  rows: 16 positions, columns: heads. Lane (r, quarter) supplies the key of position
//                8 (r / 4) + r % 4 (second product: 4 more), so that the result leaves it with head r's
//                scores of positions 8 quarter .. 8 quarter + 7:
//   O^T = V^T P^T  is fed exactly that as its second operand. The first comes from the lane's own loads:
//                8 positions x 8 neighbouring values, transposed in registers (one byte permutation for
//                every two values).
// A column is a head in both, so maximum, sum and rescaling stay within a lane, but for two exchanges
// between the quarters per tile.
//
// Probabilities enter the second product as two 16-bit parts (value and remainder): rounding them once
// to bf16 would cost as much as rounding the result does when few positions carry the weight. bf16 parts hold
// 16 bits of a probability, fp16 parts 22. With an fp16 cache they are formed 2^14 larger, and relative to a
// tile's own largest where that is far below the maximum, so that small ones keep their digits above fp16's
// smallest subnormal: one is off by at most 2^-21 of itself or 2^-39 of the maximum, in a tile far below by 2^-38 of
// that tile's largest. An F8 cache is widened to bf16 for V (its scale joins the probability) and to the type of q
// for K (its scale joins the score): both exact.
//
// Chunks of a sequence are joined by a second kernel from (max, sum, unnormalised out) in the workspace.
#include "device.h"
#include "ops.h"
#include "wave.h"

namespace aqmb {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

constexpr int kTile = 32, kChunkMax = 4096, kXcds = 8;
constexpr int kWavesSplit = 4, kWavesWhole = 8;   // per workgroup, where sequences are split and where not
// The kernel's own LDS beside its dynamic part, at most: statistics, offsets and scales of 8 waves, joined statistics.
constexpr size_t kStaticLds = kWavesWhole * (2 * 16 * 4 + 32 * 8 + 64 * 4) + 2 * 16 * 4;

// The binary32 number next to another one on the side of 0; 0 for 0 (but not for -0).
__device__ __forceinline__ float below(float x) {
  return __builtin_bit_cast(float, __builtin_elementwise_sub_sat(__builtin_bit_cast(uint32_t, x), 1u));
}

// A probability (>= 0) by its value's scale. A product of -0 (a weight of 0, or a product too small, by a negative
// scale) becomes 0, which is what below knows; the addition must not be drawn into the product.
__device__ __forceinline__ float by_scale(float p, float scale) {
#pragma clang fp contract(off)
  return p * scale + 0.f;
}

// split: two probabilities (of an 8-bit cache: times their scales) as two 16-bit parts each, cut off rather than
// rounded and from just below, so that both parts of a positive one are positive: an infinite value of V then gives infinity,
// not the NaN that inf * 0 or inf - inf would be. A zero stays zero. fp16: the first part is also 2^-24, fp16's
// smallest number, below, which leaves that much for the second; the parts together are off by at most 2^-25 or
// 2^-21 of the probability, and one below 2^-23 is its second part alone.
template <int T> struct Mma;
template <> struct Mma<AQMB_F16> {
  static __device__ __forceinline__ f32x4_t mul(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_f16x2(lo, hi); }
  static __device__ __forceinline__ void split(float x, float y, uint32_t& a, uint32_t& b) {
    const float u = fmaxf(__builtin_fmaf(x, 1.f - 0x1p-23f, -0x1p-24f), 0.f), v = fmaxf(__builtin_fmaf(y, 1.f - 0x1p-23f, -0x1p-24f), 0.f);
    a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(u, v));
    b = pack_f16x2(x - f16lo(a), y - f16hi(a));
  }
  static constexpr float kShift = 14.f;
};
template <> struct Mma<AQMB_BF16> {
  static __device__ __forceinline__ f32x4_t mul(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16x2(lo, hi); }
  static __device__ __forceinline__ void split(float x, float y, uint32_t& a, uint32_t& b) {
    a = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, below(y)), __builtin_bit_cast(uint32_t, below(x)), 0x07060302u);
    b = pack_bf16x2(x - bf16lo(a), y - bf16hi(a));
  }
  static constexpr float kShift = 0.f;
};

// A tile whose largest score is this much (in units of log 2) below the maximum so far: probabilities 2^-26 of
// its largest are still whole numbers of 2^-24.
constexpr float kFar = 12.f;
__device__ __forceinline__ float power_of_2(int e) { return __builtin_bit_cast(float, (127 + e) << 23); }

// Four e4m3 values (one dword) widened to 16 bits, exactly: one instruction for two, where the way through
// binary32 takes three (and 7 registers more: 3 workgroups on a unit, not 4). One stream of 65536: 31.4 us
// against 33.0; 128 of up to 2000: 63 against 76.
template <int T>
__device__ __forceinline__ uint2 widen_f8(uint32_t w) {
  if constexpr (T == AQMB_BF16)
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true)));
  else
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true)));
}

// Raw loads of 8 (DC >= 8) or 4 values of the cache.
template <bool F8, int N> struct Raw;
template <> struct Raw<false, 8> { typedef u32x4_t T; };
template <> struct Raw<false, 4> { typedef uint2 T; };
template <> struct Raw<true, 8> { typedef uint2 T; };
template <> struct Raw<true, 4> { typedef uint32_t T; };

template <int T, bool F8>
__device__ __forceinline__ u32x4_t as16(typename Raw<F8, 8>::T r) {
  if constexpr (F8) {
    const uint2 a = widen_f8<T>(r.x), b = widen_f8<T>(r.y);
    return u32x4_t{a.x, a.y, b.x, b.y};
  } else {
    return r;
  }
}
template <int T, bool F8>
__device__ __forceinline__ uint2 as16h(typename Raw<F8, 4>::T r) {
  if constexpr (F8) return widen_f8<T>(r);
  else return r;
}

__device__ __forceinline__ uint32_t lo_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t hi_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// f over the four quarters of a wave.
template <class F>
__device__ __forceinline__ float quarters(float x, F f) {
  return __builtin_bit_cast(float, butterfly<32>(butterfly<16>(__builtin_bit_cast(uint32_t, x), f), f));
}
__device__ __forceinline__ uint32_t max_floats(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
}

// A launch takes fewer than 2^32 threads along a dimension: longer rows of workgroups go on along the next. A
// multiple of kXcds.
constexpr int kGridX = 1 << 20;
static dim3 folded(int64_t workgroups) {
  return workgroups <= kGridX ? dim3((unsigned)workgroups) : dim3(kGridX, (unsigned)((workgroups + kGridX - 1) / kGridX));
}

struct AttnDev {
  AttnArgs a;
  int page_shift;          // log2 of page_size, -1 if it is no power of two
  uint32_t page_magic;     // 2^32 / page_size + 1, then
  uint32_t quad_magic;     // 2^32 / (head_dim / 4) + 1
  int group, head_tiles;   // query heads per key-value head, in tiles of 16
  int block, blocks;       // 0, or the tiles of the heads that share cache lines, and such blocks in all
};

// 16 bytes at a multiple of 8.
struct __attribute__((packed, aligned(8))) Half16 { uint32_t w[4]; };

// T: type of q and of the products with K; PT: type of the products with V. DC: values of V per lane
// and position, head_dim <= 16 DC.
template <int T, int PT, bool F8, int DC, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void attn_kernel(AttnDev A) {
  const AttnArgs& a = A.a;
  constexpr int kS = DC / 2;             // steps of 32 along head_dim for S
  constexpr int VN = DC >= 8 ? 8 : 4;    // values per V load
  constexpr int VL = DC / VN;            // V loads per position
  constexpr size_t E = F8 ? 1 : 2;
  extern __shared__ int pages[];         // the chunk's page numbers, -1 where there is none
  __shared__ float s_ml[kWaves][2][16], s_join[2][16];
  __shared__ __attribute__((aligned(16))) int64_t s_row[kWaves][32];      // byte offsets of a tile's positions
  __shared__ __attribute__((aligned(16))) float s_scale[kWaves][64];      // scales of its keys, then values
  static_assert(sizeof(s_ml) + sizeof(s_join) + sizeof(s_row) + sizeof(s_scale) <= kStaticLds, "launch attribute");

  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane % 16, q = lane / 16;
  // Workgroups go to the XCDs in turn. Either heads do (every XCD has a share of every sequence), or, where
  // heads share cache lines or keys, those of a (sequence, chunk) that do follow each other on one XCD, so
  // that its L2 serves all but the first; sequences are turned by one per chunk, so that an XCD does not
  // keep the same ones. Chunks come last in both: the first ones, which every sequence has, run first, and no
  // XCD is left with the late chunks that short sequences lack (64 ragged streams: 155 us, of which 30 were that).
  int kvh = blockIdx.x, ht = 0, seq = blockIdx.y, split = blockIdx.z;
  if (A.block) {
    const int id = blockIdx.y * kGridX + blockIdx.x;            // one row of workgroups, folded where it is long
    const int k = id / kXcds, unit = k / A.block * kXcds + id % kXcds, row = a.n_seqs * A.blocks;
    if (unit >= row * a.n_splits) return;
    split = unit / row;
    const int rest = unit - split * row, s = rest / A.blocks, head = (rest - s * A.blocks) * A.block + k % A.block;
    seq = (s + split) % a.n_seqs;
    kvh = head / A.head_tiles;
    ht = head % A.head_tiles;
  }
  const int h0 = kvh * A.group + ht * 16;                       // first query head
  const int nh = min(16, A.group - ht * 16);
  // Without a window the chunk's place does not depend on the length: pages, length and q are asked for
  // together, and pages past the length (there may be any number in the table) are not looked at later.
  const int len = max(0, min(a.lengths[seq], a.max_length));
  const int lo = a.window > 0 ? max(0, len - a.window) : 0;
  const int c0 = (lo & ~7) + split * a.chunk, c1 = min(len, c0 + a.chunk);
  const int reach = max(0, min(a.max_length, c0 + a.chunk) - 1);
  const int p0 = A.page_shift >= 0 ? c0 >> A.page_shift : c0 / a.page_size;
  const int np = (A.page_shift >= 0 ? reach >> A.page_shift : reach / a.page_size) - p0 + 1;
  if (c0 < a.max_length)
    for (int i = threadIdx.x; i < np; i += 64 * kWaves) {
      const int p = a.table[seq * a.table_stride + p0 + i];
      pages[i] = p >= 0 && p < a.n_pages ? p : -1;
    }

  // Q^T as the second operand: lane (r, q) holds 8 values of head r for each step s of the product. Which
  // ones is free as long as K does the same: 32 s + 8 q .., or with an 8-bit cache, where a lane loads 16
  // values at a time, 64 (s / 2) + 16 q + 8 (s % 2) ...
  auto dim_of = [&](int s) { return F8 ? 64 * (s / 2) + 16 * q + 8 * (s % 2) : 32 * s + 8 * q; };
  u32x4_t qf[kS];
  {
    const uint16_t* qr = (const uint16_t*)a.q + seq * a.q_stride + (int64_t)(h0 + min(r, nh - 1)) * a.head_dim;
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      const int d = dim_of(s);
      qf[s] = d < a.head_dim ? *(const u32x4_t*)(qr + d) : u32x4_t{0, 0, 0, 0};
    }
  }
  if (c0 >= len) {                                              // no positions here
    if (split == 0 && a.n_splits == 1) {
      for (int e = threadIdx.x; e < nh * a.head_dim; e += 64 * kWaves) {
        const int h = h0 + e / a.head_dim;
        ((uint16_t*)a.out)[seq * a.out_stride + (int64_t)h * a.head_dim + e % a.head_dim] = 0;
      }
      if (a.lse && threadIdx.x < nh) a.lse[(int64_t)seq * a.n_heads + h0 + threadIdx.x] = -__builtin_inff();
    }
    return;
  }
  __syncthreads();

  const int base = p0 * a.page_size;                            // position of the chunk's first page
  const char* kb = (const char*)a.k + (int64_t)kvh * a.head_stride * E;
  const char* vb = (const char*)a.v + (int64_t)kvh * a.head_stride * E;
  const float scale2 = a.scale * 1.4426950408889634f;           // scores in units of log 2

  f32x4_t o[DC];
#pragma unroll
  for (int e = 0; e < DC; ++e) o[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m = -__builtin_inff(), l = 0.f;

  const int first = c0 + kTile * wave;
  for (int t0 = first; t0 < c1; t0 += kTile * kWaves) {
    // One look-up for each position of the tile, by lane % 32; LDS hands the offsets (and scales) round.
    // Positions outside are read at one inside and take no part (mask).
    const int pos = t0 + lane % 32;
    const uint32_t rel = (uint32_t)(max(lo, min(pos, c1 - 1)) - base);
    const uint32_t pi = A.page_shift >= 0 ? rel >> A.page_shift : __umulhi(rel, A.page_magic);
    const int page = pages[pi], slot = (int)(rel - pi * (uint32_t)a.page_size);
    const uint32_t mask = (uint32_t)__ballot(pos >= lo && pos < c1 && page >= 0);
    const int64_t pg = max(page, 0);
    s_row[wave][lane % 32] = (pg * a.page_stride + (int64_t)slot * a.slot_stride) * (int64_t)E;
    if constexpr (F8)
      s_scale[wave][lane] = (lane < 32 ? a.k_scale : a.v_scale)[pg * a.sc_page + (int64_t)kvh * a.sc_head + (int64_t)slot * a.sc_slot];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const uint32_t vmask = mask >> (8 * q) & 0xFFu;             // bit j: position 8 q + j takes part

    // Keys of two positions, values of eight.
    u32x4_t kr[2][F8 ? kS / 2 : kS];
    typename Raw<F8, VN>::T vr[8][VL];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const char* p = kb + s_row[wave][8 * (r / 4) + r % 4 + 4 * b];
#pragma unroll
      for (int s = 0; s < (F8 ? kS / 2 : kS); ++s) {
        const int d = dim_of(F8 ? 2 * s : s);
        if constexpr (!F8) {
          kr[b][s] = *(const u32x4_t*)(p + (d < a.head_dim ? d : 0) * E);
        } else if (a.head_dim % 16 == 0) {
          kr[b][s] = __builtin_bit_cast(u32x4_t, *(const Half16*)(p + (d < a.head_dim ? d : 0)));
        } else {
          const uint2 x = *(const uint2*)(p + (d < a.head_dim ? d : 0)), y = *(const uint2*)(p + (d + 8 < a.head_dim ? d + 8 : 0));
          kr[b][s] = u32x4_t{x.x, x.y, y.x, y.y};
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const char* p = vb + s_row[wave][8 * q + j];
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        const int d = r * DC + i * VN;
        vr[j][i] = *(const typename Raw<F8, VN>::T*)(p + (d < a.head_dim ? d : 0) * E);
      }
    }
    // The 8 scales of this lane's positions, of keys (which = 0) or values (1); read when they are needed.
    auto scales = [&](int which, float* to) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4_t x = *(const f32x4_t*)&s_scale[wave][32 * which + 8 * q + 4 * h];
#pragma unroll
        for (int e = 0; e < 4; ++e) to[4 * h + e] = x[e];
      }
    };

    f32x4_t sa = {0.f, 0.f, 0.f, 0.f}, sb = sa;
    const bool ragged = a.head_dim % (F8 ? 64 : 32) != 0;       // steps that reach past head_dim
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      u32x4_t ka, kc;
      if constexpr (F8) {
        const int h = 2 * (s % 2);
        ka = as16<T, true>(make_uint2(kr[0][s / 2][h], kr[0][s / 2][h + 1]));
        kc = as16<T, true>(make_uint2(kr[1][s / 2][h], kr[1][s / 2][h + 1]));
      } else {
        ka = kr[0][s];
        kc = kr[1][s];
      }
      if (ragged && dim_of(s) >= a.head_dim) ka = kc = u32x4_t{0, 0, 0, 0};
      sa = Mma<T>::mul(ka, qf[s], sa);
      sb = Mma<T>::mul(kc, qf[s], sb);
    }
    float p[8], sc[8];
    if constexpr (F8) scales(0, sc);
    float top = -__builtin_inff();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      p[j] = (j < 4 ? sa[j] : sb[j - 4]) * scale2;
      if constexpr (F8) p[j] *= sc[j];
      if (!(vmask >> j & 1)) p[j] = -__builtin_inff();
      top = fmaxf(top, p[j]);
    }
    top = quarters(top, max_floats);
    const float m2 = fmaxf(m, top);
    float mu = m2 == -__builtin_inff() ? 0.f : m2 - Mma<PT>::kShift;
    // fp16 parts of a tile far below the maximum would have few digits left or none: they are formed 2^up larger,
    // and the sums (at most 2^42) with them for the length of this tile.
    int up = 0;
    if constexpr (PT == AQMB_F16) {
      up = m2 - top > kFar ? (int)fminf(m2 - top, 60.f) : 0;
      mu -= (float)up;
    }
    if (t0 != first && __any(m2 > m || up > 0)) {
      float f = __builtin_amdgcn_exp2f(m2 == -__builtin_inff() ? 0.f : m - m2);
      if constexpr (PT == AQMB_F16) f = up > 0 ? power_of_2(up) : f;
      l *= f;
#pragma unroll
      for (int e = 0; e < DC; ++e) o[e] *= f;
    }
    m = m2;
    if constexpr (F8) scales(1, sc);
    uint32_t ph[4], pl[4];
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      float x = __builtin_amdgcn_exp2f(p[j] - mu), y = __builtin_amdgcn_exp2f(p[j + 1] - mu);
      l += x + y;
      if constexpr (F8) {
        x = vmask >> j & 1 ? by_scale(x, sc[j]) : 0.f;
        y = vmask >> (j + 1) & 1 ? by_scale(y, sc[j + 1]) : 0.f;
      }
      Mma<PT>::split(x, y, ph[j / 2], pl[j / 2]);
    }
    const u32x4_t pho = {ph[0], ph[1], ph[2], ph[3]}, plo = {pl[0], pl[1], pl[2], pl[3]};

    // V^T: values of 8 positions, transposed. A position that takes no part must be 0, not garbage; rows of
    // V^T past head_dim may be anything, they are rows of a result that nobody reads.
#pragma unroll
    for (int i = 0; i < DC / 4; ++i) {                           // 4 values at a time
      uint2 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (VN == 4) {
          v[j] = as16h<PT, F8>(vr[j][i]);
        } else if constexpr (F8) {
          v[j] = widen_f8<PT>(i % 2 ? vr[j][i / 2].y : vr[j][i / 2].x);
        } else {
          v[j] = make_uint2(vr[j][i / 2][2 * (i % 2)], vr[j][i / 2][2 * (i % 2) + 1]);
        }
      }
      if (mask != 0xFFFFFFFFu) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = vmask >> j & 1 ? v[j] : make_uint2(0, 0);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        u32x4_t w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t x = e < 2 ? v[2 * j].x : v[2 * j].y, y = e < 2 ? v[2 * j + 1].x : v[2 * j + 1].y;
          w[j] = e % 2 ? hi_halves(x, y) : lo_halves(x, y);
        }
        o[4 * i + e] = Mma<PT>::mul(w, pho, o[4 * i + e]);
        o[4 * i + e] = Mma<PT>::mul(w, plo, o[4 * i + e]);
      }
    }
    if constexpr (PT == AQMB_F16) {
      if (__any(up > 0)) {
        const float f = power_of_2(-up);
        l *= f;
#pragma unroll
        for (int e = 0; e < DC; ++e) o[e] *= f;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }

  // The quarters' sums of one head, then the waves.
  l = quarters(l, add_floats);
  if (q == 0) {
    s_ml[wave][0][r] = m;
    s_ml[wave][1][r] = l;
  }
  __syncthreads();                        // also: every wave is done with pages
  float M = -__builtin_inff(), L = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_ml[w][0][r]);
  const float Mu = M == -__builtin_inff() ? 0.f : M;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) L += s_ml[w][1][r] * __builtin_amdgcn_exp2f(s_ml[w][0][r] - Mu);
  const float mine = __builtin_amdgcn_exp2f(m - Mu);            // 0 for a wave without positions
  // The waves' sums, [kWaves][nh][head_dim + 4]: 4 values at a time, the pad turns a column of heads
  // over all banks.
  const int pitch = a.head_dim + 4;
  float* so = (float*)pages;
  if (r < nh) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < DC; e += 4) {
        const int d = (4 * q + i) * DC + e;
        if (d < a.head_dim)
          *(f32x4_t*)(so + (wave * nh + r) * pitch + d) =
              f32x4_t{o[e][i] * mine, o[e + 1][i] * mine, o[e + 2][i] * mine, o[e + 3][i] * mine};
      }
  }
  if (wave == 0 && q == 0) {              // the joined statistics, for the lines below
    s_join[0][r] = M;
    s_join[1][r] = L;
  }
  __syncthreads();
  // A sum is 0 only where no position takes part, NaN where a score is: then out and lse are NaN too.
  const bool one = a.n_splits == 1;
  const int quads = a.head_dim / 4;
  for (int e = threadIdx.x; e < nh * quads; e += 64 * kWaves) {
    const int h = (int)__umulhi((uint32_t)e, A.quad_magic), d = (e - h * quads) * 4;
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += *(const f32x4_t*)(so + (w * nh + h) * pitch + d);
    if (one) {
      const float sum = s_join[1][h];
      if (sum > 0.f) v /= sum;
      uint16_t* out = (uint16_t*)a.out + seq * a.out_stride + (int64_t)(h0 + h) * a.head_dim + d;
      *(uint2*)out = make_uint2(Mma<T>::pack(v[0], v[1]), Mma<T>::pack(v[2], v[3]));
    } else {
      *(f32x4_t*)(a.part + (((int64_t)seq * a.n_heads + h0 + h) * a.n_splits + split) * a.head_dim + d) = v;
    }
  }
  if (threadIdx.x < nh) {
    const float mm = s_join[0][threadIdx.x], sum = s_join[1][threadIdx.x];
    const int64_t at = (int64_t)seq * a.n_heads + h0 + threadIdx.x;
    if (!one) {
      float* ml = a.part + (int64_t)a.n_seqs * a.n_heads * a.n_splits * a.head_dim;
      ml[(at * a.n_splits + split) * 2] = mm;
      ml[(at * a.n_splits + split) * 2 + 1] = sum;
    } else if (a.lse) {
      a.lse[at] = sum == 0.f ? -__builtin_inff() : (mm - Mma<PT>::kShift + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
    }
  }
}

// Joins the chunks of a (sequence, head): head_dim / 4 lanes read a chunk's sum. Up to kFewChunks, those
// lanes take one chunk after the other (with the loads under way together) and a workgroup has several
// heads; beyond, a workgroup has one head and each group of lanes every so-many-th chunk with a running
// maximum of its own, and the groups meet in LDS. 64 streams x 32 heads x 2 chunks: 7.3 us by the second
// form, 4.8 by the first; 16 chunks of one stream 3.8 and 4.0. Between these the limit is a guess: nothing was timed.
constexpr int kJoin = 512, kJoinFew = 256, kFewChunks = 4;

__device__ __forceinline__ int chunks_of(const AttnArgs& a, int seq) {
  const int len = max(0, min(a.lengths[seq], a.max_length));
  const int lo = a.window > 0 ? max(0, len - a.window) : 0;
  return len > 0 ? (len - (lo & ~7) + a.chunk - 1) / a.chunk : 0;
}
template <int T>
__device__ __forceinline__ void store_joined(const AttnArgs& a, int64_t at, int seq, int d, f32x4_t v, float top, float sum,
                                             float shift) {
  if (sum > 0.f) v /= sum;
  uint16_t* out = (uint16_t*)a.out + seq * a.out_stride + (at - (int64_t)seq * a.n_heads) * a.head_dim + d;
  *(uint2*)out = make_uint2(Mma<T>::pack(v[0], v[1]), Mma<T>::pack(v[2], v[3]));
  if (a.lse && d == 0)
    a.lse[at] = sum == 0.f ? -__builtin_inff() : (top - shift + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

// chunk i's statistics and sum added to a running (M, L, v)
__device__ __forceinline__ void join_one(float m, float l, f32x4_t x, float& M, float& L, f32x4_t& v) {
  const float m2 = fmaxf(M, m), mu = m2 == -__builtin_inff() ? 0.f : m2;
  const float f = __builtin_amdgcn_exp2f(M - mu), e = __builtin_amdgcn_exp2f(m - mu);
  L = L * f + l * e;
  v = v * f + x * e;
  M = m2;
}

template <int T>
__global__ __launch_bounds__(kJoinFew) void attn_join_few_kernel(AttnArgs a, float shift) {
  const int quads = a.head_dim / 4, heads = kJoinFew / quads, g = threadIdx.x / quads, d = threadIdx.x % quads * 4;
  const int64_t at = ((int64_t)blockIdx.y * kGridX + blockIdx.x) * heads + g;
  if (g >= heads || at >= (int64_t)a.n_seqs * a.n_heads) return;
  const int seq = (int)(at / a.n_heads), n = chunks_of(a, seq);
  const float* ml = a.part + (int64_t)a.n_seqs * a.n_heads * a.n_splits * a.head_dim + at * a.n_splits * 2;
  const float* part = a.part + at * a.n_splits * a.head_dim + d;
  float M = -__builtin_inff(), L = 0.f;
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = 0; i < n; ++i) join_one(ml[2 * i], ml[2 * i + 1], *(const f32x4_t*)(part + i * a.head_dim), M, L, v);
  store_joined<T>(a, at, seq, d, v, M, L, shift);
}

template <int T>
__global__ __launch_bounds__(kJoin) void attn_join_kernel(AttnArgs a, float shift) {
  __shared__ __attribute__((aligned(16))) float so[kJoin][4];
  __shared__ float sm[kJoin], sl[kJoin];
  const int seq = blockIdx.y, n = chunks_of(a, seq);
  const int64_t at = (int64_t)seq * a.n_heads + blockIdx.x;
  const float* ml = a.part + (int64_t)a.n_seqs * a.n_heads * a.n_splits * a.head_dim + at * a.n_splits * 2;
  const float* part = a.part + at * a.n_splits * a.head_dim;
  const int quads = a.head_dim / 4, groups = kJoin / quads, g = threadIdx.x / quads, d = threadIdx.x % quads * 4;
  float M = -__builtin_inff(), L = 0.f;
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
  if (g < groups) {
#pragma unroll 4
    for (int i = g; i < n; i += groups)
      join_one(ml[2 * i], ml[2 * i + 1], *(const f32x4_t*)(part + (int64_t)i * a.head_dim + d), M, L, v);
  }
  sm[threadIdx.x] = M;
  sl[threadIdx.x] = L;
  *(f32x4_t*)so[threadIdx.x] = v;
  __syncthreads();
  if (threadIdx.x >= quads) return;
  const int used = min(groups, n);
#pragma unroll 4
  for (int k = 1; k < used; ++k) {
    const int e = k * quads + threadIdx.x;
    join_one(sm[e], sl[e], *(const f32x4_t*)so[e], M, L, v);
  }
  store_joined<T>(a, at, seq, d, v, M, L, shift);
}


AttnPlan attn_plan(int n_heads, int n_kv, int head_dim, int n_seqs, int max_length, int window, int n_cu) {
  // A window reaches from the 8 positions that its first one is in.
  const int64_t span = window > 0 && window < max_length ? (int64_t)window + 7 : max_length;
  const int64_t groups = (int64_t)n_seqs * n_kv * ((n_heads / n_kv + 15) / 16);

  // Workgroups along a sequence: two on every unit, five where several sequences (whose lengths differ) need to
  // be levelled out: three run at once with a 16-bit cache, four with an 8-bit one. One sequence of 131072: 97 us
  // with two, 104 with four. Ragged streams, over eight sets of lengths, with four, five, six and eight: 32 of up
  // to 6000, 16 bits, 89, 87, 90, 88 us; 200 of up to 1500 124, 121, 121, 125. 8 bits, with five, six and eight: 64
  // of up to 8192 122, 121, 131; 8 of up to 16000 44, 50, 48.
  const int64_t want = ((n_seqs > 1 ? 5 : 2) * (int64_t)n_cu + groups - 1) / groups;
  int64_t chunk = (span + want - 1) / want;
  const int64_t unit = kTile * kWavesSplit;
  chunk = (chunk + unit - 1) / unit * unit;
  chunk = chunk < unit ? unit : chunk > kChunkMax ? kChunkMax : chunk;
  AttnPlan p;
  // Short sequences stay whole, with twice the waves, which saves the second launch; where they leave most of the
  // card idle, a quarter less is short (384 positions with heads of 128; from there to about 450 there is little in it). Calls in sequence, whole and split, 8 key-value heads of 128 (queries 4
  // times as many): one sequence of 300, 6.8 and 8.5 us; of 400, 7.7 and 7.9; of 500, 8.3 and 7.9; 64 of up to 500,
  // 16.6 and 18.9. Heads of 64: one of 700, 7.3 and 7.8 us; of 1000, 8.8 and 7.8; 64 of up to 1000, 16.3 and 19.8.
  // Heads of 256, 2 of 250: 9.2 and 9.9.
  const int whole = head_dim <= 64 ? 1024 : head_dim <= 128 ? 512 : 256;
  p.waves = kWavesSplit;
  if (span <= (head_dim <= 128 && groups < n_cu / 2 ? whole - whole / 4 : whole) && span > chunk) {
    p.waves = kWavesWhole;
    chunk = (span + kTile - 1) / kTile * kTile;
  }
  const int64_t n = span > 0 ? (span + chunk - 1) / chunk : 1;
  p.chunk = (int)chunk;
  p.n_splits = (int)n;
  p.bytes = n == 1 ? 0 : (size_t)n_seqs * n_heads * n * (head_dim + 2) * sizeof(float);
  return p;
}

template <int T, int PT, bool F8>
static hipError_t go(const AttnArgs& a, hipStream_t st) {
  AttnDev A;
  A.a = a;
  // Quotients by multiplication: exact while numerator times divisor stays below 2^32 (positions of a chunk
  // and a page, at most 36896, by 32768; 16 heads by 64).
  A.page_shift = (a.page_size & (a.page_size - 1)) == 0 ? __builtin_ctz((unsigned)a.page_size) : -1;
  A.page_magic = a.page_size > 1 ? (uint32_t)((1ull << 32) / (uint32_t)a.page_size + 1) : 0;
  A.quad_magic = (uint32_t)((1ull << 32) / (uint32_t)(a.head_dim / 4) + 1);
  A.group = a.n_heads / a.n_kv;
  A.head_tiles = (A.group + 15) / 16;
  const int nh = A.group < 16 ? A.group : 16;
  const size_t tab = (size_t)(a.chunk / a.page_size + 2) * sizeof(int);
  const size_t acc = (size_t)a.waves * nh * (a.head_dim + 4) * sizeof(float);
  const size_t lds = tab > acc ? tab : acc;
  // Heads share cache lines (128 bytes) where tokens are outermost in a page and a head does not fill whole
  // lines. Under 192 bytes they are taken in the smallest blocks that do; 25 ragged streams of up to 4557, 8 heads:
  // of 160 bytes in fours and each by itself, 47.8 us both (64 of up to 2000: 55.6 and 58.6; 4 of up to 20000:
  // 32 and 42; all 8 heads on one XCD: 58, 62 and 37); of 96, 41.3 and 47.0; of 192, 52.0 and 48.3; of 64, 33.3
  // and 35.7. Tiles of heads share the keys and values themselves.
  const int bytes = a.head_dim * (F8 ? 1 : 2);
  int share = 1;
  if (a.sc_head == 1 && bytes < 192)
    while (share < a.n_kv && share * bytes % 128 != 0) share *= 2;
  if (a.n_kv % share != 0) share = a.n_kv;
  A.block = share * A.head_tiles > 1 ? share * A.head_tiles : 0;
  A.blocks = a.n_kv / share;
  const int64_t units = (int64_t)a.n_seqs * a.n_splits * A.blocks;
  const int64_t ids = (units + kXcds - 1) / kXcds * kXcds * A.block;
  if (ids > 0x7FFFFFFF - kGridX) return hipErrorInvalidValue;
  const dim3 grid = A.block ? folded(ids) : dim3(a.n_kv, a.n_seqs, a.n_splits);
  hipError_t e = hipSuccess;
  auto run = [&](auto kernel) {
    if (lds + kStaticLds > 65536) e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e == hipSuccess) kernel<<<grid, 64 * a.waves, lds, st>>>(A);
    if (e == hipSuccess) e = hipGetLastError();
  };
  if (a.waves == kWavesSplit) {
    if (a.head_dim <= 64) run(attn_kernel<T, PT, F8, 4, kWavesSplit>);
    else if (a.head_dim <= 128) run(attn_kernel<T, PT, F8, 8, kWavesSplit>);
    else run(attn_kernel<T, PT, F8, 16, kWavesSplit>);
  } else {
    if (a.head_dim <= 64) run(attn_kernel<T, PT, F8, 4, kWavesWhole>);
    else if (a.head_dim <= 128) run(attn_kernel<T, PT, F8, 8, kWavesWhole>);
    else run(attn_kernel<T, PT, F8, 16, kWavesWhole>);
  }
  if (e != hipSuccess || a.n_splits == 1) return e;
  if (a.n_splits <= kFewChunks) {
    const int heads = kJoinFew / (a.head_dim / 4);
    const int64_t all = (int64_t)a.n_heads * a.n_seqs;
    attn_join_few_kernel<T><<<folded((all + heads - 1) / heads), kJoinFew, 0, st>>>(a, Mma<PT>::kShift);
  } else {
    attn_join_kernel<T><<<dim3(a.n_heads, a.n_seqs), kJoin, 0, st>>>(a, Mma<PT>::kShift);
  }
  return hipGetLastError();
}

hipError_t launch_attention(const AttnArgs& a, aqmb_dtype dtype, bool f8, hipStream_t st) {
  if (f8) return dtype == AQMB_F16 ? go<AQMB_F16, AQMB_BF16, true>(a, st) : go<AQMB_BF16, AQMB_BF16, true>(a, st);
  return dtype == AQMB_F16 ? go<AQMB_F16, AQMB_F16, false>(a, st) : go<AQMB_BF16, AQMB_BF16, false>(a, st);
}

}  // namespace aqmb
