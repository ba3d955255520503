// Decode product with 4-bit weights, a scale (and zero point) for every group of a row:
//
//   y[b][i] = sum_g s[i][g] sx[b][g] (sum_{t in g} q[i][t] x[b][t] - z[i][g] sum_{t in g} x[b][t])
//
// A wave multiplies tiles of 16 rows x 128 inputs by up to 16 rows of x on the matrix cores: four
// 16 x 16 x 32 products, each fed by one dword of nibbles per lane. The nibbles become operands
// without a conversion, because the layout of the tile puts them where a mask leaves numbers that the
// matrix cores read as they are:
//   fp16  0x4C00 | q << 6 is 16 + q; the 16 joins the zero point
//   bf16  0x4180 | q << 3 is 16 + q
//   int8  q itself
// An e4m3 x is widened to fp16, exactly, and takes the fp16 form. Cheaper forms were dropped because
// they lose digits: the subnormals 0x000q of fp16 and 0x0q of e4m3 stand for q 2^-24 and q 2^-9, but the
// matrix cores line products up by their unnormalised exponents, and a sum of them keeps only about 17
// bits (measured: 1.1e-4 of the result at 4096 x 4096).
// A dword of eight weights costs 3 (int8) or 8 vector instructions. sum x is a second product with a row
// of ones: it arrives in every lane that needs it, with the same grouping and order of sums.
#include <type_traits>

#include "device.h"
#include "ops.h"

namespace aqmb {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

// ------------------------------------------------------------------ layout
// One thread per dword of the tiles.
__global__ void w4_pack_kernel(const uint8_t* w, uint32_t* tiles, int d_out, int d_in, int n_kt, size_t n) {
  const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n) return;
  const int s = i % 4, lane = i / 4 % 64;
  const size_t tile = i / 256;
  const int row = (int)(tile / n_kt) * kW4Rows + lane % 16;
  const int k0 = (int)(tile % n_kt) * kW4Cols + 32 * s + 8 * (lane / 16);
  const size_t pitch = ((size_t)d_in + 1) / 2;
  uint32_t v = 0;
  for (int p = 0; p < 8; ++p) {
    const int k = k0 + (p < 4 ? 2 * p : 2 * p - 7);
    if (row < d_out && k < d_in) {
      const uint32_t b = w[(size_t)row * pitch + k / 2];
      v |= (k % 2 ? b >> 4 : b & 15u) << (4 * p);
    }
  }
  tiles[i] = v;
}

// Scales and zero points of a tile, [row / 4][group][row % 4]: a lane's share is one piece.
__global__ void w4_pack_scales_kernel(const uint16_t* s, const uint8_t* z, uint16_t* so, uint8_t* zo, int d_out,
                                      int groups, int n_kt, int per, size_t n) {
  const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n) return;
  const size_t tile = i / (16 * per);
  const int e = (int)(i % (16 * per));
  const int row = (int)(tile / n_kt) * kW4Rows + e / (4 * per) * 4 + e % 4, g = (int)(tile % n_kt) * per + e / 4 % per;
  const bool in = row < d_out && g < groups;
  so[i] = in ? s[(size_t)row * groups + g] : 0;
  if (z) zo[i] = in ? z[(size_t)row * groups + g] : 0;
  else if (i < 16 * per) zo[i] = 8;                    // one tile's
}

hipError_t launch_w4_pack(const W4& L, const uint8_t* weights, const uint16_t* scales, const uint8_t* zeros,
                          hipStream_t st) {
  const int g = L.d.group_size, groups = (L.d.d_in - 1) / g + 1, per = kW4Cols / g;
  const size_t n = (size_t)L.n_rt * L.n_kt * 256, ns = (size_t)L.n_rt * L.n_kt * per * 16;
  w4_pack_kernel<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(weights, (uint32_t*)L.tiles, L.d.d_out, L.d.d_in, L.n_kt, n);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  w4_pack_scales_kernel<<<(unsigned)((ns + 255) / 256), 256, 0, st>>>(scales, zeros, L.scales, L.zeros, L.d.d_out,
                                                                     groups, L.n_kt, per, ns);
  return hipGetLastError();
}

// ------------------------------------------------------------------ product
struct W4Args {
  const u32x4_t* tiles;
  const uint16_t* scales;
  const uint8_t* zeros;
  size_t zero_pitch;       // from tile to tile; 0 where all are 8
  const void* x;
  const float* x_scales;
  void* y;
  int64_t x_stride, y_stride;
  int d_out, d_in, n_kt, batch;
  int x_groups;            // scales of a row of x
  int y_dtype;
};

// 16 bytes of a row of x from element k on: rows start at any element, which 16-byte loads allow on gfx950.
struct __attribute__((packed, aligned(1))) Bytes16 { uint64_t lo, hi; };

// The same at the end of a row, zeros from element d_in on: the row's last 16 bytes, moved down by
// those that lie before k.
template <typename E>
__device__ __forceinline__ Bytes16 load_end(const E* row, int k, int d_in) {
  constexpr int kN = 16 / sizeof(E);
  Bytes16 v = {0, 0};
  if (k >= d_in) return v;
  if (d_in < kN) {                                    // k = 0: the whole row
#pragma unroll 1
    for (int i = 0; i < d_in; ++i) {
      const uint64_t e = row[i];
      const int s = 8 * (int)sizeof(E) * i;
      if (s < 64) v.lo |= e << s;
      else v.hi |= e << (s - 64);
    }
    return v;
  }
  const int past = max(k - (d_in - kN), 0) * (int)sizeof(E);      // 0..15 bytes
  v = *(const Bytes16*)(row + min(k, d_in - kN));
  const int s = 8 * (past % 8);
  if (past >= 8) v = {v.hi, 0};
  if (s) v = {v.lo >> s | v.hi << (64 - s), v.hi >> s};
  return v;
}

// Four e4m3 values as fp16, exactly.
__device__ __forceinline__ uint2 widen_f8(uint32_t w) {
  return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true)));
}

// How each type of x meets the nibbles. X: 8 neighbouring inputs of one row. kSixteens comes in a register
// (o): "and" and "or" are one instruction then, which takes at most one constant.
template <int XT> struct Op;
struct F16Form {
  typedef f16x8_t V;
  typedef f32x4_t C;
  static constexpr int kZero = 16;
  static constexpr uint32_t kSixteens = 0x4C004C00u;
  static __device__ __forceinline__ V weights(uint32_t w, uint32_t o) {
    const uint32_t m = 0x03C003C0u;
    return __builtin_bit_cast(V, u32x4_t{((w << 6) & m) | o, ((w << 2) & m) | o, ((w >> 2) & m) | o, ((w >> 6) & m) | o});
  }
  static __device__ __forceinline__ V ones() {
    return __builtin_bit_cast(V, u32x4_t{0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u});
  }
  static __device__ __forceinline__ C mul(V a, V b, C c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Op<AQMB_F16> : F16Form {
  typedef u32x4_t X;
  static __device__ __forceinline__ V operand(X x) { return __builtin_bit_cast(V, x); }
};
template <> struct Op<AQMB_F8> : F16Form {
  typedef uint2 X;
  static __device__ __forceinline__ V operand(X x) {
    const uint2 a = widen_f8(x.x), b = widen_f8(x.y);
    return __builtin_bit_cast(V, u32x4_t{a.x, a.y, b.x, b.y});
  }
};
template <> struct Op<AQMB_BF16> {
  typedef u32x4_t X;
  typedef bf16x8_t V;
  typedef f32x4_t C;
  static constexpr int kZero = 16;
  static constexpr uint32_t kSixteens = 0x41804180u;
  static __device__ __forceinline__ V weights(uint32_t w, uint32_t o) {
    const uint32_t m = 0x00780078u;
    return __builtin_bit_cast(V, u32x4_t{((w << 3) & m) | o, ((w >> 1) & m) | o, ((w >> 5) & m) | o, ((w >> 9) & m) | o});
  }
  static __device__ __forceinline__ V ones() {
    return __builtin_bit_cast(V, u32x4_t{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
  }
  static __device__ __forceinline__ V operand(X x) { return __builtin_bit_cast(V, x); }
  static __device__ __forceinline__ C mul(V a, V b, C c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Op<AQMB_I8> {
  typedef uint2 X;
  typedef long V;
  typedef i32x4_t C;
  static constexpr int kZero = 0;
  static constexpr uint32_t kSixteens = 0;
  static __device__ __forceinline__ V weights(uint32_t w, uint32_t) {
    const uint32_t m = 0x0F0F0F0Fu;
    return (long)((uint64_t)((w >> 4) & m) << 32 | (w & m));
  }
  static __device__ __forceinline__ V ones() { return 0x0101010101010101l; }
  // The masks leave weights 0, 4, 1, 5 and 2, 6, 3, 7; x has to follow.
  static __device__ __forceinline__ V operand(X x) {
    const uint32_t lo = __builtin_amdgcn_perm(x.y, x.x, 0x05010400u);
    const uint32_t hi = __builtin_amdgcn_perm(x.y, x.x, 0x07030602u);
    return (long)((uint64_t)hi << 32 | lo);
  }
  static __device__ __forceinline__ C mul(V a, V b, C c) { return __builtin_amdgcn_mfma_i32_16x16x32_i8(a, b, c, 0, 0, 0); }
};

// The scales (fp16) and zero points (uint8) that a lane needs of a tile: 4 rows of every group.
template <int N> struct Piece;
template <> struct Piece<4> {
  uint2 s; uint32_t z;
  __device__ __forceinline__ uint32_t scale(int e) const { return e < 2 ? s.x : s.y; }
  __device__ __forceinline__ uint32_t zero(int) const { return z; }
};
template <> struct Piece<8> {
  u32x4_t s; uint2 z;
  __device__ __forceinline__ uint32_t scale(int e) const { return s[e / 2]; }
  __device__ __forceinline__ uint32_t zero(int e) const { return e < 4 ? z.x : z.y; }
};
template <> struct Piece<16> {
  u32x4_t s, s2; u32x4_t z;
  __device__ __forceinline__ uint32_t scale(int e) const { return e < 8 ? s[e / 2] : s2[e / 2 - 4]; }
  __device__ __forceinline__ uint32_t zero(int e) const { return z[e / 4]; }
};

// A workgroup of W waves takes R tiles of 16 rows, which share x and its sums; wave w takes the input
// tiles w, w + W, ..., the next one under way while it works on one, and the waves' sums meet in LDS.
// G: the group size.
//
// x is read by rows (16 bytes a lane, neighbouring lanes neighbouring bytes) and brought into operand
// order through LDS: loads in operand order would have every lane on a row of its own, which costs the
// address unit a cycle a lane (4096 x 11008 at 16 rows of int8: 15 us so, of which the loads of x were 5).
// The 16-byte chunks of a row are stored at their number xor the row's, so that reads of 16 rows at
// one chunk spread over all banks. What bounds the kernel is instructions more than bytes, most of all
// those that a wave spends before its few turns of the loop: tile numbers are scalar, addresses of x
// advance by one addition, the ragged last tile has code of its own.
//
// Loads of the next tile are straight code (a choice between two values of a register would have to wait
// for both): the number of row loads NL is a parameter, symmetric layers have a piece of eights for zero
// points, one scale per row is one group.
template <int XT, int G, int R, int W, int NL>
__global__ __launch_bounds__(64 * W) void w4_kernel(W4Args a) {
  typedef Op<XT> O;
  typedef typename O::C C;
  typedef typename std::conditional<XT == AQMB_F16 || XT == AQMB_BF16, uint16_t, uint8_t>::type E;
  constexpr bool kWide = sizeof(E) == 2;
  constexpr int kSteps = G / 32, kGroups = kW4Cols / G;
  constexpr int kChunks = kW4Cols * (int)sizeof(E) / 16, kRows = 64 / kChunks;
  constexpr int kSlab = 16 * kChunks * 16;              // bytes of x a wave holds in LDS
  constexpr int kPart = R * 16 * 17 * 4;                // bytes of its sums, in the same place afterwards
  __shared__ __attribute__((aligned(16))) unsigned char lds[W * (kSlab > kPart ? kSlab : kPart)];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int n = lane % 16, q = lane / 16;
  unsigned char* slab = lds + wave * kSlab;
  const int rt0 = blockIdx.x * R, n_rt = (a.d_out - 1) / kW4Rows + 1;
  size_t tile0[R];                                      // of the strip's row tiles; the last may repeat
#pragma unroll
  for (int r = 0; r < R; ++r) tile0[r] = (size_t)min(rt0 + r, n_rt - 1) * a.n_kt;

  // This lane's part of the loads of x: row lane / kChunks (+ kRows per load), chunk lane % kChunks.
  const int k_lane = lane % kChunks * (16 / (int)sizeof(E));
  const E* xp[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i)
    xp[i] = (const E*)a.x + (int64_t)min(i * kRows + lane / kChunks, a.batch - 1) * a.x_stride;
  Bytes16 x[NL];
  auto load_x = [&](int kt) {
    if ((kt + 1) * kW4Cols <= a.d_in) {
#pragma unroll
      for (int i = 0; i < NL; ++i) x[i] = *(const Bytes16*)(xp[i] + (kt * kW4Cols + k_lane));
    } else {
#pragma unroll
      for (int i = 0; i < NL; ++i) x[i] = load_end(xp[i], kt * kW4Cols + k_lane, a.d_in);
    }
  };
  const float* xs = kWide ? nullptr : a.x_scales + (int64_t)min(n, a.batch - 1) * a.x_groups;
  struct Tile {
    u32x4_t w;
    Piece<4 * kGroups> p;
  };
  auto load_tile = [&](size_t tile) {
    Tile t;
    // Cached, not streaming: models of up to the Infinity Cache's 256 MB then find their weights there at the
    // next step (4096 x 11008 int8 at 16 rows: 7.4 against 9.7 us), for 3 to 5 % more where they do not fit.
    t.w = a.tiles[tile * 64 + lane];
    const uint16_t* s = a.scales + tile * (16 * kGroups);
    t.p.s = *(const decltype(t.p.s)*)(s + 4 * kGroups * q);
    if constexpr (kGroups == 4) t.p.s2 = *(const u32x4_t*)(s + 4 * kGroups * q + 8);
    t.p.z = *(const decltype(t.p.z)*)(a.zeros + tile * a.zero_pitch + 4 * kGroups * q);
    return t;
  };
  // Groups from the last of d_in on have scale 0 and x 0; an x scale there does not exist.
  float sx[kGroups], sx2[kGroups];
  auto load_sx = [&](float* to, int kt) {
    if constexpr (!kWide)
#pragma unroll
      for (int g = 0; g < kGroups; ++g) to[g] = xs[min(kt * kGroups + g, a.x_groups - 1)];
  };

  float tot[R][4];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < 4; ++i) tot[r][i] = 0.f;
  uint32_t sixteens = O::kSixteens;
  if constexpr (O::kSixteens != 0) asm("" : "+v"(sixteens));
  Tile cur[R];
  if (wave < a.n_kt) {
#pragma unroll
    for (int r = 0; r < R; ++r) cur[r] = load_tile(tile0[r] + wave);
    load_sx(sx, wave);
    load_x(wave);
  }
#pragma unroll 1
  for (int kt = wave; kt < a.n_kt; kt += W) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = i * kRows + lane / kChunks;
      *(u32x4_t*)(slab + (row * kChunks + (lane % kChunks ^ row % kChunks)) * 16) = __builtin_bit_cast(u32x4_t, x[i]);
    }
    // Lanes read what others of the wave wrote; LDS serves a wave's accesses in order.
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    Tile next[R];
    if (kt + W < a.n_kt) {
#pragma unroll
      for (int r = 0; r < R; ++r) next[r] = load_tile(tile0[r] + kt + W);
      load_sx(sx2, kt + W);
      load_x(kt + W);
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      // Rows of the slab past the batch hold anything: columns of the product that nobody reads.
      typename O::V v[kSteps];
      C ax = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int byte = (32 * (g * kSteps + s) + 8 * q) * (int)sizeof(E);
        v[s] = O::operand(*(const typename O::X*)(slab + (n * kChunks + (byte / 16 ^ n % kChunks)) * 16 + byte % 16));
        ax = O::mul(O::ones(), v[s], ax);
      }
      const C off = ax * -O::kZero;                      // the operands' offset, off before the products come
#pragma unroll
      for (int r = 0; r < R; ++r) {
        C acc = off;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) acc = O::mul(O::weights(cur[r].w[g * kSteps + s], sixteens), v[s], acc);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = 4 * g + i;                       // of the lane's piece
          const float s = e % 2 ? f16hi(cur[r].p.scale(e)) : f16lo(cur[r].p.scale(e));
          const float z = (float)((cur[r].p.zero(e) >> (8 * i)) & 0xFFu);
          float p = (float)acc[i] - z * (float)ax[i];     // int8: all of it exact, below 2^18
          if constexpr (!kWide) p *= sx[g];
          tot[r][i] += s * p;
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int r = 0; r < R; ++r) cur[r] = next[r];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) sx[g] = sx2[g];
  }
  __syncthreads();                                       // the slabs become the waves' sums
  float (*part)[R][16][17] = (float (*)[R][16][17])lds;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < 4; ++i) part[wave][r][4 * q + i][n] = tot[r][i];
  __syncthreads();
  for (int e = threadIdx.x; e < R * 256; e += 64 * W) {
    const int row = e % 16, b = e / 16 % 16, r = e / 256, out = (rt0 + r) * kW4Rows + row;
    if (b >= a.batch || out >= a.d_out) continue;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) v += part[k][r][row][b];
    const size_t at = (size_t)b * a.y_stride + out;
    if (a.y_dtype == AQMB_F16) OutT<AQMB_F16>::store(a.y, at, v);
    else if (a.y_dtype == AQMB_BF16) OutT<AQMB_BF16>::store(a.y, at, v);
    else OutT<AQMB_F32>::store(a.y, at, v);
  }
}

template <int XT, int G, int R, int W>
static hipError_t by_batch(const W4Args& a, hipStream_t st) {
  constexpr bool kWide = XT == AQMB_F16 || XT == AQMB_BF16;
  const int blocks = ((a.d_out - 1) / kW4Rows + R) / R;
  if (a.batch <= (kWide ? 4 : 8)) w4_kernel<XT, G, R, W, 1><<<blocks, 64 * W, 0, st>>>(a);
  else if (!kWide || a.batch <= 8) w4_kernel<XT, G, R, W, 2><<<blocks, 64 * W, 0, st>>>(a);
  else if constexpr (kWide) w4_kernel<XT, G, R, W, 4><<<blocks, 64 * W, 0, st>>>(a);
  return hipGetLastError();
}
// Row tiles per workgroup: as many as give every compute unit one workgroup (or one a round, of at most
// 4 tiles), so that no round is partly filled and x is read once for all of them. 11008 x 4096 (688 row
// tiles, 256 units), groups of 64 with zero points, 11 rows: 1 tile 11.6 us, 2 tiles 9.9, 3 tiles 8.9, 4 tiles
// 10.7; 14336 x 4096 e4m3, 16 rows: 1 tile 14.0, 2 tiles 10.0, 4 tiles 9.7.
//
// Waves: 8, and 16 where registers allow and turns are long. One tile, 4096 x 11008 int8 at 16 rows: 7.3 us with
// 16, 7.9 with 8. Two tiles, 6000 x 9000, groups of 64, one row of bf16 8.9 and 9.6, 16 rows of e4m3 9.7 and 10.6, but of
// int8 6.6 and 6.3 at 4200 x 4096; groups of 32 spill. Three with 12, groups of 64, 14 rows of bf16: 13.3 and 14.0 at
// 11008 x 8000, but 10.4 and 9.4 at 11008 x 4099: left at 8. Where there are too few input tiles for them, more waves only
// cost their start.
template <int XT, int G>
static hipError_t go(const W4Args& a, int n_cu, hipStream_t st) {
  const int n_rt = (a.d_out - 1) / kW4Rows + 1, rounds = (n_rt - 1) / (4 * n_cu) + 1;
  switch ((n_rt - 1) / (n_cu * rounds) + 1) {
    case 1: return a.n_kt > 8 ? by_batch<XT, G, 1, 16>(a, st) : by_batch<XT, G, 1, 8>(a, st);
    case 2:
      if constexpr (XT != AQMB_I8 && G >= 64) {
        if (a.n_kt > 16) return by_batch<XT, G, 2, 16>(a, st);
      }
      return by_batch<XT, G, 2, 8>(a, st);
    case 3: return by_batch<XT, G, 3, 8>(a, st);
    default: return by_batch<XT, G, 4, 8>(a, st);
  }
}
template <int XT>
static hipError_t by_group(const W4Args& a, int g, int n_cu, hipStream_t st) {
  return g == 32 ? go<XT, 32>(a, n_cu, st) : g == 64 ? go<XT, 64>(a, n_cu, st) : go<XT, 128>(a, n_cu, st);
}

hipError_t launch_w4_gemv(const W4& L, const void* x, aqmb_dtype x_dtype, int64_t x_stride, const float* x_scales,
                          int x_scale_group, int batch, void* y, aqmb_dtype y_dtype, int64_t y_stride, hipStream_t st) {
  const int g = L.d.group_size;
  W4Args a = {(const u32x4_t*)L.tiles, L.scales, L.zeros, L.asymmetric ? (size_t)(kW4Rows * kW4Cols / g) : 0, x, x_scales, y, x_stride, y_stride,
              L.d.d_out, L.d.d_in, L.n_kt, batch, x_scale_group ? (L.d.d_in - 1) / g + 1 : 1, (int)y_dtype};
  switch (x_dtype) {
    case AQMB_F16: return by_group<AQMB_F16>(a, g, L.n_cu, st);
    case AQMB_BF16: return by_group<AQMB_BF16>(a, g, L.n_cu, st);
    case AQMB_F8: return by_group<AQMB_F8>(a, g, L.n_cu, st);
    default: return by_group<AQMB_I8>(a, g, L.n_cu, st);
  }
}

}  // namespace aqmb
