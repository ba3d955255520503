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
// so a dword of eight weights costs 3 (int8) or 8 vector instructions. sum x is a second product with a row
// of ones: it arrives in every lane that needs it, with the same grouping and order of sums.
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
  if (zo) zo[i] = in ? z[(size_t)row * groups + g] : 0;
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
  const void* x;
  const float* x_scales;
  void* y;
  int64_t x_stride, y_stride;
  int d_out, d_in, n_kt, batch;
  int x_groups;            // 0 for one scale per row, else scales per row
  int y_dtype;
};

// x[k .. k + 7] of a row: rows start at any element, which 8- and 16-byte loads allow on gfx950.
struct __attribute__((packed, aligned(2))) X16 { uint32_t w[4]; };
struct __attribute__((packed, aligned(1))) X8 { uint32_t w[2]; };

struct Load16 {
  typedef X16 X;
  static __device__ __forceinline__ X load(const void* row, int k) { return *(const X16*)((const uint16_t*)row + k); }
  // The same at the end of a row: zeros from d_in on.
  static __device__ __forceinline__ X load_end(const void* row, int k, int d_in) {
    if (k + 8 <= d_in) return load(row, k);
    X16 r = {{0, 0, 0, 0}};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (k + i < d_in) r.w[i / 2] |= (uint32_t)((const uint16_t*)row)[k + i] << (16 * (i % 2));
    return r;
  }
};
struct Load8 {
  typedef X8 X;
  static __device__ __forceinline__ X load(const void* row, int k) { return *(const X8*)((const uint8_t*)row + k); }
  static __device__ __forceinline__ X load_end(const void* row, int k, int d_in) {
    if (k + 8 <= d_in) return load(row, k);
    X8 r = {{0, 0}};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (k + i < d_in) r.w[i / 4] |= (uint32_t)((const uint8_t*)row)[k + i] << (8 * (i % 4));
    return r;
  }
};

// Four e4m3 values as fp16.
__device__ __forceinline__ uint2 widen_f8(uint32_t w) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return make_uint2(pack_f16x2(a.x, a.y), pack_f16x2(b.x, b.y));
}

// How each type of x meets the nibbles.
template <int XT> struct Op;
struct F16Form {
  typedef f16x8_t V;
  typedef f32x4_t C;
  static constexpr float kZero = 16.f;
  static __device__ __forceinline__ V weights(uint32_t w) {
    const uint32_t m = 0x03C003C0u, o = 0x4C004C00u;
    return __builtin_bit_cast(V, u32x4_t{((w << 6) & m) | o, ((w << 2) & m) | o, ((w >> 2) & m) | o, ((w >> 6) & m) | o});
  }
  static __device__ __forceinline__ V ones() {
    return __builtin_bit_cast(V, u32x4_t{0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u});
  }
  static __device__ __forceinline__ C mul(V a, V b, C c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Op<AQMB_BF16> : Load16 {
  typedef bf16x8_t V;
  typedef f32x4_t C;
  static constexpr float kZero = 16.f;
  static __device__ __forceinline__ V weights(uint32_t w) {
    const uint32_t m = 0x00780078u, o = 0x41804180u;
    return __builtin_bit_cast(V, u32x4_t{((w << 3) & m) | o, ((w >> 1) & m) | o, ((w >> 5) & m) | o, ((w >> 9) & m) | o});
  }
  static __device__ __forceinline__ V ones() {
    return __builtin_bit_cast(V, u32x4_t{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
  }
  static __device__ __forceinline__ V operand(X x) { return __builtin_bit_cast(V, x); }
  static __device__ __forceinline__ C mul(V a, V b, C c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Op<AQMB_F16> : F16Form, Load16 {
  static __device__ __forceinline__ V operand(X x) { return __builtin_bit_cast(V, x); }
};
template <> struct Op<AQMB_F8> : F16Form, Load8 {
  static __device__ __forceinline__ V operand(X x) {
    const uint2 a = widen_f8(x.w[0]), b = widen_f8(x.w[1]);
    return __builtin_bit_cast(V, u32x4_t{a.x, a.y, b.x, b.y});
  }
};
template <> struct Op<AQMB_I8> : Load8 {
  typedef long V;
  typedef i32x4_t C;
  static __device__ __forceinline__ V weights(uint32_t w) {
    const uint32_t m = 0x0F0F0F0Fu;
    return (long)((uint64_t)((w >> 4) & m) << 32 | (w & m));
  }
  static __device__ __forceinline__ V ones() { return 0x0101010101010101l; }
  // The masks leave weights 0, 4, 1, 5 and 2, 6, 3, 7; x has to follow.
  static __device__ __forceinline__ V operand(X x) {
    const uint32_t lo = __builtin_amdgcn_perm(x.w[1], x.w[0], 0x05010400u);
    const uint32_t hi = __builtin_amdgcn_perm(x.w[1], x.w[0], 0x07030602u);
    return (long)((uint64_t)hi << 32 | lo);
  }
  static __device__ __forceinline__ C mul(V a, V b, C c) { return __builtin_amdgcn_mfma_i32_16x16x32_i8(a, b, c, 0, 0, 0); }
};

// The scales (fp16) and zero points (uint8) that a lane needs of a tile: 4 rows of every group.
template <int N> struct Piece;
template <> struct Piece<4> { uint2 s; uint32_t z; };
template <> struct Piece<8> { u32x4_t s; uint2 z; };
template <> struct Piece<16> { u32x4_t s, s2; u32x4_t z; };

// A workgroup of W waves takes one tile of 16 rows; wave w takes the input tiles w, w + W, ... and the
// waves' sums meet in LDS. kAhead tiles (weights, scales and x) are under way at any time: a row tile
// is read by few waves, so the bytes in flight come from depth. G: the group size.
template <int XT, int G, int W>
__global__ __launch_bounds__(64 * W) void w4_kernel(W4Args a) {
  typedef Op<XT> O;
  typedef typename O::C C;
  constexpr bool kWide = XT == AQMB_F16 || XT == AQMB_BF16;
  constexpr int kSteps = G / 32, kGroups = kW4Cols / G, kAhead = W == 16 || G == 32 ? 2 : 4;
  __shared__ float part[W][16][17];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int n = lane % 16, q = lane / 16;
  const int col = n < a.batch ? n : a.batch - 1;     // the columns past the batch repeat its last row
  const char* xr = (const char*)a.x + (int64_t)col * a.x_stride * (kWide ? 2 : 1);
  const float* xs = a.x_scales && a.x_groups ? a.x_scales + (int64_t)col * a.x_groups : nullptr;
  const size_t tile0 = (size_t)blockIdx.x * a.n_kt;

  u32x4_t w[kAhead];
  typename O::X x[kAhead][4];
  Piece<4 * kGroups> sz[kAhead];
  float sx[kAhead][kGroups];
  auto fetch = [&](int u, int kt) {
    const size_t tile = tile0 + kt;
    w[u] = __builtin_nontemporal_load((const u32x4_t*)a.tiles + tile * 64 + lane);
    const size_t at = tile * (16 * kGroups) + 4 * kGroups * q;
    if constexpr (kGroups == 1) {
      sz[u].s = *(const uint2*)(a.scales + at);
      sz[u].z = a.zeros ? *(const uint32_t*)(a.zeros + at) : 0x08080808u;
    } else if constexpr (kGroups == 2) {
      sz[u].s = *(const u32x4_t*)(a.scales + at);
      sz[u].z = a.zeros ? *(const uint2*)(a.zeros + at) : make_uint2(0x08080808u, 0x08080808u);
    } else {
      sz[u].s = *(const u32x4_t*)(a.scales + at);
      sz[u].s2 = *(const u32x4_t*)(a.scales + at + 8);
      sz[u].z = a.zeros ? *(const u32x4_t*)(a.zeros + at) : u32x4_t{0x08080808u, 0x08080808u, 0x08080808u, 0x08080808u};
    }
    const int k = kt * kW4Cols + 8 * q;
    if (kt * kW4Cols + kW4Cols <= a.d_in) {
#pragma unroll
      for (int d = 0; d < 4; ++d) x[u][d] = O::load(xr, k + 32 * d);
    } else {
#pragma unroll
      for (int d = 0; d < 4; ++d) x[u][d] = O::load_end(xr, k + 32 * d, a.d_in);
    }
    // Groups from the last of d_in on have scale 0 and x 0; an x scale there does not exist.
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      sx[u][g] = 1.f;
      if constexpr (!kWide)
        if (xs) sx[u][g] = xs[min(kt * kGroups + g, a.x_groups - 1)];
    }
  };

  float tot[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
    if (wave + u * W < a.n_kt) fetch(u, wave + u * W);
  for (int kt0 = wave; kt0 < a.n_kt; kt0 += kAhead * W) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int kt = kt0 + u * W;
      if (kt >= a.n_kt) break;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        C acc, ax;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = ax[i] = 0;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const typename O::V v = O::operand(x[u][g * kSteps + s]);
          ax = O::mul(O::ones(), v, ax);
          acc = O::mul(O::weights(w[u][g * kSteps + s]), v, acc);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = 4 * g + i;                     // of the lane's piece
          uint32_t sw, zw;
          if constexpr (kGroups == 1) {
            sw = e < 2 ? sz[u].s.x : sz[u].s.y;
            zw = sz[u].z;
          } else if constexpr (kGroups == 2) {
            sw = sz[u].s[e / 2];
            zw = e < 4 ? sz[u].z.x : sz[u].z.y;
          } else {
            sw = e < 8 ? sz[u].s[e / 2] : sz[u].s2[e / 2 - 4];
            zw = sz[u].z[e / 4];
          }
          float s = e % 2 ? f16hi(sw) : f16lo(sw);
          if constexpr (!kWide) s *= sx[u][g];
          const int z = (int)((zw >> (8 * i)) & 0xFFu);
          if constexpr (XT == AQMB_I8) tot[i] += s * (float)(acc[i] - z * ax[i]);
          else tot[i] += s * (acc[i] - ((float)z + O::kZero) * ax[i]);
        }
      }
      if (kt + kAhead * W < a.n_kt) fetch(u, kt + kAhead * W);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) part[wave][4 * q + i][n] = tot[i];
  __syncthreads();
  for (int e = threadIdx.x; e < 256; e += 64 * W) {
    const int row = e % 16, b = e / 16, out = blockIdx.x * kW4Rows + row;
    if (b >= a.batch || out >= a.d_out) continue;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) v += part[k][row][b];
    if (a.x_scales && !a.x_groups) v *= a.x_scales[b];
    const size_t at = (size_t)b * a.y_stride + out;
    if (a.y_dtype == AQMB_F16) OutT<AQMB_F16>::store(a.y, at, v);
    else if (a.y_dtype == AQMB_BF16) OutT<AQMB_BF16>::store(a.y, at, v);
    else OutT<AQMB_F32>::store(a.y, at, v);
  }
}

template <int XT, int G>
static hipError_t go(const W4Args& a, int n_cu, hipStream_t st) {
  const int n_rt = (a.d_out - 1) / kW4Rows + 1;
  // Waves per row tile: enough for 16 waves on every compute unit, never more than input tiles.
  const int want = (16 * n_cu + n_rt - 1) / n_rt;
  if (want > 8 && a.n_kt > 8) w4_kernel<XT, G, 16><<<n_rt, 1024, 0, st>>>(a);
  else if (want > 4 && a.n_kt > 4) w4_kernel<XT, G, 8><<<n_rt, 512, 0, st>>>(a);
  else w4_kernel<XT, G, 4><<<n_rt, 256, 0, st>>>(a);
  return hipGetLastError();
}
template <int XT>
static hipError_t by_group(const W4Args& a, int g, int n_cu, hipStream_t st) {
  return g == 32 ? go<XT, 32>(a, n_cu, st) : g == 64 ? go<XT, 64>(a, n_cu, st) : go<XT, 128>(a, n_cu, st);
}

hipError_t launch_w4_gemv(const W4& L, const void* x, aqmb_dtype x_dtype, int64_t x_stride, const float* x_scales,
                          int x_scale_group, int batch, void* y, aqmb_dtype y_dtype, int64_t y_stride, hipStream_t st) {
  const int g = L.d.group_size;
  W4Args a = {(const u32x4_t*)L.tiles, L.scales, L.zeros, x, x_scales, y, x_stride, y_stride,
              L.d.d_out, L.d.d_in, L.n_kt, batch, x_scale_group ? (L.d.d_in - 1) / g + 1 : 0, (int)y_dtype};
  switch (x_dtype) {
    case AQMB_F16: return by_group<AQMB_F16>(a, g, L.n_cu, st);
    case AQMB_BF16: return by_group<AQMB_BF16>(a, g, L.n_cu, st);
    case AQMB_F8: return by_group<AQMB_F8>(a, g, L.n_cu, st);
    default: return by_group<AQMB_I8>(a, g, L.n_cu, st);
  }
}

}  // namespace aqmb
