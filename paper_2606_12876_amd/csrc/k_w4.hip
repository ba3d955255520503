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

// Scales and zero points, one thread per (row tile, group, row).
__global__ void w4_pack_scales_kernel(const uint16_t* s, const uint8_t* z, uint16_t* so, uint8_t* zo, int d_out,
                                      int groups, int padded, size_t n) {
  const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n) return;
  const int row = (int)(i / 16 / padded) * kW4Rows + i % 16, g = (int)(i / 16 % padded);
  const bool in = row < d_out && g < groups;
  so[i] = in ? s[(size_t)row * groups + g] : 0;
  if (zo) zo[i] = in ? z[(size_t)row * groups + g] : 0;
}

hipError_t launch_w4_pack(const W4& L, const uint8_t* weights, const uint16_t* scales, const uint8_t* zeros,
                          hipStream_t st) {
  const int g = L.d.group_size, groups = (L.d.d_in + g - 1) / g, padded = L.n_kt * (kW4Cols / g);
  const size_t n = (size_t)L.n_rt * L.n_kt * 256, ns = (size_t)L.n_rt * padded * 16;
  w4_pack_kernel<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(weights, (uint32_t*)L.tiles, L.d.d_out, L.d.d_in, L.n_kt, n);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  w4_pack_scales_kernel<<<(unsigned)((ns + 255) / 256), 256, 0, st>>>(scales, zeros, L.scales, L.zeros, L.d.d_out,
                                                                     groups, padded, ns);
  return hipGetLastError();
}

// ------------------------------------------------------------------ product
struct W4Args {
  const uint4* tiles;
  const uint16_t* scales;
  const uint8_t* zeros;
  const void* x;
  const float* x_scales;
  void* y;
  int64_t x_stride, y_stride;
  int d_out, d_in, n_kt, batch, x_groups;   // x_groups: 0 for one scale per row, else scales per row
};

// How each type of x meets the nibbles.
template <int XT> struct Op;
template <> struct Op<AQMB_F16> {
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
template <> struct Op<AQMB_BF16> {
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
  static __device__ __forceinline__ C mul(V a, V b, C c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Op<AQMB_F8> : Op<AQMB_F16> {};
template <> struct Op<AQMB_I8> {
  typedef long V;
  typedef i32x4_t C;
  static __device__ __forceinline__ V weights(uint32_t w) {
    const uint32_t m = 0x0F0F0F0Fu;
    return (long)((uint64_t)((w >> 4) & m) << 32 | (w & m));
  }
  static __device__ __forceinline__ V ones() { return 0x0101010101010101l; }
  static __device__ __forceinline__ C mul(V a, V b, C c) { return __builtin_amdgcn_mfma_i32_16x16x32_i8(a, b, c, 0, 0, 0); }
};

struct __attribute__((packed, aligned(2))) X16 { uint32_t w[4]; };
struct __attribute__((packed, aligned(1))) X8 { uint32_t w[2]; };

// Four e4m3 values as fp16.
__device__ __forceinline__ uint2 widen_f8(uint32_t w) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return make_uint2(pack_f16x2(a.x, a.y), pack_f16x2(b.x, b.y));
}

// x[k .. k + 7] of one row as an operand, zeros from d_in on. x of 16 bits (and e4m3, widened) is used
// in its own order: the nibbles were laid out for it. The int8 masks leave bytes 0, 4, 1, 5 and 2, 6, 3, 7.
template <int XT>
__device__ __forceinline__ typename Op<XT>::V load_x(const void* row, int k, int d_in) {
  typedef typename Op<XT>::V V;
  if constexpr (XT == AQMB_F16 || XT == AQMB_BF16) {
    const uint16_t* p = (const uint16_t*)row + k;
    X16 r = {{0, 0, 0, 0}};
    if (k + 8 <= d_in) {
      r = *(const X16*)p;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (k + i < d_in) r.w[i / 2] |= (uint32_t)p[i] << (16 * (i % 2));
    }
    return __builtin_bit_cast(V, r);
  } else {
    const uint8_t* p = (const uint8_t*)row + k;
    X8 r = {{0, 0}};
    if (k + 8 <= d_in) {
      r = *(const X8*)p;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (k + i < d_in) r.w[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
    }
    if constexpr (XT == AQMB_F8) {
      const uint2 a = widen_f8(r.w[0]), b = widen_f8(r.w[1]);
      return __builtin_bit_cast(V, u32x4_t{a.x, a.y, b.x, b.y});
    } else {
      const uint32_t lo = __builtin_amdgcn_perm(r.w[1], r.w[0], 0x05010400u);
      const uint32_t hi = __builtin_amdgcn_perm(r.w[1], r.w[0], 0x07030602u);
      return (V)((uint64_t)hi << 32 | lo);
    }
  }
}

// A workgroup of W waves takes R tiles of 16 rows; wave w takes the input tiles w, w + W, ... and the
// waves' sums meet in LDS. G: the group size.
template <int XT, int YT, int G, int R, int W>
__global__ __launch_bounds__(64 * W) void w4_kernel(W4Args a) {
  typedef Op<XT> O;
  typedef typename O::C C;
  constexpr int kSteps = G / 32, kGroups = kW4Cols / G;
  __shared__ float part[W][R][16][17];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int n = lane % 16, q = lane / 16;
  const int col = n < a.batch ? n : a.batch - 1;     // the columns past the batch repeat its last row
  const char* xr = (const char*)a.x + (int64_t)col * a.x_stride * (XT == AQMB_F16 || XT == AQMB_BF16 ? 2 : 1);
  const float* xs = a.x_scales && a.x_groups ? a.x_scales + (int64_t)col * a.x_groups : nullptr;
  const int n_rt = (a.d_out + kW4Rows - 1) / kW4Rows;
  const int rt0 = blockIdx.x * R;
  const size_t tile_pitch = (size_t)a.n_kt * 64;

  float tot[R][4];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < 4; ++i) tot[r][i] = 0.f;

  for (int kt = wave; kt < a.n_kt; kt += W) {
    uint4 w[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int rt = rt0 + r < n_rt ? rt0 + r : n_rt - 1;
      w[r] = load_stream16(a.tiles + rt * tile_pitch + (size_t)kt * 64 + lane);
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      C acc[R], ax;
#pragma unroll
      for (int i = 0; i < 4; ++i) ax[i] = 0;
#pragma unroll
      for (int r = 0; r < R; ++r) acc[r] = ax;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int d = g * kSteps + s;
        const typename O::V x = load_x<XT>(xr, kt * kW4Cols + 32 * d + 8 * q, a.d_in);
        ax = O::mul(O::ones(), x, ax);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const uint32_t dw = d == 0 ? w[r].x : d == 1 ? w[r].y : d == 2 ? w[r].z : w[r].w;
          acc[r] = O::mul(O::weights(dw), x, acc[r]);
        }
      }
      // Groups from the last of d_in on have scale 0 and x 0; an x scale there does not exist.
      const int gi = kt * kGroups + g;
      const float sx = xs && gi < a.x_groups ? xs[gi] : 1.f;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int rt = rt0 + r < n_rt ? rt0 + r : n_rt - 1;
        const size_t at = ((size_t)rt * a.n_kt * kGroups + gi) * 16 + 4 * q;
        const uint2 sw = *(const uint2*)(a.scales + at);
        const uint32_t zw = a.zeros ? *(const uint32_t*)(a.zeros + at) : 0x08080808u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float s = f16_to_f32((i < 2 ? sw.x : sw.y) >> (16 * (i % 2)) & 0xFFFFu);
          if constexpr (XT == AQMB_I8) {
            const int z = (int)((zw >> (8 * i)) & 0xFFu);
            tot[r][i] += (s * sx) * (float)(acc[r][i] - z * ax[i]);
          } else {
            const float z = (float)((zw >> (8 * i)) & 0xFFu) + O::kZero;
            tot[r][i] += (s * sx) * (acc[r][i] - z * ax[i]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < 4; ++i) part[wave][r][4 * q + i][n] = tot[r][i];
  __syncthreads();
  for (int e = threadIdx.x; e < R * 256; e += 64 * W) {
    const int row = e % 16, b = e / 16 % 16, r = e / 256;
    const int out = (rt0 + r) * kW4Rows + row;
    if (b >= a.batch || out >= a.d_out) continue;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) v += part[k][r][row][b];
    if (a.x_scales && !a.x_groups) v *= a.x_scales[b];
    OutT<YT>::store(a.y, (size_t)b * a.y_stride + out, v);
  }
}

template <int XT, int YT, int G>
static hipError_t go(const W4Args& a, hipStream_t st) {
  const int n_rt = (a.d_out + kW4Rows - 1) / kW4Rows;
  w4_kernel<XT, YT, G, 1, 4><<<n_rt, 256, 0, st>>>(a);
  return hipGetLastError();
}
template <int XT, int YT>
static hipError_t by_group(const W4Args& a, int g, hipStream_t st) {
  return g == 32 ? go<XT, YT, 32>(a, st) : g == 64 ? go<XT, YT, 64>(a, st) : go<XT, YT, 128>(a, st);
}
template <int XT>
static hipError_t by_out(const W4Args& a, int g, aqmb_dtype yt, hipStream_t st) {
  return yt == AQMB_F16 ? by_group<XT, AQMB_F16>(a, g, st) : yt == AQMB_BF16 ? by_group<XT, AQMB_BF16>(a, g, st)
                                                                            : by_group<XT, AQMB_F32>(a, g, st);
}

hipError_t launch_w4_gemv(const W4& L, const void* x, aqmb_dtype x_dtype, int64_t x_stride, const float* x_scales,
                          int x_scale_group, int batch, void* y, aqmb_dtype y_dtype, int64_t y_stride, hipStream_t st) {
  const int g = L.d.group_size;
  W4Args a = {(const uint4*)L.tiles, L.scales, L.zeros, x, x_scales, y, x_stride, y_stride,
              L.d.d_out, L.d.d_in, L.n_kt, batch, x_scale_group ? (L.d.d_in + g - 1) / g : 0};
  switch (x_dtype) {
    case AQMB_F16: return by_out<AQMB_F16>(a, g, y_dtype, st);
    case AQMB_BF16: return by_out<AQMB_BF16>(a, g, y_dtype, st);
    case AQMB_F8: return by_out<AQMB_F8>(a, g, y_dtype, st);
    default: return by_out<AQMB_I8>(a, g, y_dtype, st);
  }
}

}  // namespace aqmb
