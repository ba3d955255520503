// Root-mean-square norm with the residual's addition and 16-bit, binary32 or 8-bit output.
//
//   h = x + r,  r' = round(h),  v = h * (1 / sqrt(mean(h^2) + eps)) * (w + w0)
//
// A row is read once and stays in registers: NT threads own 8 consecutive columns each, NV times
// over, so the sum of squares, the largest magnitude of a scale group (g / 8 neighbouring lanes) and
// the output need no second pass over memory. Bound by HBM for many rows (8192 x 4096 bf16 with a
// residual to e4m3: 43 us, 5.5 TB/s, more than a large copy's rate), by latency (load, two reductions,
// store) for few (one row of 4096: 1.9 us).
#include "device.h"
#include "ops.h"
#include "wave.h"

namespace aqmb {

// 8 consecutive 16-bit elements. Rows may start at any element: the 16-byte access needs no alignment
// beyond the element's on gfx950.
struct __attribute__((packed, aligned(2))) Raw8 { uint32_t w[4]; };
struct __attribute__((packed, aligned(2))) Raw4 { uint32_t w[2]; };
struct __attribute__((packed, aligned(2))) Raw2 { uint32_t w; };

// Columns c .. c + 7 of a row. What reaches over the row's end is its last 8 columns, for shift8 to put right:
// one load for every lane and no branch around it (element by element, with a wait for each, 4000 rows of 4095
// took 42 us, not 30). Those of its columns that belong to another thread, which may be storing to them in
// place, are among what is shifted out. kShort: rows may have fewer than 8 columns, 0 past the end.
template <bool kShort>
__device__ __forceinline__ Raw8 load8(const uint16_t* row, int c, int cols) {
  if (kShort && cols < 8) {
    Raw8 r = {{0, 0, 0, 0}};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) r.w[i / 2] |= (uint32_t)row[c + i] << (16 * (i % 2));
    return r;
  }
  return *(const Raw8*)(row + min(c, cols - 8));
}

// past elements to the left, 0 from the right.
__device__ __forceinline__ void shift8(Raw8& r, int past) {
  uint32_t a = r.w[0], b = r.w[1], c = r.w[2], d = r.w[3];
  const bool four = past & 4, two = past & 2;
  const uint32_t odd = 16 * (past & 1);
  a = four ? c : a, b = four ? d : b, c = four ? 0 : c, d = four ? 0 : d;
  a = two ? b : a, b = two ? c : b, c = two ? d : c, d = two ? 0 : d;
  a = __builtin_amdgcn_alignbit(b, a, odd);
  b = __builtin_amdgcn_alignbit(c, b, odd);
  c = __builtin_amdgcn_alignbit(d, c, odd);
  d >>= odd;
  const bool none = past >= 8;
  r = Raw8{{none ? 0 : a, none ? 0 : b, none ? 0 : c, none ? 0 : d}};
}

template <int DT>
__device__ __forceinline__ void widen8(const Raw8& r, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = DT == AQMB_F16 ? f16lo(r.w[i]) : bf16lo(r.w[i]);
    f[2 * i + 1] = DT == AQMB_F16 ? f16hi(r.w[i]) : bf16hi(r.w[i]);
  }
}

template <int DT>
__device__ __forceinline__ void store8_16(uint16_t* p, const float* f, int n) {
  Raw8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r.w[i] = DT == AQMB_F16 ? pack_f16x2(f[2 * i], f[2 * i + 1]) : pack_bf16x2(f[2 * i], f[2 * i + 1]);
  if (n >= 8) {
    *(Raw8*)p = r;
  } else if (n > 0) {
    if (n & 4) *(Raw4*)p = Raw4{{r.w[0], r.w[1]}}, p += 4, r.w[0] = r.w[2], r.w[1] = r.w[3];
    if (n & 2) *(Raw2*)p = Raw2{r.w[0]}, p += 2, r.w[0] = r.w[1];
    if (n & 1) *p = (uint16_t)r.w[0];
  }
}

struct __attribute__((packed, aligned(4))) F4 { float f[4]; };
struct __attribute__((packed, aligned(4))) F2 { float f[2]; };
struct __attribute__((packed, aligned(1))) B8 { uint32_t w[2]; };
struct __attribute__((packed, aligned(1))) B4 { uint32_t w; };
struct __attribute__((packed, aligned(1))) B2 { uint16_t w; };

template <int NT>
__device__ __forceinline__ float row_sum(float v, float* lds) {
  v = __builtin_bit_cast(float, over_lanes<(NT < 64 ? NT : 64)>(__builtin_bit_cast(uint32_t, v), add_floats));
  if constexpr (NT > 64) {
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) v += lds[i];
  }
  return v;
}

// Largest of the magnitudes as bits: above every finite value come infinity and then the NaNs, so one
// integer maximum also says whether a value is not finite.
template <int NT>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t* lds) {
  v = over_lanes<(NT < 64 ? NT : 64)>(v, max_bits);
  if constexpr (NT > 64) {
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) v = max(v, lds[i]);
  }
  return v;
}

// NT threads per row: up to 64, part of a wave or a wave (256 / NT rows per workgroup); else the workgroup.
template <int DT, int NT, int NV>
__global__ __launch_bounds__(NT <= 64 ? 256 : NT) void norm_kernel(NormArgs a) {
  __shared__ float lds_sum[16];
  __shared__ uint32_t lds_max[16];
  constexpr bool kShort = NT == 16;
  const int t = NT <= 64 ? threadIdx.x % NT : threadIdx.x;
  const int64_t row = NT <= 64 ? (int64_t)blockIdx.x * (256 / NT) + threadIdx.x / NT : blockIdx.x;
  if (NT <= 64 && row >= a.rows) return;      // all lanes of the row, and no barrier below for NT <= 64
  const uint16_t* x = (const uint16_t*)a.x + row * a.x_stride;
  const uint16_t* r = a.residual ? (const uint16_t*)a.residual + row * a.residual_stride : nullptr;

  // All loads first.
  float h[NV][8];
  Raw8 hx[NV], hr[NV], w[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) hx[i] = load8<kShort>(x, (i * NT + t) * 8, a.cols);
  if (r) {
#pragma unroll
    for (int i = 0; i < NV; ++i) hr[i] = load8<kShort>(r, (i * NT + t) * 8, a.cols);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) w[i] = load8<kShort>((const uint16_t*)a.weight, (i * NT + t) * 8, a.cols);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int past = (i * NT + t) * 8 - (a.cols - 8);
    if (past > 0 && !(kShort && a.cols < 8)) {
      shift8(hx[i], past);
      if (r) shift8(hr[i], past);
      shift8(w[i], past);
    }
    widen8<DT>(hx[i], h[i]);
    if (r) {
      float f[8];
      widen8<DT>(hr[i], f);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i][j] += f[j];
    }
  }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * NT + t) * 8;
    if (r) store8_16<DT>((uint16_t*)a.residual_out + row * a.residual_stride + c, h[i], a.cols - c);
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += h[i][j] * h[i][j];
  }
  ss = row_sum<NT>(ss, lds_sum);
  // Reciprocal and root by the instructions, an ulp each (rsqrtf takes care of subnormals): a launch of few rows
  // is bound by its waves' instructions, and the sum before them is off by more.
  const float inv = rsqrtf(ss * __builtin_amdgcn_rcpf((float)a.cols) + a.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float f[8];
    widen8<DT>(w[i], f);
#pragma unroll
    for (int j = 0; j < 8; ++j) h[i][j] = h[i][j] * inv * (f[j] + a.weight_offset);
    // Columns past the end hold h = 0; an infinite offset or inv would make them NaN.
    const int c = (i * NT + t) * 8;
    if (a.cols - c < 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j >= a.cols) h[i][j] = 0.f;
    }
  }

  if (a.y_dtype == AQMB_F16 || a.y_dtype == AQMB_BF16) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * NT + t) * 8;
      uint16_t* y = (uint16_t*)a.y + row * a.y_stride + c;
      if (a.y_dtype == AQMB_F16) store8_16<AQMB_F16>(y, h[i], a.cols - c);
      else store8_16<AQMB_BF16>(y, h[i], a.cols - c);
    }
    return;
  }
  if (a.y_dtype == AQMB_F32) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * NT + t) * 8, n = a.cols - c;
      float* y = (float*)a.y + row * a.y_stride + c;
      if (n >= 8) {
        ((F4*)y)[0] = F4{{h[i][0], h[i][1], h[i][2], h[i][3]}};
        ((F4*)y)[1] = F4{{h[i][4], h[i][5], h[i][6], h[i][7]}};
      } else if (n > 0) {
        f32x4_t f = {h[i][0], h[i][1], h[i][2], h[i][3]};
        if (n & 4) {
          *(F4*)y = F4{{f[0], f[1], f[2], f[3]}};
          y += 4;
          f = f32x4_t{h[i][4], h[i][5], h[i][6], 0.f};
        }
        if (n & 2) *(F2*)y = F2{{f[0], f[1]}};
        if (n & 1) y[n & 2] = n & 2 ? f[2] : f[0];
      }
    }
    return;
  }

  // 8 bits. The group's largest magnitude: g / 8 neighbouring lanes, or the whole row.
  const int g = a.scale_group;
  const float top = a.y_dtype == AQMB_F8 ? 448.f : 127.f;
  uint32_t m[NV];
  uint32_t all = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    m[i] = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m[i] = max(m[i], __builtin_bit_cast(uint32_t, h[i][j]) & 0x7FFFFFFFu);
    all = max(all, m[i]);
  }
  if (g == 0) {
    all = row_max<NT>(all, lds_max);
#pragma unroll
    for (int i = 0; i < NV; ++i) m[i] = all;
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      m[i] = over_lanes<4>(m[i], max_bits);
      if (g >= 64) m[i] = butterfly<4>(m[i], max_bits);
      if (g >= 128) m[i] = butterfly<8>(m[i], max_bits);
    }
  }
  const int shift = g == 0 ? 31 : g == 32 ? 5 : g == 64 ? 6 : 7;      // column -> group
  const int n_groups = ((a.cols - 1) >> shift) + 1;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * NT + t) * 8, n = a.cols - c;
    if (n <= 0) continue;
    const Scaling sc = scaling_of(m[i], top);
    const float mul = sc.mul;
    if ((c & ((1u << shift) - 1)) == 0) a.scales[row * n_groups + (c >> shift)] = sc.scale;
    B8 b;
    if (a.y_dtype == AQMB_F8) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        int w8 = __builtin_amdgcn_cvt_pk_fp8_f32(h[i][4 * k] * mul, h[i][4 * k + 1] * mul, 0, false);
        b.w[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(h[i][4 * k + 2] * mul, h[i][4 * k + 3] * mul, w8, true);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        // 1.5 2^23 + v rounds v to an integer, whose two's complement is the sum's low bits.
        uint32_t u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = __builtin_bit_cast(uint32_t, __builtin_fmaf(h[i][4 * k + j], mul, 12582912.f));
        b.w[k] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], 0x0C0C0400u),
                                       __builtin_amdgcn_perm(u[1], u[0], 0x0C0C0400u), 0x05040100u);
      }
    }
    if (!sc.finite) b.w[0] = b.w[1] = 0;
    uint8_t* y = (uint8_t*)a.y + row * a.y_stride + c;
    if (n >= 8) {
      *(B8*)y = b;
    } else {
      if (n & 4) *(B4*)y = B4{b.w[0]}, y += 4, b.w[0] = b.w[1];
      if (n & 2) *(B2*)y = B2{(uint16_t)b.w[0]}, y += 2, b.w[0] >>= 16;
      if (n & 1) *y = (uint8_t)b.w[0];
    }
  }
}

template <int DT, int NT, int NV>
static hipError_t go(const NormArgs& a, hipStream_t st) {
  const int blocks = NT <= 64 ? (a.rows - 1) / (256 / NT) + 1 : a.rows;
  norm_kernel<DT, NT, NV><<<blocks, NT <= 64 ? 256 : NT, 0, st>>>(a);
  return hipGetLastError();
}

// (Times below are of launches in a row, which is a little more than the kernel's own.)
// Threads for a row: one 8-column piece each as far as that goes (a launch of few rows is bound by its
// chain of loads, reductions and cold code: 4096 columns, 1 row: 512 threads x 1 piece 2.4 us, 256 x 2 2.5,
// 128 x 4 3.1, 1024 x 1 3.1; 8192 rows 46.0, 45.5, 47.3 and 50.6 us) and no more threads than pieces. 128
// columns, 65536 rows: 16 threads 15.6 us, 32 19.3. From 257 columns a wave's lanes are half idle and many rows
// gain by two pieces (512 columns, 16384 rows: 14.6 against 15.1 us; 64 rows: 2.7 against 2.5). Above 768
// pieces two cost few rows nothing (8192 columns, 1 row: 512 x 2 2.8 us, 1024 x 1 2.9; 4096 rows: 46.2, 48.4).
template <int DT>
static hipError_t choose(const NormArgs& a, hipStream_t st) {
  const int v = (a.cols + 7) / 8;
  if (v <= 16) return go<DT, 16, 1>(a, st);
  if (v <= 32) return go<DT, 32, 1>(a, st);
  if (v <= 64) return a.rows >= 4096 ? go<DT, 32, 2>(a, st) : go<DT, 64, 1>(a, st);
  if (v <= 128) return go<DT, 128, 1>(a, st);
  if (v <= 256) return go<DT, 256, 1>(a, st);
  if (v <= 384) return go<DT, 384, 1>(a, st);
  if (v <= 512) return go<DT, 512, 1>(a, st);
  if (v <= 768) return go<DT, 768, 1>(a, st);
  if (v <= 1024) return go<DT, 512, 2>(a, st);
  if (v <= 1536) return go<DT, 768, 2>(a, st);
  if (v <= 2048) return go<DT, 1024, 2>(a, st);
  return go<DT, 1024, 4>(a, st);
}

hipError_t launch_rms_norm(const NormArgs& a, aqmb_dtype dtype, hipStream_t st) {
  return dtype == AQMB_F16 ? choose<AQMB_F16>(a, st) : choose<AQMB_BF16>(a, st);
}

}  // namespace aqmb
