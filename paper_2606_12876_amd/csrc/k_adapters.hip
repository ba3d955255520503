// Low-rank adapters of many requests beside one projection, out_i = base_i + s_n B_n (A_n x_i), n = index_i.
//
// Two launches: t = A_n x (binary32, partial sums over parts of the inputs side by side in the workspace), then
// out = base + B_n (s_n t). Both take 64 neighbouring rows at a time and sort them by adapter with wave-wide votes: a
// tile is up to 16 of them that share an adapter, the columns of one matrix instruction, with 16 rows of A or B as
// its rows. So each row meets only its own adapter, in any order of the indexes, without atomics, and what
// an adapter weighs is read once per tile. Few rows are bound by the adapters' bytes and two launches' latency, many by x, base
// and out.
#include "device.h"
#include "ops.h"

namespace aqmb {

namespace {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
struct __attribute__((packed, aligned(2))) Raw8 { uint32_t w[4]; };
struct __attribute__((packed, aligned(4))) F4 { float f[4]; };

constexpr int kRows = 64;      // rows that a wave sorts by adapter

// Values k .. k + 7 of a row of n, 0 from n on. Rows may start at any element.
__device__ __forceinline__ u32x4_t load8(const uint16_t* row, int k) {
  const Raw8 r = *(const Raw8*)(row + k);
  return u32x4_t{r.w[0], r.w[1], r.w[2], r.w[3]};
}
__device__ __forceinline__ u32x4_t load8(const uint16_t* row, int k, int n) {
  if (k + 8 <= n) return load8(row, k);
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (k + j < n) w[j / 2] |= (uint32_t)row[k + j] << (16 * (j % 2));
  return u32x4_t{w[0], w[1], w[2], w[3]};
}

template <int DT>
__device__ __forceinline__ f32x4_t mma(u32x4_t a, u32x4_t b, f32x4_t c) {
  if constexpr (DT == AQMB_F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// Up to 16 of the 64 rows from row0 on that share an adapter (-1: none).
struct Tile {
  bool found;
  int adapter, count;
  int row;             // of slot lane % 16; slots past count repeat the first
};

// Tile number `want` of these rows, in the order of their adapters' first rows. All lanes of the wave take part.
__device__ __forceinline__ Tile find_tile(const AdapterArgs& a, int row0, int want) {
  const int lane = threadIdx.x % 64, r = row0 + lane;
  const bool in = r < a.n_rows;
  int n = in ? a.index[r] : -1;
  if ((unsigned)n >= (unsigned)a.ad.n_adapters) n = -1;
  uint64_t todo = __ballot(in);
  Tile t = {false, -1, 0, row0};
  int seen = 0;
  while (todo) {
    const int leader = __builtin_ctzll(todo), own = __builtin_amdgcn_readlane(n, leader);
    const uint64_t mask = __ballot(in && n == own);
    todo &= ~mask;
    const int tiles = (__builtin_popcountll(mask) + 15) / 16;
    if (want < seen + tiles) {
      const int first = (want - seen) * 16;
      const int at = __builtin_popcountll(mask & ((1ull << lane) - 1)) - first;
      const bool mine = (mask >> lane & 1) && at >= 0 && at < 16;
      t.found = true;
      t.adapter = own;
      t.count = min(__builtin_popcountll(mask) - first, 16);
      // Each row's lane sends its number to its slot (the others to a lane that no one asks), then all read theirs.
      const int sent = __builtin_amdgcn_ds_permute((mine ? at : 63) * 4, r);
      const int slot = lane % 16;
      t.row = __builtin_amdgcn_ds_bpermute((slot < t.count ? slot : 0) * 4, sent);
      return t;
    }
    seen += tiles;
  }
  return t;
}

__device__ __forceinline__ int own_rank(const AdapterArgs& a, int adapter) {
  return a.ad.ranks ? min(max(a.ad.ranks[adapter], 0), a.ad.rank) : a.ad.rank;
}

// acc[m] += rows 16 m .. of A times the tile's rows of x, over inputs k0 .. k1 - 1 (k0 a multiple of 32).
template <int DT, int RT>
__device__ __forceinline__ void shrink(const AdapterArgs& a, const Tile& t, int rank, int k0, int k1, f32x4_t* acc) {
  const int lane = threadIdx.x % 64, i = lane % 16, kg = lane / 16 * 8, d_in = a.ad.d_in;
  const uint16_t* x = (const uint16_t*)a.x + t.row * a.x_stride;
  const uint16_t* w = (const uint16_t*)a.ad.a + (int64_t)t.adapter * a.ad.rank * d_in;
  const uint16_t* row[RT];
#pragma unroll
  for (int m = 0; m < RT; ++m) row[m] = w + (int64_t)min(16 * m + i, rank - 1) * d_in;
  const int whole = min(k1, d_in / 32 * 32);
  int k = k0;
#pragma unroll 4
  for (; k < whole; k += 32) {
    const u32x4_t xv = load8(x, k + kg);
#pragma unroll
    for (int m = 0; m < RT; ++m)
      if (16 * m < rank) acc[m] = mma<DT>(load8(row[m], k + kg), xv, acc[m]);
  }
  if (k < k1) {                       // the last inputs, fewer than 32
    const u32x4_t xv = load8(x, k + kg, d_in);
#pragma unroll
    for (int m = 0; m < RT; ++m)
      if (16 * m < rank) acc[m] = mma<DT>(load8(row[m], k + kg, d_in), xv, acc[m]);
  }
}

// kFew: one tile per workgroup, its waves side by side along the inputs; else a wave per tile.
template <int DT, int RT, bool kFew>
__global__ __launch_bounds__(256) void shrink_kernel(AdapterArgs a) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, steps = (a.ad.d_in + 31) / 32;
  const int64_t pitch = (int64_t)a.n_rows * a.t_stride;
  if constexpr (kFew) {
    __shared__ __align__(16) float lds[2][4][256];
    const Tile t = find_tile(a, 0, blockIdx.x);
    if (!t.found || t.adapter < 0) return;               // the whole workgroup
    const int rank = own_rank(a, t.adapter);
    if (rank == 0) return;
    const int parts = 4 * a.splits, part = blockIdx.y * 4 + wave;
    f32x4_t acc[RT] = {};
    shrink<DT, RT>(a, t, rank, (int)((int64_t)steps * part / parts) * 32,
                   min((int)((int64_t)steps * (part + 1) / parts) * 32, a.ad.d_in), acc);
#pragma unroll
    for (int m = 0; m < RT; ++m) {
      if (16 * m >= rank) break;                         // the whole workgroup
      *(f32x4_t*)&lds[m % 2][wave][lane * 4] = acc[m];
      __syncthreads();
      if (wave == m % 4 && lane % 16 < t.count) {
        f32x4_t s = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < 4; ++w) s += *(const f32x4_t*)&lds[m % 2][w][lane * 4];
        *(f32x4_t*)(a.t + blockIdx.y * pitch + (int64_t)t.row * a.t_stride + 16 * m + lane / 16 * 4) = s;
      }
    }
  } else {
    for (int want = wave;; want += 4) {
      const Tile t = find_tile(a, blockIdx.x * kRows, want);
      if (!t.found) return;
      if (t.adapter < 0) continue;
      const int rank = own_rank(a, t.adapter);
      if (rank == 0) continue;
      f32x4_t acc[RT] = {};
      shrink<DT, RT>(a, t, rank, (int)((int64_t)steps * blockIdx.y / a.splits) * 32,
                     min((int)((int64_t)steps * (blockIdx.y + 1) / a.splits) * 32, a.ad.d_in), acc);
      if (lane % 16 < t.count) {
#pragma unroll
        for (int m = 0; m < RT; ++m)
          if (16 * m < rank)
            *(f32x4_t*)(a.t + blockIdx.y * pitch + (int64_t)t.row * a.t_stride + 16 * m + lane / 16 * 4) = acc[m];
      }
    }
  }
}

// Eight binary32 values as 16-bit parts that add up to them: three for bf16 (exactly, short of subnormals), two for
// fp16 (22 bits of the largest; the caller brings them into fp16's range).
template <int DT> struct Parts;
template <> struct Parts<AQMB_BF16> {
  static constexpr int kN = 3;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16x2(lo, hi); }
  static __device__ __forceinline__ float lo(uint32_t w) { return bf16lo(w); }
  static __device__ __forceinline__ float hi(uint32_t w) { return bf16hi(w); }
};
template <> struct Parts<AQMB_F16> {
  static constexpr int kN = 2;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_f16x2(lo, hi); }
  static __device__ __forceinline__ float lo(uint32_t w) { return f16lo(w); }
  static __device__ __forceinline__ float hi(uint32_t w) { return f16hi(w); }
};
template <int DT>
__device__ __forceinline__ void split(float* f, u32x4_t* out) {
  typedef Parts<DT> P;
#pragma unroll
  for (int p = 0; p < P::kN; ++p)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = P::pack(f[2 * j], f[2 * j + 1]);
      out[p][j] = w;
      f[2 * j] -= P::lo(w);
      f[2 * j + 1] -= P::hi(w);
    }
}

// 16 neighbouring values of a row of outputs, from element o on.
template <int YT>
__device__ __forceinline__ void load16(const void* row, int o, int n, float* f) {
  if constexpr (YT == AQMB_F32) {
    const float* p = (const float*)row + o;
    if (o + 16 <= n) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const F4 v = *(const F4*)(p + 4 * j);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[4 * j + e] = v.f[e];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) f[j] = o + j < n ? p[j] : 0.f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const u32x4_t v = load8((const uint16_t*)row, o + 8 * j, n);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[8 * j + 2 * e] = YT == AQMB_F16 ? f16lo(v[e]) : bf16lo(v[e]);
        f[8 * j + 2 * e + 1] = YT == AQMB_F16 ? f16hi(v[e]) : bf16hi(v[e]);
      }
    }
  }
}
template <int YT>
__device__ __forceinline__ void store16(void* row, int o, int n, const float* f) {
  if constexpr (YT == AQMB_F32) {
    float* p = (float*)row + o;
    if (o + 16 <= n) {
#pragma unroll
      for (int j = 0; j < 4; ++j) *(F4*)(p + 4 * j) = F4{{f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]}};
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (o + j < n) p[j] = f[j];
    }
  } else {
    uint16_t* p = (uint16_t*)row + o;
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = YT == AQMB_F16 ? pack_f16x2(f[2 * j], f[2 * j + 1]) : pack_bf16x2(f[2 * j], f[2 * j + 1]);
    if (o + 16 <= n) {
      *(Raw8*)p = Raw8{{w[0], w[1], w[2], w[3]}};
      *(Raw8*)(p + 8) = Raw8{{w[4], w[5], w[6], w[7]}};
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (o + j < n) p[j] = (uint16_t)(w[j / 2] >> (16 * (j % 2)));
    }
  }
}

// Outputs o0 .. o1 - 1 (o0 a multiple of 64) of the tile's rows.
template <int DT, int YT, int KT>
__device__ __forceinline__ void expand(const AdapterArgs& a, const Tile& t, int o0, int o1) {
  constexpr int kParts = Parts<DT>::kN, kSize = YT == AQMB_F32 ? 4 : 2;
  const int lane = threadIdx.x % 64, i = lane % 16, q = lane / 16, d_out = a.ad.d_out;
  const bool on = i < t.count;
  const char* base = (const char*)a.base + t.row * a.base_stride * kSize;
  char* out = (char*)a.out + t.row * a.out_stride * kSize;
  const int rank = t.adapter < 0 ? 0 : own_rank(a, t.adapter);
  if (rank == 0) {
    if (a.base == a.out || !on) return;
    for (int o = o0 + 16 * q; o < o1; o += 64) {
      float f[16];
      load16<YT>(base, o, d_out, f);
      store16<YT>(out, o, d_out, f);
    }
    return;
  }

  // The row's t: partial sums added up, scaled, 0 from the adapter's rank on.
  float v[KT][8];
  const float s = a.ad.scales ? a.ad.scales[t.adapter] : 1.f;
  const float* tp = a.t + (int64_t)t.row * a.t_stride + 8 * q;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[kt][j] = 0.f;
    if (32 * kt + 8 * q < rank) {
      for (int p = 0; p < a.splits; ++p) {
        const f32x4_t* w = (const f32x4_t*)(tp + p * (int64_t)a.n_rows * a.t_stride + 32 * kt);
        const f32x4_t lo = w[0], hi = w[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[kt][j] += lo[j], v[kt][4 + j] += hi[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[kt][j] = 32 * kt + 8 * q + j < rank ? v[kt][j] * s : 0.f;
    }
  }
  float back = 1.f;
  if constexpr (DT == AQMB_F16) {
    // By a power of two, so that the row's largest magnitude is in [2^13, 2^14): in fp16's range, the parts far
    // from its subnormals.
    uint32_t big = 0;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int j = 0; j < 8; ++j) big = max(big, __builtin_bit_cast(uint32_t, v[kt][j]) & 0x7FFFFFFFu);
    big = max(big, (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (lane ^ 16), (int)big));
    big = max(big, (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (lane ^ 32), (int)big));
    const int ex = min(max((int)(big >> 23), 14), 254);    // the exponent that goes to 13
    const float fwd = __builtin_bit_cast(float, (uint32_t)(267 - ex) << 23);
    back = __builtin_bit_cast(float, (uint32_t)(ex - 13) << 23);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[kt][j] *= fwd;
  }
  u32x4_t tv[KT][kParts];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) split<DT>(v[kt], tv[kt]);

  // Row i of matrix tile m is output 16 (i / 4) + 4 m + i % 4 of 64: so a lane's results are 16 neighbours.
  const uint16_t* b = (const uint16_t*)a.ad.b + (int64_t)t.adapter * d_out * a.ad.rank;
  for (int o = o0; o < o1; o += 64) {
    float f[16];
    if (on) load16<YT>(base, o + 16 * q, d_out, f);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const uint16_t* w = b + (int64_t)min(o + i / 4 * 16 + 4 * m + i % 4, d_out - 1) * a.ad.rank;
      f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
        if (32 * kt < rank) {
          const u32x4_t wv = load8(w, 32 * kt + 8 * q, rank);
#pragma unroll
          for (int p = kParts - 1; p >= 0; --p) acc = mma<DT>(wv, tv[kt][p], acc);
        }
#pragma unroll
      for (int j = 0; j < 4; ++j) f[4 * m + j] = DT == AQMB_F16 ? fmaf(acc[j], back, f[4 * m + j]) : f[4 * m + j] + acc[j];
    }
    if (on) store16<YT>(out, o + 16 * q, d_out, f);
  }
}

// kFew: blockIdx.y tile; else blockIdx.y 64 rows, a wave per tile.
template <int DT, int YT, int KT, bool kFew>
__global__ __launch_bounds__(256) void expand_kernel(AdapterArgs a) {
  const int wave = threadIdx.x / 64;
  if constexpr (kFew) {
    const Tile t = find_tile(a, 0, blockIdx.y);
    const int o0 = (blockIdx.x * 4 + wave) * a.per_wave;
    if (t.found && o0 < a.ad.d_out) expand<DT, YT, KT>(a, t, o0, min(o0 + a.per_wave, a.ad.d_out));
  } else {
    const int o0 = blockIdx.x * a.per_wave;
    for (int want = wave;; want += 4) {
      const Tile t = find_tile(a, blockIdx.y * kRows, want);
      if (!t.found) return;
      expand<DT, YT, KT>(a, t, o0, min(o0 + a.per_wave, a.ad.d_out));
    }
  }
}

template <int DT, int RT>
hipError_t go_shrink(const AdapterArgs& a, const AdapterPlan& p, hipStream_t st) {
  if (p.few) shrink_kernel<DT, RT, true><<<dim3(p.tiles, p.splits), 256, 0, st>>>(a);
  else shrink_kernel<DT, RT, false><<<dim3((a.n_rows + kRows - 1) / kRows, p.splits), 256, 0, st>>>(a);
  return hipGetLastError();
}
template <int DT, int YT, int KT>
hipError_t go_expand(const AdapterArgs& a, const AdapterPlan& p, hipStream_t st) {
  const unsigned parts = (a.ad.d_out + a.per_wave - 1) / a.per_wave;
  if (p.few) expand_kernel<DT, YT, KT, true><<<dim3((parts + 3) / 4, p.tiles), 256, 0, st>>>(a);
  else expand_kernel<DT, YT, KT, false><<<dim3(parts, (a.n_rows + kRows - 1) / kRows), 256, 0, st>>>(a);
  return hipGetLastError();
}
template <int DT, int YT>
hipError_t by_rank(const AdapterArgs& a, const AdapterPlan& p, hipStream_t st) {
  const int r = a.ad.rank;
  return r <= 32 ? go_expand<DT, YT, 1>(a, p, st) : r <= 64 ? go_expand<DT, YT, 2>(a, p, st)
         : r <= 128 ? go_expand<DT, YT, 4>(a, p, st) : go_expand<DT, YT, 8>(a, p, st);
}
template <int DT>
hipError_t both(const AdapterArgs& a, const AdapterPlan& p, aqmb_dtype y, hipStream_t st) {
  const int r = a.ad.rank;
  const hipError_t e = r <= 16 ? go_shrink<DT, 1>(a, p, st) : r <= 32 ? go_shrink<DT, 2>(a, p, st)
                       : r <= 64 ? go_shrink<DT, 4>(a, p, st) : r <= 128 ? go_shrink<DT, 8>(a, p, st) : go_shrink<DT, 16>(a, p, st);
  if (e != hipSuccess) return e;
  return y == AQMB_F16 ? by_rank<DT, AQMB_F16>(a, p, st) : y == AQMB_BF16 ? by_rank<DT, AQMB_BF16>(a, p, st)
                                                                          : by_rank<DT, AQMB_F32>(a, p, st);
}

}  // namespace

AdapterPlan adapter_plan(const aqmb_adapters& ad, int n_rows) {
  AdapterPlan p;
  const int steps = (ad.d_in + 31) / 32;
  p.few = n_rows <= kRows;
  const int groups = n_rows < ad.n_adapters + 1 ? n_rows : ad.n_adapters + 1;
  p.tiles = groups + 3 < n_rows ? groups + 3 : n_rows;
  if (p.few) {
    p.splits = steps / 16;
    if (p.splits > 8) p.splits = 8;
    p.per_wave = 64;
  } else {
    const int blocks = (n_rows + kRows - 1) / kRows;
    p.splits = 512 / blocks;
    if (p.splits > steps / 8) p.splits = steps / 8;
    if (p.splits > 8) p.splits = 8;
    p.per_wave = 256;
  }
  if (p.splits < 1) p.splits = 1;
  p.t_stride = (ad.rank + 15) / 16 * 16;
  p.bytes = (size_t)p.splits * n_rows * p.t_stride * 4;
  return p;
}

hipError_t launch_adapters(AdapterArgs a, const AdapterPlan& p, aqmb_dtype y, hipStream_t st) {
  a.t_stride = p.t_stride;
  a.splits = p.splits;
  a.per_wave = p.per_wave;
  return a.ad.dtype == AQMB_F16 ? both<AQMB_F16>(a, p, y, st) : both<AQMB_BF16>(a, p, y, st);
}

}  // namespace aqmb
