// Low-rank adapters of many requests beside one projection, out_i = base_i + s_n B_n (A_n x_i), n = index_i.
//
// Two launches: t = A_n x (binary32, partial sums over parts of the inputs side by side in the workspace), then
// out = base + B_n (s_n t). Rows that share an adapter are the columns of matrix instructions, 16 each, with 16 rows of A
// or outputs of B: each row meets only its own adapter, in any order of the indexes, without atomics on results. Few rows:
// every wave finds its 16 by votes over 64 rows' indexes; the adapters' bytes and the latency of two launches bound them
// (one row, rank 16, 4096 x 4096: 3.5 + 4.9 us). Many: a first launch sorts the rows by adapter into tiles of 64; bound by x, base,
// out and t, which all eight L2s read, since neighbouring workgroups take other outputs of the same rows (8192 rows, 4096 x
// 4096, rank 32: sort 10 us, t 14.3 us, 4.7 TB/s, the outputs 34 us, 165 MB at 4.9 TB/s, 28 of them t; rank 128: 9.9, 31
// and 83 us, the last 263 MB at 3.2 TB/s, 118 of them t).
#include "device.h"
#include "ops.h"

namespace aqmb {

namespace {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
struct __attribute__((packed, aligned(2))) Raw8 { uint32_t w[4]; };
struct __attribute__((packed, aligned(4))) F4 { float f[4]; };

__device__ __forceinline__ void lds_order() {      // a wave's LDS accesses run in order; the compiler's do now too
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

constexpr int kRows = 64;      // rows that a wave looks at
constexpr int kFewWaves = 8;   // of a workgroup that sums over the inputs for one tile
constexpr int kMaxSplits = 4;
constexpr int kMaxAdapters = AQMB_MAX_ADAPTERS;     // the sort's bins

// Values k .. k + 7 of a row of n, 0 from n on. Rows may start at any element.
__device__ __forceinline__ u32x4_t load8(const uint16_t* row, uint32_t k) {
  const Raw8 r = *(const Raw8*)(row + k);
  return u32x4_t{r.w[0], r.w[1], r.w[2], r.w[3]};
}
__device__ __forceinline__ u32x4_t load8(const uint16_t* row, int k, int n) {
  if (k + 8 <= n) return load8(row, k);
  if (k >= n) return u32x4_t{0, 0, 0, 0};
  uint64_t lo = 0, hi = 0;
  if (n >= 8) {                   // the row's last 8 values, moved down by those before k
    const u32x4_t v = load8(row, n - 8);
    lo = (uint64_t)v.y << 32 | v.x, hi = (uint64_t)v.w << 32 | v.z;
    const int past = k - (n - 8);
    if (past >= 4) lo = hi, hi = 0;
    const int s = 16 * (past % 4);
    if (s) lo = lo >> s | hi << (64 - s), hi >>= s;
  } else {
    for (int j = 0; k + j < n; ++j)
      if (j < 4) lo |= (uint64_t)row[k + j] << (16 * j);
      else hi |= (uint64_t)row[k + j] << (16 * (j - 4));
  }
  return u32x4_t{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// The same in two steps without a branch, n >= 8: a row's last 8 values, and these moved down by those before k. Many loads
// first, then the moves: each in one piece would wait for its own.
__device__ __forceinline__ u32x4_t load8_last(const uint16_t* row, int k, int n) { return load8(row, min(k, n - 8)); }
__device__ __forceinline__ u32x4_t moved8(u32x4_t v, int k, int n) {
  const int past = max(k - (n - 8), 0);
  uint32_t a = v.x, b = v.y, c = v.z, d = v.w;
  const bool four = past & 4, two = past & 2;
  const uint32_t odd = 16 * (past & 1);
  a = four ? c : a, b = four ? d : b, c = four ? 0 : c, d = four ? 0 : d;
  a = two ? b : a, b = two ? c : b, c = two ? d : c, d = two ? 0 : d;
  a = __builtin_amdgcn_alignbit(b, a, odd), b = __builtin_amdgcn_alignbit(c, b, odd), c = __builtin_amdgcn_alignbit(d, c, odd);
  d >>= odd;
  const bool none = past >= 8;
  return u32x4_t{none ? 0 : a, none ? 0 : b, none ? 0 : c, none ? 0 : d};
}

// Eight values from p on, loaded and then put together. A 16-byte load that does not start at a multiple of 4 bytes takes
// several times as long, so where such addresses come (kOdd) it starts 2 bytes lower, inside the same aligned 4 bytes as *p
// (of a tensor's first row these are the two bytes before the tensor; they are shifted out), and the last value has a load of its own.
template <bool kOdd> struct Loaded8 {
  u32x4_t v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = load8(p, 0u); }
  __device__ __forceinline__ u32x4_t value(const uint16_t*) const { return v; }
};
template <> struct Loaded8<true> {
  u32x4_t v;
  uint32_t last;
  __device__ __forceinline__ void load(const uint16_t* p) {
    v = load8((const uint16_t*)((uintptr_t)p & ~(uintptr_t)2), 0u);
    last = p[7];
  }
  __device__ __forceinline__ u32x4_t value(const uint16_t* p) const {
    const uint32_t s = ((uintptr_t)p & 2) * 8;
    return u32x4_t{__builtin_amdgcn_alignbit(v.y, v.x, s), __builtin_amdgcn_alignbit(v.z, v.y, s),
                   __builtin_amdgcn_alignbit(v.w, v.z, s), __builtin_amdgcn_alignbit(last, v.w, s)};
  }
};

template <int DT>
__device__ __forceinline__ f32x4_t mma(u32x4_t a, u32x4_t b, f32x4_t c) {
  if constexpr (DT == AQMB_F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// Of 64 rows from row0 on: lane l has row row0 + l and the number of its adapter (-1: none).
struct Rows {
  int row, adapter;
  bool in;
};
__device__ __forceinline__ Rows rows_at(const AdapterArgs& a, int row0) {
  Rows r;
  r.row = row0 + threadIdx.x % 64;
  r.in = r.row < a.n_rows;
  r.adapter = r.in ? a.index[r.row] : -1;
  if ((unsigned)r.adapter >= (unsigned)a.ad.n_adapters) r.adapter = -1;
  return r;
}
// Up to 16 of them that share an adapter.
struct Tile {
  int adapter, count;
  int row;             // of slot lane % 16; slots past count repeat the first
};
// The rows of `mask` from number `first` on. All lanes of the wave take part.
__device__ __forceinline__ Tile tile_of(const Rows& r, uint64_t mask, int adapter, int first) {
  const int lane = threadIdx.x % 64;
  Tile t;
  t.adapter = adapter;
  t.count = min(__builtin_popcountll(mask) - first, 16);
  // Each row's lane sends its number to its slot; the others to lane 63, which is no slot then. Then all read theirs.
  const int at = __builtin_popcountll(mask & ((1ull << lane) - 1)) - first;
  const bool mine = (mask >> lane & 1) && at >= 0 && at < t.count;
  const int sent = __builtin_amdgcn_ds_permute((mine ? at : 63) * 4, r.row);
  const int slot = lane % 16;
  t.row = __builtin_amdgcn_ds_bpermute((slot < t.count ? slot : 0) * 4, sent);
  return t;
}
// The tile of 16 that starts with row `start`, if one does: every 16th of its adapter's rows among its 64 starts one.
__device__ __forceinline__ bool tile_at(const AdapterArgs& a, int start, Tile& t) {
  const Rows r = rows_at(a, start / kRows * kRows);
  const int l = start % kRows, n = __builtin_amdgcn_readlane(r.adapter, l);
  const uint64_t mask = __ballot(r.in && r.adapter == n);
  const int first = __builtin_popcountll(mask & ((1ull << l) - 1));
  if (first % 16) return false;
  t = tile_of(r, mask, n, first);
  return true;
}

__device__ __forceinline__ int own_rank(const AdapterArgs& a, int adapter) {
  return adapter < 0 ? 0 : a.ad.ranks ? min(max(a.ad.ranks[adapter], 0), a.ad.rank) : a.ad.rank;
}

// Few rows: blockIdx.x is the row that a tile starts with, blockIdx.y a part of the inputs, which the waves share out,
// blockIdx.z 64 values of t (with all of a rank above 64 in one workgroup no loads were ahead of the products: 3 adapters of
// rank 128, 1552 x 2104, one row 21 us a call, now 12).
// kOne: one workgroup a unit, by the registers that it may take.
template <int DT, int RT, bool kOdd, bool kOne>
__global__ __launch_bounds__(64 * kFewWaves) __attribute__((amdgpu_waves_per_eu(2, kOne ? 2 : 8))) void shrink_few(AdapterArgs a) {
  constexpr int U = RT <= 2 ? 4 : 2;                 // steps of 32 inputs loaded at once
  __shared__ __align__(16) float lds[2][kFewWaves][256];
  __shared__ int slots[16];
  Tile t;
  if (!tile_at(a, blockIdx.x, t)) return;
  const int m0 = 64 * blockIdx.z, rank = own_rank(a, t.adapter) - m0;
  if (rank <= 0) return;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, i = lane % 16, kg = lane / 16 * 8, d_in = a.ad.d_in;
  const uint16_t* x = (const uint16_t*)a.x + t.row * a.x_stride + kg;
  const uint16_t* w[RT];
#pragma unroll
  for (int m = 0; m < RT; ++m)
    w[m] = (const uint16_t*)a.ad.a + ((int64_t)t.adapter * a.ad.rank + m0 + min(16 * m + i, rank - 1)) * d_in + kg;

  f32x4_t acc[RT] = {};
  const int steps = (d_in + 31) / 32, parts = a.splits * kFewWaves, p = blockIdx.y * kFewWaves + wave;
  const int k0 = (int)((int64_t)steps * p / parts) * 32, k1 = min((int)((int64_t)steps * (p + 1) / parts) * 32, d_in);
  const int whole = k0 + (k1 - k0) / (32 * U) * (32 * U);
  struct Batch { Loaded8<kOdd> x[U], w[U][RT]; };
  const auto load = [&](Batch& b, int k) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      b.x[u].load(x + (uint32_t)(k + 32 * u));
#pragma unroll
      for (int m = 0; m < RT; ++m)
        if (16 * m < rank) b.w[u][m].load(w[m] + (uint32_t)(k + 32 * u));
    }
  };
  const auto multiply = [&](const Batch& b) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const u32x4_t xv = b.x[u].value(x);                          // steps of 32: p's two low bits are those of the row
#pragma unroll
      for (int m = 0; m < RT; ++m)
        if (16 * m < rank) acc[m] = mma<DT>(b.w[u][m].value(w[m]), xv, acc[m]);
    }
  };
  if (whole > k0) {
    Batch now, next;
    load(now, k0);
    for (int k = k0 + 32 * U; k < whole; k += 32 * U) {
      load(next, k);
      multiply(now);
      now = next;
    }
    multiply(now);
  }
  if (d_in < 8) {                                                  // one step, by single values
    if (whole < k1) {
      const u32x4_t xv = load8(x - kg, kg, d_in);
#pragma unroll
      for (int m = 0; m < RT; ++m)
        if (16 * m < rank) acc[m] = mma<DT>(load8(w[m] - kg, kg, d_in), xv, acc[m]);
    }
  } else if (whole < k1) {                                         // fewer than U steps, the last of fewer inputs, loaded at once
    Batch b;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = whole + 32 * u;
      if (k >= k1) break;
      b.x[u].load(x - kg + min(k + kg, d_in - 8));
#pragma unroll
      for (int m = 0; m < RT; ++m)
        if (16 * m < rank) b.w[u][m].load(w[m] - kg + min(k + kg, d_in - 8));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = whole + 32 * u;
      if (k >= k1) break;
      const u32x4_t xv = moved8(b.x[u].value(x - kg + min(k + kg, d_in - 8)), k + kg, d_in);
#pragma unroll
      for (int m = 0; m < RT; ++m)
        if (16 * m < rank) acc[m] = mma<DT>(moved8(b.w[u][m].value(w[m] - kg + min(k + kg, d_in - 8)), k + kg, d_in), xv, acc[m]);
    }
  }

  // The waves' sums added up, 16 values of t at a time.
  float* out = a.t + (int64_t)blockIdx.y * a.n_rows * a.t_stride + m0;
  if (threadIdx.x < 16) slots[threadIdx.x] = t.row;
#pragma unroll
  for (int m = 0; m < RT; ++m) {
    if (16 * m >= rank) break;                                     // the whole workgroup
    *(f32x4_t*)&lds[m % 2][wave][lane * 4] = acc[m];
    __syncthreads();
    for (int e = threadIdx.x; e < 256; e += 64 * kFewWaves) {
      float s = 0.f;
#pragma unroll
      for (int n = 0; n < kFewWaves; ++n) s += lds[m % 2][n][e];
      const int l = e / 4, slot = l % 16;
      if (slot < t.count) out[(int64_t)slots[slot] * a.t_stride + 16 * m + l / 16 * 4 + e % 4] = s;
    }
  }
}

// Many rows: blockIdx.x is a tile of 64 rows, blockIdx.y a part of the inputs, a wave for 16 rows. Steps of 64 inputs go
// through LDS, where eight lanes side by side write 128 bytes of a row: rows side by side in the lanes, as
// the matrix instructions take them, would make every lane an access of its own to the vector cache. The eight pieces of
// a row are swapped by the row against bank conflicts.
template <int DT, int RT>
__global__ __launch_bounds__(256, 2) void shrink_many(AdapterArgs a) {
  constexpr int kAhead = RT <= 2 ? 2 : 1;                          // steps whose loads are under way
  constexpr int kW = (RT + 1) / 2;                                 // pieces of A of a thread
  __shared__ u32x4_t xs[2][64 * 8], ws[2][RT * 16 * 8];
  if ((int)blockIdx.x >= *a.n_tiles) return;
  const int4 tile = a.tiles[blockIdx.x];
  const int rank = own_rank(a, tile.x);
  if (rank == 0) return;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, i = lane % 16, q = lane / 16, d_in = a.ad.d_in;
  // This thread's pieces: of rows r and r + 32 of x, and of rows r + 32 j of A.
  const int r = threadIdx.x / 8, piece = threadIdx.x % 8;
  const uint16_t* x[2];
  const uint16_t* w[kW];
#pragma unroll
  for (int j = 0; j < 2; ++j)
    x[j] = (const uint16_t*)a.x + a.order[tile.y + min(r + 32 * j, tile.z - 1)] * a.x_stride;
#pragma unroll
  for (int j = 0; j < kW; ++j) w[j] = (const uint16_t*)a.ad.a + ((int64_t)tile.x * a.ad.rank + min(r + 32 * j, rank - 1)) * d_in;
  const int steps = d_in / 64;                                     // whole ones; the rest is the last part's
  const int s0 = (int)((int64_t)steps * blockIdx.y / a.splits), s1 = (int)((int64_t)steps * (blockIdx.y + 1) / a.splits);

  struct Step { u32x4_t x[2], w[kW]; };
  const auto load = [&](Step& b, int s) {
#pragma unroll
    for (int j = 0; j < 2; ++j) b.x[j] = load8(x[j], 64 * s + 8 * piece);
#pragma unroll
    for (int j = 0; j < kW; ++j)
      if (32 * j < rank) b.w[j] = load8(w[j], 64 * s + 8 * piece);
  };
  const auto place = [&](const Step& b, int n) {
#pragma unroll
    for (int j = 0; j < 2; ++j) xs[n][(r + 32 * j) * 8 + (piece ^ (r % 8))] = b.x[j];
#pragma unroll
    for (int j = 0; j < kW; ++j)
      if (RT % 2 == 0 || r < 16) ws[n][(r + 32 * j) * 8 + (piece ^ (r % 8))] = b.w[j];
  };
  f32x4_t acc[RT] = {};
  const auto multiply = [&](int n) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = i * 8 + ((4 * h + q) ^ (i % 8));
      const u32x4_t xv = xs[n][wave * 128 + at];
#pragma unroll
      for (int m = 0; m < RT; ++m)
        if (16 * m < rank) acc[m] = mma<DT>(ws[n][m * 128 + at], xv, acc[m]);
    }
  };
  Step ahead[kAhead];
#pragma unroll
  for (int n = 0; n < kAhead; ++n)
    if (s0 + n < s1) load(ahead[n], s0 + n);
#pragma unroll 1
  for (int first = s0; first < s1; first += 2 * kAhead) {
#pragma unroll
    for (int n = 0; n < 2 * kAhead; ++n) {
      const int s = first + n;
      if (s >= s1) break;
      place(ahead[n % kAhead], n % 2);
      if (s + kAhead < s1) load(ahead[n % kAhead], s + kAhead);
      __syncthreads();
      multiply(n % 2);
    }
  }
  if (d_in % 64 && blockIdx.y + 1 == (unsigned)a.splits) {
    __syncthreads();
    Step b;
#pragma unroll
    for (int j = 0; j < 2; ++j) b.x[j] = load8(x[j], 64 * steps + 8 * piece, d_in);
#pragma unroll
    for (int j = 0; j < kW; ++j)
      if (32 * j < rank) b.w[j] = load8(w[j], 64 * steps + 8 * piece, d_in);
    place(b, 0);
    __syncthreads();
    multiply(0);
  }
  if (16 * wave + i >= tile.z) return;
  float* out = a.t + ((int64_t)blockIdx.y * a.n_rows + a.order[tile.y + 16 * wave + i]) * a.t_stride + 4 * q;
#pragma unroll
  for (int m = 0; m < RT; ++m)
    if (16 * m < rank) *(f32x4_t*)(out + 16 * m) = acc[m];
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
// What the second launch keeps in LDS: 128 outputs' weights of a step of 32 of the rank, output 8 c + n as row 16 n + c,
// where the matrix instructions take it, 64 bytes a row, the four pieces swapped by c / 4 against bank conflicts; and t's
// operands of every step and part.
typedef u32x4_t WeightsLds[8][68];
template <int DT> using OperandsLds = u32x4_t[Parts<DT>::kN][64];

// Which of a lane's 8 values are an adapter's own, the first `left`, as a mask.
__device__ __forceinline__ u32x4_t own_values(int left) {
  return u32x4_t{left >= 2 ? 0xFFFFFFFFu : left == 1 ? 0xFFFFu : 0, left >= 4 ? 0xFFFFFFFFu : left == 3 ? 0xFFFFu : 0,
                 left >= 6 ? 0xFFFFFFFFu : left == 5 ? 0xFFFFu : 0, left >= 8 ? 0xFFFFFFFFu : left == 7 ? 0xFFFFu : 0};
}

// s_n t of 16 rows (`row` for slot lane % 16) as the second product's operands, into to[step][part][lane]; the factor of the
// rows' results (fp16) into back. By one wave, or by kWaves of a workgroup (all of them), a step each in turn.
template <int DT, int kWaves>
__device__ __forceinline__ void operands(const AdapterArgs& a, int row, int rank, float scale, OperandsLds<DT>* to, float* back,
                                         uint32_t (*bigs)[16]) {
  typedef Parts<DT> P;
  const int lane = threadIdx.x % 64, q = lane / 16, steps = (rank + 31) / 32, wave = kWaves > 1 ? threadIdx.x / 64 : 0;
  const float* tp = a.t + (int64_t)row * a.t_stride + 8 * q;
  struct Sums { f32x4_t lo[kMaxSplits], hi[kMaxSplits]; };
  const auto load = [&](int kt, Sums& s) {
#pragma unroll
    for (int p = 0; p < kMaxSplits; ++p) {
      s.lo[p] = s.hi[p] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (p < a.splits && 32 * kt + 8 * q < a.t_stride) {    // not by rank, which may still be on its way
        const f32x4_t* from = (const f32x4_t*)(tp + p * (int64_t)a.n_rows * a.t_stride + 32 * kt);
        s.lo[p] = from[0], s.hi[p] = from[1];
      }
    }
  };
  const auto put = [&](int kt, float* v) {
#pragma unroll
    for (int p = 0; p < P::kN; ++p) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        w[j] = P::pack(v[2 * j], v[2 * j + 1]);
        v[2 * j] -= P::lo(w[j]);
        v[2 * j + 1] -= P::hi(w[j]);
      }
      to[kt][p][lane] = u32x4_t{w[0], w[1], w[2], w[3]};
    }
  };
  uint32_t big = 0;
  // Partial sums added up, scaled, 0 from the adapter's rank on. fp16's are kept where their parts will be.
  const auto take = [&](int kt, Sums& s) {
#pragma unroll
    for (int p = 1; p < kMaxSplits; ++p) s.lo[0] += s.lo[p], s.hi[0] += s.hi[p];
    const f32x4_t l = s.lo[0], h = s.hi[0];
    float v[8] = {l.x, l.y, l.z, l.w, h.x, h.y, h.z, h.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 32 * kt + 8 * q + j < rank ? v[j] * scale : 0.f;
    if constexpr (DT == AQMB_F16) {
#pragma unroll
      for (int j = 0; j < 8; ++j) big = max(big, __builtin_bit_cast(uint32_t, v[j]) & 0x7FFFFFFFu);
      to[kt][0][lane] = __builtin_bit_cast(u32x4_t, f32x4_t{v[0], v[1], v[2], v[3]});
      to[kt][1][lane] = __builtin_bit_cast(u32x4_t, f32x4_t{v[4], v[5], v[6], v[7]});
    } else {
      put(kt, v);
    }
  };
  constexpr int kAhead = kWaves > 1 ? 1 : 2;                 // steps on their way at once
  Sums s[kAhead];
  load(wave, s[0]);
  for (int kt = wave; kt < steps; kt += kAhead * kWaves) {
#pragma unroll
    for (int n = 0; n < kAhead; ++n)
      if ((n || kt != wave) && kt + n * kWaves < steps) load(kt + n * kWaves, s[n]);
#pragma unroll
    for (int n = 0; n < kAhead; ++n)
      if (kt + n * kWaves < steps) take(kt + n * kWaves, s[n]);
  }
  if constexpr (DT == AQMB_F16) {
    // By a power of two, so that the row's largest magnitude is in [2^13, 2^14): in fp16's range, the parts far
    // from its subnormals.
    big = max(big, (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (lane ^ 16), (int)big));
    big = max(big, (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (lane ^ 32), (int)big));
    if constexpr (kWaves > 1) {
      if (lane < 16) bigs[wave][lane] = big;
      __syncthreads();
#pragma unroll
      for (int n = 0; n < kWaves; ++n) big = max(big, bigs[n][lane % 16]);
    }
    const int ex = min(max((int)(big >> 23), 14), 254);      // the exponent that goes to 13
    const float fwd = __builtin_bit_cast(float, (uint32_t)(267 - ex) << 23);
    if (wave == 0 && lane < 16) back[lane] = __builtin_bit_cast(float, (uint32_t)(ex - 13) << 23);
    for (int kt = wave; kt < steps; kt += kWaves) {
      const f32x4_t l = __builtin_bit_cast(f32x4_t, to[kt][0][lane]) * fwd, h = __builtin_bit_cast(f32x4_t, to[kt][1][lane]) * fwd;
      float v[8] = {l.x, l.y, l.z, l.w, h.x, h.y, h.z, h.w};
      put(kt, v);
    }
  }
}

// 8 neighbouring outputs of a row as they are stored (16 bits or, kWide, binary32).
template <bool kWide> struct Eight { u32x4_t v[kWide ? 2 : 1]; };
// From element o on. kEights: rows of a multiple of 8 elements, so that all 8 exist or none (then others are read).
template <bool kWide, bool kEights>
__device__ __forceinline__ Eight<kWide> load_y(const void* row, int o, int n) {
  Eight<kWide> r;
  if constexpr (kWide) {
    const float* p = (const float*)row + (kEights ? min(o, n - 8) : o);
    if (kEights || o + 8 <= n) {
      r.v[0] = __builtin_bit_cast(u32x4_t, *(const F4*)p);
      r.v[1] = __builtin_bit_cast(u32x4_t, *(const F4*)(p + 4));
    } else {
      f32x4_t lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
      if (o < n) lo.x = p[0];
      if (o + 1 < n) lo.y = p[1];
      if (o + 2 < n) lo.z = p[2];
      if (o + 3 < n) lo.w = p[3];
      if (o + 4 < n) hi.x = p[4];
      if (o + 5 < n) hi.y = p[5];
      if (o + 6 < n) hi.z = p[6];
      r.v[0] = __builtin_bit_cast(u32x4_t, lo), r.v[1] = __builtin_bit_cast(u32x4_t, hi);
    }
  } else {
    r.v[0] = kEights ? load8((const uint16_t*)row, min(o, n - 8)) : load8((const uint16_t*)row, o, n);
  }
  return r;
}
template <bool kWide, bool kEights, bool kStream>
__device__ __forceinline__ void store_y(void* row, int o, int n, const Eight<kWide>& r) {
  typedef u32x4_t __attribute__((aligned(2))) Unaligned;
  if (o >= n) return;
  if (kStream && kEights) {
#pragma unroll
    for (int h = 0; h < (kWide ? 2 : 1); ++h)
      __builtin_nontemporal_store(r.v[h], (Unaligned*)((char*)row + (int64_t)o * (kWide ? 4 : 2) + 16 * h));
    return;
  }
  if constexpr (kWide) {
    float* p = (float*)row + o;
    if (kEights || o + 8 <= n) {
      *(F4*)p = __builtin_bit_cast(F4, r.v[0]);
      *(F4*)(p + 4) = __builtin_bit_cast(F4, r.v[1]);
    } else {
      const f32x4_t lo = __builtin_bit_cast(f32x4_t, r.v[0]), hi = __builtin_bit_cast(f32x4_t, r.v[1]);
      p[0] = lo.x;
      if (o + 1 < n) p[1] = lo.y;
      if (o + 2 < n) p[2] = lo.z;
      if (o + 3 < n) p[3] = lo.w;
      if (o + 4 < n) p[4] = hi.x;
      if (o + 5 < n) p[5] = hi.y;
      if (o + 6 < n) p[6] = hi.z;
    }
  } else {
    uint16_t* p = (uint16_t*)row + o;
    const u32x4_t v = r.v[0];
    if (kEights || o + 8 <= n) {
      *(Raw8*)p = __builtin_bit_cast(Raw8, v);
    } else {
      p[0] = (uint16_t)v.x;
      if (o + 1 < n) p[1] = (uint16_t)(v.x >> 16);
      if (o + 2 < n) p[2] = (uint16_t)v.y;
      if (o + 3 < n) p[3] = (uint16_t)(v.y >> 16);
      if (o + 4 < n) p[4] = (uint16_t)v.z;
      if (o + 5 < n) p[5] = (uint16_t)(v.z >> 16);
      if (o + 6 < n) p[6] = (uint16_t)v.w;
    }
  }
}
// r += back * d[n][j], n < 8, rounded once (back is a power of two, 1 where kScaled is not set).
template <bool kWide, bool kScaled>
__device__ __forceinline__ void add_y(Eight<kWide>& r, const f32x4_t (&d)[8], int j, float back, bool f16) {
  const auto sum = [&](float x, float y) { return kScaled ? fmaf(y, back, x) : x + y; };
  if constexpr (kWide) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4_t f = __builtin_bit_cast(f32x4_t, r.v[h]);
      r.v[h] = __builtin_bit_cast(u32x4_t, f32x4_t{sum(f.x, d[4 * h][j]), sum(f.y, d[4 * h + 1][j]), sum(f.z, d[4 * h + 2][j]),
                                                   sum(f.w, d[4 * h + 3][j])});
    }
  } else {
    const auto two = [&](uint32_t w, float x, float y) {
      return f16 ? pack_f16x2(sum(f16lo(w), x), sum(f16hi(w), y)) : pack_bf16x2(sum(bf16lo(w), x), sum(bf16hi(w), y));
    };
    r.v[0] = u32x4_t{two(r.v[0].x, d[0][j], d[1][j]), two(r.v[0].y, d[2][j], d[3][j]), two(r.v[0].z, d[4][j], d[5][j]),
                     two(r.v[0].w, d[6][j], d[7][j])};
  }
}

// Few rows: blockIdx.y is the row that a tile starts with, each of four waves takes 128 outputs. Lane (q, c) of 4 x 16 has outputs 8 c .. 8 c + 7 of 128 of rows 4 q .. 4 q + 3: a quarter of the wave reads and
// writes 256 bytes of a row at once (with lanes side by side on different rows every lane was an access of its own to the
// vector cache, which bound the kernel). Bound by latency (4.9 us) or the adapters' bytes
// (32 rows of some 25 adapters of rank 64, 11008 outputs: 13 us).
template <int DT, bool kWide, bool kEights>
__global__ __launch_bounds__(256, kWide || !kEights ? 2 : 3) void expand_few(AdapterArgs a) {
  constexpr int kParts = Parts<DT>::kN, kSize = kWide ? 4 : 2;
  extern __shared__ __align__(16) char all[];            // the waves' weights, t's operands
  __shared__ float back[16];
  __shared__ uint32_t bigs[4][16];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = lane % 16, q = lane / 16, d_out = a.ad.d_out, stack = a.ad.rank;
  WeightsLds& weights = ((WeightsLds*)all)[wave];
  OperandsLds<DT>* const operand = (OperandsLds<DT>*)(all + 4 * sizeof(WeightsLds));
  Tile t;
  if (!tile_at(a, blockIdx.y, t)) return;                // the whole workgroup
  const int o = (blockIdx.x * 4 + wave) * 128;
  int rank = stack;
  int row[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) row[j] = __builtin_amdgcn_ds_bpermute(4 * (4 * q + j), t.row);
  const auto store_rows = [&](const Eight<kWide>* y) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (4 * q + j < t.count)
        store_y<kWide, kEights, false>((char*)a.out + row[j] * (a.out_stride * kSize), o + 8 * c, d_out, y[j]);
  };
  // Weights in pieces of 8: `pieces` lanes side by side (a power of two) to an output's row of a step.
  const uint16_t* b = (const uint16_t*)a.ad.b + (int64_t)t.adapter * d_out * stack;
  const auto shift_of = [&](int kt) { const int left = (kt < 2 ? stack : rank) - 32 * kt; return left > 16 ? 2 : left > 8 ? 1 : 0; };
  const auto load_w = [&](u32x4_t* w, int kt) {
    const int shift = shift_of(kt), l = lane, k = 32 * kt + 8 * (l & ((1 << shift) - 1));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= 2 << shift) break;
      const uint32_t r = min(o + ((64 * j + l) >> shift), d_out - 1) * (uint32_t)stack;     // below 2^31
      if constexpr (kEights) w[j] = load8(b, r + min(k, stack - 8));
      else w[j] = stack >= 8 ? load8_last(b + r, k, stack) : load8(b + r, k, stack);
    }
  };
  const auto place_w = [&](const u32x4_t* w, int kt) {
    const int shift = shift_of(kt), l = lane;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= 2 << shift) break;
      const int o = (64 * j + l) >> shift, piece = l & ((1 << shift) - 1);
      weights[o % 8][o / 8 * 4 + (piece ^ (o / 32))] = kEights || stack < 8 ? w[j] : moved8(w[j], 32 * kt + 8 * piece, stack);
    }
  };
  // Two steps' weights and the rows of base are on their way while t and the adapter's rank come.
  u32x4_t w[2][8];
  Eight<kWide> y[4];
  if (o < d_out) {
    if (t.adapter >= 0) load_w(w[0], 0);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      y[j] = load_y<kWide, kEights>((const char*)a.base + row[j] * (a.base_stride * kSize), o + 8 * c, d_out);
    if (t.adapter >= 0 && stack > 32) load_w(w[1], 1);
  }
  rank = own_rank(a, t.adapter);
  if (rank == 0) {
    if (a.base != a.out && o < d_out) store_rows(y);
    return;
  }
  const u32x4_t mask = own_values(rank - (rank - 1) / 32 * 32 - 8 * q);      // of the last step
  operands<DT, 4>(a, t.row, rank, a.ad.scales ? a.ad.scales[t.adapter] : 1.f, operand, back, bigs);
  __syncthreads();
  if (o >= d_out) return;

  f32x4_t acc[8] = {};
  const auto step = [&](u32x4_t* w, int kt) {
    lds_order();
    place_w(w, kt);
    if (32 * (kt + 2) < rank) load_w(w, kt + 2);
    lds_order();
    u32x4_t tv[kParts];
#pragma unroll
    for (int p = 0; p < kParts; ++p) tv[p] = operand[kt][p][lane];
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      u32x4_t wv = weights[n][c * 4 + (q ^ (c / 4))];
      if (32 * (kt + 1) >= rank) wv &= mask;
#pragma unroll
      for (int p = kParts - 1; p >= 0; --p) acc[n] = mma<DT>(tv[p], wv, acc[n]);
    }
  };
  for (int kt = 0; 32 * kt < rank; kt += 2) {
    step(w[0], kt);
    if (32 * (kt + 1) < rank) step(w[1], kt + 1);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) add_y<kWide, DT == AQMB_F16>(y[j], acc, j, DT == AQMB_F16 ? back[4 * q + j] : 1.f, a.y_f16);
  store_rows(y);
}

// Many: a tile of 64 rows, four waves with 16 each, and a.per_group outputs. As expand_few, but the waves bring the weights
// into LDS together, into one of two places while the other is read (each its own: 8192 rows of 4096 outputs at rank 32
// 41 us, now 34; a call at rank 128 165 us, now 134), and the next outputs of base are loaded a step ahead. Four
// waves a SIMD where the registers suffice (two: 38 us; five spill).
template <int DT, bool kWide, bool kEights>
__global__ __launch_bounds__(256, kWide || !kEights ? 3 : 4) void expand_many(AdapterArgs a) {
  typedef Parts<DT> P;
  constexpr int kParts = P::kN, kSize = kWide ? 4 : 2;
  extern __shared__ __align__(16) char all[];
  WeightsLds* const shared = (WeightsLds*)all;                               // two
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = lane % 16, q = lane / 16, d_out = a.ad.d_out, stack = a.ad.rank;
  // Neighbours in the grid take neighbouring outputs of the same rows.
  const int parts = (d_out + a.per_group - 1) / a.per_group, at_tile = blockIdx.x / parts;
  if (at_tile >= *a.n_tiles) return;
  const int4 tile = a.tiles[at_tile];
  const int first = 16 * wave, count = min(max(tile.z - first, 0), 16), rank = own_rank(a, tile.x);
  const int o0 = (blockIdx.x - at_tile * parts) * a.per_group, o1 = min(o0 + a.per_group, d_out);
  if (rank == 0 && (a.base == a.out || count == 0)) return;                  // of a whole tile, or of a wave that copies nothing
  // The wave's rows 4 q + j; for those that do not exist the tile's first.
  int row[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) row[j] = a.order[tile.y + (4 * q + j < count ? first + 4 * q + j : 0)];
  // A value that the compiler takes for new in every step: addresses made from it are not kept in registers between steps.
  const auto fresh = [](int v) { asm volatile("" : "+v"(v)); return v; };
  const auto load_rows = [&](Eight<kWide>* y, int o) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      y[j] = load_y<kWide, kEights>((const char*)a.base + fresh(row[j]) * (a.base_stride * kSize), o + 8 * c, d_out);
  };
  const auto store_rows = [&](const Eight<kWide>* y, int o) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (4 * q + j < count)
        store_y<kWide, kEights, true>((char*)a.out + fresh(row[j]) * (a.out_stride * kSize), o + 8 * c, d_out, y[j]);
  };
  Eight<kWide> y[4];
  if (rank == 0) {
    for (int o = o0; o < o1; o += 128) {
      load_rows(y, o);
      store_rows(y, o);
    }
    return;
  }

  // A thread's one or two pieces of 8 of a step's 128 x 32 weights; `pieces` threads side by side to an output's row.
  const uint16_t* b = (const uint16_t*)a.ad.b + (int64_t)tile.x * d_out * stack;
  const auto load_w = [&](u32x4_t* w, int o, int kt) {
    const int left = rank - 32 * kt, shift = left > 16 ? 2 : left > 8 ? 1 : 0, k = 32 * kt + 8 * (threadIdx.x & ((1 << shift) - 1));
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int at = (256 * j + (int)threadIdx.x) >> shift;
      if (at >= 128) continue;
      const uint32_t r = min(o + at, d_out - 1) * (uint32_t)stack;           // below 2^31
      if constexpr (kEights) w[j] = load8(b, r + min(k, stack - 8));
      else w[j] = stack >= 8 ? load8_last(b + r, k, stack) : load8(b + r, k, stack);
    }
  };
  const auto place_w = [&](const u32x4_t* w, WeightsLds& to, int kt) {
    const int left = rank - 32 * kt, shift = left > 16 ? 2 : left > 8 ? 1 : 0, piece = threadIdx.x & ((1 << shift) - 1);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int at = (256 * j + (int)threadIdx.x) >> shift;
      if (at < 128)
        to[at % 8][at / 8 * 4 + (piece ^ (at / 32))] = kEights || stack < 8 ? w[j] : moved8(w[j], 32 * kt + 8 * piece, stack);
    }
  };
  u32x4_t w[2];
  load_w(w, o0, 0);
  load_rows(y, o0);
  OperandsLds<DT>* const t = (OperandsLds<DT>*)(all + 2 * sizeof(WeightsLds)) + wave * ((stack + 31) / 32);
  __shared__ float backs[4][16];
  if (count)
    operands<DT, 1>(a, a.order[tile.y + (c < count ? first + c : 0)], rank, a.ad.scales ? a.ad.scales[tile.x] : 1.f, t, backs[wave], nullptr);

  int n = 0;
  for (int o = o0; o < o1; o += 128) {
    const bool more = o + 128 < o1;
    Eight<kWide> next[4];
    if (more && count) load_rows(next, o + 128);
    f32x4_t acc[8] = {};
    for (int kt = 0; 32 * kt < rank; ++kt, n ^= 1) {
      const bool last = 32 * (kt + 1) >= rank;
      place_w(w, shared[n], kt);
      if (!last) load_w(w, o, kt + 1);
      else if (more) load_w(w, o + 128, 0);
      __syncthreads();
      if (count == 0) continue;
      u32x4_t tv[kParts];
#pragma unroll
      for (int p = 0; p < kParts; ++p) tv[p] = t[kt][p][lane];
      u32x4_t mask;
      if (last) mask = own_values(rank - 32 * kt - 8 * q);
#pragma unroll
      for (int m = 0; m < 8; ++m) {
        u32x4_t wv = shared[n][m][c * 4 + (q ^ (c / 4))];
        if (last) wv &= mask;
#pragma unroll
        for (int p = kParts - 1; p >= 0; --p) acc[m] = mma<DT>(tv[p], wv, acc[m]);
      }
    }
    if (count == 0) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) add_y<kWide, DT == AQMB_F16>(y[j], acc, j, DT == AQMB_F16 ? backs[wave][4 * q + j] : 1.f, a.y_f16);
    store_rows(y, o);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = next[j];
  }
}

// Many rows sorted by adapter (those without one last), and cut into tiles of up to 64 (adapter, first, count): one workgroup
// counts, adds up and places. Rows of one adapter come in any order, which nothing depends on. 8192 rows 10 us; above, the
// indexes are read twice: 65536 rows in spans of 8 adapters 66 us, of 64 in any order 74.
__global__ __launch_bounds__(1024) void sort_kernel(AdapterArgs a) {
  __shared__ int bins[kMaxAdapters + 1], sums[2][16];
  constexpr int kEach = 8;       // rows of a thread at once
  const int n_bins = a.ad.n_adapters + 1, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  for (int i = threadIdx.x; i < n_bins; i += 1024) bins[i] = 0;
  __syncthreads();
  // The bins of kEach rows a thread, and each one's place in its bin; a wave's rows that all have one adapter take
  // theirs at once.
  int n[kEach], at[kEach];
  const auto take = [&](int r0) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int r = r0 + 1024 * j + threadIdx.x;
      n[j] = r < a.n_rows ? a.index[r] : -1;
      if ((unsigned)n[j] >= (unsigned)a.ad.n_adapters) n[j] = a.ad.n_adapters;
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const bool in = r0 + 1024 * j + threadIdx.x < a.n_rows;
      const uint64_t all = __ballot(in);
      const bool one = (all & ~__ballot(n[j] == __builtin_amdgcn_readfirstlane(n[j]))) == 0;
      at[j] = 0;
      if (in && (!one || lane == 0)) at[j] = atomicAdd(&bins[n[j]], one ? __builtin_popcountll(all) : 1);
      if (one) at[j] = __builtin_amdgcn_readfirstlane(at[j]) + lane;
    }
  };
  const auto place = [&](int r0) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int r = r0 + 1024 * j + threadIdx.x;
      if (r < a.n_rows) a.order[at[j]] = r;
    }
  };
  const bool once = a.n_rows <= 1024 * kEach;          // the places of the first pass are kept
  for (int r0 = 0; r0 < a.n_rows; r0 += 1024 * kEach) take(r0);
  __syncthreads();
  // Each thread's bins, neighbours; their rows and tiles before it.
  const int per = (n_bins + 1023) / 1024, b0 = threadIdx.x * per, b1 = min(b0 + per, n_bins);
  int rows = 0, tiles = 0;
  for (int i = b0; i < b1; ++i) rows += bins[i], tiles += (bins[i] + 63) / 64;
  int before[2] = {rows, tiles};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int own = before[k];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int v = __builtin_amdgcn_ds_bpermute(4 * (lane - d), before[k]);
      if (lane >= d) before[k] += v;
    }
    if (lane == 63) sums[k][wave] = before[k];
    before[k] -= own;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k)
    for (int w = 0; w < wave; ++w) before[k] += sums[k][w];
  // No store to memory before the barriers: they would wait for it.
  int start = before[0];
  for (int i = b0; i < b1; ++i) {
    const int count = bins[i];
    bins[i] = start;
    start += count;
  }
  __syncthreads();
  int at_tile = before[1];
  for (int i = b0; i < b1; ++i) {
    const int r0 = bins[i], count = (i + 1 < n_bins ? bins[i + 1] : a.n_rows) - r0;
    for (int j = 0; j < count; j += 64) a.tiles[at_tile++] = make_int4(i < a.ad.n_adapters ? i : -1, r0 + j, min(count - j, 64), 0);
  }
  if (threadIdx.x == 1023) *a.n_tiles = at_tile;
  if (once) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) at[j] += bins[n[j]];
    place(0);
  } else {
    __syncthreads();
    for (int r0 = 0; r0 < a.n_rows; r0 += 1024 * kEach) {
      take(r0);
      place(r0);
    }
  }
}

template <int DT, int RT>
hipError_t go_shrink(const AdapterArgs& a, const AdapterPlan& p, hipStream_t st) {
  if (p.few) {
    constexpr int kMost = RT <= 4 ? RT : 4;
    const dim3 grid(a.n_rows, p.splits, (a.ad.rank + 63) / 64);
    // Rows at addresses that are no multiples of 4 bytes.
    const bool odd = ((uintptr_t)a.x | (uintptr_t)a.ad.a) % 4 || a.x_stride % 2 || a.ad.d_in % 2;
    // Most workgroups have no tile and end at once; where few have one, two of them would share a unit while others are idle.
    // 4096 x 4096, shared and one a unit: 48 workgroups with a tile at least (150 rows, 4 adapters of rank 64) 21.2 us a call and
    // 18.1, 96 (8 adapters) 21.4 and 18.1, 144 (12) 21.5 and 21.7; 64 (250 rows, 4 of rank 32) 15.4 and 14.3, 96 (6) 15.2 and 15.0,
    // 160 (10) 15.0 and 16.5; 128 (128 rows, 16 of rank 16) 11.5 and 12.3; 104 (40 rows, 13 of
    // rank 128, 11008 outputs) 30.4 and 26.2. Else up to 64 rows the same.
    const int groups = (a.n_rows + kRows - 1) / kRows * min(a.ad.n_adapters, kRows);
    const bool one = max(a.n_rows / 16, min(groups, a.n_rows)) * (int)(grid.y * grid.z) <= 100;
    const auto kernel = odd ? one ? shrink_few<DT, kMost, true, true> : shrink_few<DT, kMost, true, false>
                            : one ? shrink_few<DT, kMost, false, true> : shrink_few<DT, kMost, false, false>;
    kernel<<<grid, 64 * kFewWaves, 0, st>>>(a);
  } else {
    shrink_many<DT, RT><<<dim3(p.tiles, p.splits), 256, 0, st>>>(a);
  }
  return hipGetLastError();
}
template <int DT, bool kWide, bool kEights>
hipError_t go_expand(const AdapterArgs& a, const AdapterPlan& p, hipStream_t st) {
  const size_t operands = (a.ad.rank + 31) / 32 * sizeof(OperandsLds<DT>);
  if (p.few) {                         // within 64 KiB of LDS at any rank
    expand_few<DT, kWide, kEights><<<dim3((a.ad.d_out + 511) / 512, a.n_rows), 256, 4 * sizeof(WeightsLds) + operands, st>>>(a);
  } else {
    const int parts = (a.ad.d_out + a.per_group - 1) / a.per_group;
    const size_t lds = 2 * sizeof(WeightsLds) + 4 * operands;
    const auto kernel = expand_many<DT, kWide, kEights>;
    if (lds + 256 > 65536) {           // with the kernel's own
      // The limit is the kernel's, not the call's: what the largest rank takes, so that no thread lowers another's.
      constexpr int kMost = 2 * sizeof(WeightsLds) + 4 * ((AQMB_MAX_RANK + 31) / 32) * sizeof(OperandsLds<DT>);
      const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kMost);
      if (e != hipSuccess) return e;
    }
    kernel<<<p.tiles * parts, 256, lds, st>>>(a);      // below 2^24: check_adapters
  }
  return hipGetLastError();
}
template <int DT, bool kWide>
hipError_t go_expand(const AdapterArgs& a, const AdapterPlan& p, hipStream_t st) {
  return a.ad.rank % 8 || a.ad.d_out % 8 ? go_expand<DT, kWide, false>(a, p, st) : go_expand<DT, kWide, true>(a, p, st);
}
template <int DT>
hipError_t both(const AdapterArgs& a, const AdapterPlan& p, aqmb_dtype y, hipStream_t st) {
  const int r = a.ad.rank;
  hipError_t e;
  if (!p.few) {
    sort_kernel<<<1, 1024, 0, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  e = r <= 16 ? go_shrink<DT, 1>(a, p, st) : r <= 32 ? go_shrink<DT, 2>(a, p, st)
                       : r <= 64 ? go_shrink<DT, 4>(a, p, st) : r <= 128 ? go_shrink<DT, 8>(a, p, st) : go_shrink<DT, 16>(a, p, st);
  if (e != hipSuccess) return e;
  return y == AQMB_F32 ? go_expand<DT, true>(a, p, st) : go_expand<DT, false>(a, p, st);
}

}  // namespace

// Few rows take a look at 64 rows for every tile of 16; above 256 a sort of its own (4 us for 100 rows, 10 for 8192) and
// tiles of 64 rows are cheaper. Rank 16, 4096 x 4096, 4 adapters in spans: 128 rows 11.8 us against 17.4, 256 16.1 and 18.2,
// 384 22.7 and 18.4; 64 adapters in any order: 12.1 and 20.5, 20.3 and 22.4, 27.3 and 23.8; rank 64, 11008 outputs, 8
// adapters: 25.7 and 26.7, 32.2 and 31.5, 46 and 33.7. Parts of the inputs: as many steps for each wave as it loads at
// once, at least, few rows; about 512 workgroups, many. Many: 256 outputs a workgroup (8192 rows: 128 take 76 us against 67,
// 512 70), 128 where that leaves fewer than 512 (1024 rows 20.9 us against 23.0, 300 18.4 against 21.0).
constexpr int kFewRows = 256;
AdapterPlan adapter_plan(const aqmb_adapters& ad, int n_rows) {
  AdapterPlan p;
  const int steps = (ad.d_in + 31) / 32;
  p.few = n_rows <= kFewRows;
  const int groups = n_rows < ad.n_adapters + 1 ? n_rows : ad.n_adapters + 1;
  p.tiles = groups + (n_rows - groups) / 64;
  p.per_group = 0;
  if (p.few) {
    p.splits = steps / (kFewWaves * (ad.rank <= 32 ? 4 : 2));
  } else {
    p.splits = 512 / ((n_rows + kRows - 1) / kRows);
    if (p.splits > steps / 16) p.splits = steps / 16;
    p.per_group = (int64_t)p.tiles * ((ad.d_out + 255) / 256) < 512 ? 128 : 256;
  }
  if (p.splits > kMaxSplits) p.splits = kMaxSplits;
  if (p.splits < 1) p.splits = 1;
  p.t_stride = (ad.rank + 15) / 16 * 16;
  p.bytes = (size_t)p.splits * n_rows * p.t_stride * 4;
  // Many: behind t the number of tiles, the tiles and the rows' order.
  p.at_tiles = p.bytes;
  if (!p.few) p.bytes += 16 + (size_t)p.tiles * 16 + ((size_t)n_rows + 3) / 4 * 16;
  return p;
}

hipError_t launch_adapters(AdapterArgs a, const AdapterPlan& p, aqmb_dtype y, hipStream_t st) {
  a.t_stride = p.t_stride;
  a.splits = p.splits;
  a.per_group = p.per_group;
  a.y_f16 = y == AQMB_F16;
  a.n_tiles = (int*)((char*)a.t + p.at_tiles);
  a.tiles = (int4*)((char*)a.t + p.at_tiles + 16);
  a.order = (int*)(a.tiles + p.tiles);
  return a.ad.dtype == AQMB_F16 ? both<AQMB_F16>(a, p, y, st) : both<AQMB_BF16>(a, p, y, st);
}

}  // namespace aqmb
