// Log probabilities of given tokens, entropy and the largest values of every row of logits, in one pass over them.
//
//   p = 2^t, t = (x - M) scale / log 2,  s = sum p,  u = sum p t,  M the largest x
//   lse = scale M + log s,  log p_t = scale (x_t - M) - log s,  entropy = log s - log 2 u / s
//
// A lane keeps M, s and u of what it has seen and brings them to a new M once per tile. The largest n_top values are
// kept per wave as sorted 64-bit keys (the value's order, then the lower index) in LDS; a new value has to reach the last of
// them, or that of the workgroup's other waves, and few do. Few rows are cut into chunks, which a second launch joins.
// Many rows without top values are bound by the vector instructions and the logits' bytes alike (2600 rows of 50001 bf16: 63 us, 4.1
// TB/s, 10 instructions a value), with 20 top values by the keys (4096 rows of 32000: 103 us); few rows by latency.
#include "device.h"
#include "ops.h"
#include "wave.h"

// Products are fused with additions only where that is written: every instance of the kernels rounds alike, whatever
// outputs are asked for.
#pragma clang fp contract(off)

namespace aqmb {

namespace {

typedef uint64_t u64x2_t __attribute__((ext_vector_type(2)));
struct __attribute__((packed, aligned(2))) Raw16 { uint32_t w[4]; };

constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f, kInf = __builtin_inff();
constexpr float kLowest = -3.402823466e38f;
constexpr float kFar = -1000.f;  // 2^t is 0 there and below: u's factor stays finite
constexpr int kList = 128;       // keys a wave may hold before it sorts: the top ones and a wave's 64 more

template <int DT> constexpr int kEach = DT == AQMB_F32 ? 4 : 8;     // values of a 16-byte load
template <int DT> constexpr int kPiece = 64 * kEach<DT>;            // values of a wave's load

template <int DT>
__device__ __forceinline__ float value(const void* row, int i) {
  if constexpr (DT == AQMB_F32) return ((const float*)row)[i];
  else if constexpr (DT == AQMB_F16) return f16_to_f32(((const uint16_t*)row)[i]);
  else return bf16lo(((const uint16_t*)row)[i]);
}

template <int DT>
__device__ __forceinline__ void widen(const Raw16& r, float* x) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t w = r.w[j];
    if constexpr (DT == AQMB_F32) {
      x[j] = __builtin_bit_cast(float, w);
    } else {
      x[2 * j] = DT == AQMB_F16 ? f16lo(w) : bf16lo(w);
      x[2 * j + 1] = DT == AQMB_F16 ? f16hi(w) : bf16hi(w);
    }
  }
}

struct Run { float m, s, u; };
// Both brought to the larger of their maxima; the same whichever comes first, so that all lanes get one result. Of an empty one (m = -infinity) s and u are 0.
__device__ __forceinline__ Run join(const Run& a, const Run& b, float c) {
  const float m = fmaxf(a.m, b.m), ref = m == -kInf ? 0.f : m;
  const float ta = (a.m - ref) * c, tb = (b.m - ref) * c;
  const float fa = __builtin_amdgcn_exp2f(ta), fb = __builtin_amdgcn_exp2f(tb);
  return {m, fa * a.s + fb * b.s, fa * fmaf(fmaxf(ta, kFar), a.s, a.u) + fb * fmaf(fmaxf(tb, kFar), b.s, b.u)};
}
// All lanes' runs joined: the largest m first, then what they are at that.
__device__ __forceinline__ Run over_wave(const Run& r, float c) {
  const float m = __builtin_bit_cast(float, over_lanes<64>(__builtin_bit_cast(uint32_t, r.m), [](uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
  }));
  const float t = (r.m - (m == -kInf ? 0.f : m)) * c, f = __builtin_amdgcn_exp2f(t);
  const float s = f * r.s, u = f * fmaf(fmaxf(t, kFar), r.s, r.u);
  return {m, __builtin_bit_cast(float, over_lanes<64>(__builtin_bit_cast(uint32_t, s), add_floats)),
          __builtin_bit_cast(float, over_lanes<64>(__builtin_bit_cast(uint32_t, u), add_floats))};
}

// Larger for a larger value and, among equal ones (-0 and 0 are), for a lower index. Never 0 for a value above -infinity.
__device__ __forceinline__ uint32_t order(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  return b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unorder(uint32_t o) {
  return __builtin_bit_cast(float, o ^ ((uint32_t)((int)~o >> 31) | 0x80000000u));
}
__device__ __forceinline__ uint64_t key_of(float x, int i) { return (uint64_t)order(x) << 32 | (uint32_t)~i; }

__device__ __forceinline__ void lds_order() {      // a wave's LDS accesses run in order; the compiler's do now too
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// A wave's largest keys, in LDS: n of them, of which a new one has to reach `least`.
struct TopList {
  uint64_t* list;              // of kList, 16-byte aligned
  int n, top;
  uint64_t least;

  // The list's keys sorted, largest first, and cut to `top`; if so many are there, `least` is the last. Each key's place is
  // the number of larger ones.
  __device__ __forceinline__ void sort() {
    const int lane = threadIdx.x % 64;
    if (lane < 8 && n + lane < kList) list[n + lane] = 0;        // the loop below counts in eights
    lds_order();
    const uint64_t a = lane < n ? list[lane] : 0, b = lane + 64 < n ? list[lane + 64] : 0;
    int pa = 0, pb = 0;
    for (int i = 0; i < n; i += 8) {
      u64x2_t k[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) k[j] = *(const u64x2_t*)(list + i + 2 * j);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        pa += (k[j].x > a) + (k[j].y > a);
        if (n > 64) pb += (k[j].x > b) + (k[j].y > b);
      }
    }
    lds_order();
    if (lane < n && pa < top) list[pa] = a;
    if (lane + 64 < n && pb < top) list[pb] = b;
    lds_order();
    n = min(n, top);
    if (n == top) least = list[n - 1];
  }
  // The keys of the lanes that say so and reach `least`.
  __device__ __forceinline__ void push(uint64_t key, bool in) {
    in = in && key >= least;
    uint64_t mask = __ballot(in);
    if (mask == 0) return;
    if (n + __builtin_popcountll(mask) > kList) {
      sort();
      in = in && key >= least;
      mask = __ballot(in);
    }
    put(key, mask);
  }
  __device__ __forceinline__ void put(uint64_t key, uint64_t mask) {
    const int lane = threadIdx.x % 64;
    if (mask >> lane & 1) list[n + __builtin_popcountll(mask & ((1ull << lane) - 1))] = key;
    n += __builtin_popcountll(mask);
  }
  // `least` from one value of every lane, in the order's bits: `top` lanes reach it, if so many lanes have one. Not
  // quite the largest such bound: its first bits.
  __device__ __forceinline__ void start(uint32_t o) {
    uint32_t p = 0;
#pragma unroll
    for (int bit = 31; bit >= 18; --bit)
      if (__builtin_popcountll(__ballot(o >= (p | 1u << bit))) >= top) p |= 1u << bit;
    least = (uint64_t)p << 32;
  }
};

// The first 64 tokens that are asked for and their logits, on their way early; lane l has number l.
struct Asked {
  int64_t token;
  float x;
};
template <int DT>
__device__ __forceinline__ Asked asked(const LogProbArgs& a, int64_t row) {
  const int lane = threadIdx.x % 64;
  Asked r = {-1, 0.f};
  if (lane < a.n_targets) {
    r.token = a.targets[row * a.n_targets + lane];
    const char* z = (const char*)a.logits + row * a.stride * (DT == AQMB_F32 ? 4 : 2);
    if (r.token >= 0 && r.token < a.vocab) r.x = value<DT>(z, (int)r.token);
  }
  return r;
}

// What a row has come to, by one wave: keys sorted in `sorted`, n of them.
template <int DT>
__device__ __forceinline__ void finish(const LogProbArgs& a, int64_t row, const Run& r, const Asked& early, const uint64_t* sorted, int n) {
  const int lane = threadIdx.x % 64;
  const char* z = (const char*)a.logits + row * a.stride * (DT == AQMB_F32 ? 4 : 2);
  const bool bad = !(r.s >= 0.f) || r.m == kInf, none = r.s == 0.f;
  const float nan = __builtin_nanf(""), ls = logf(r.s);
  // By halves: the difference itself may overflow.
  const auto log_p = [&](float x) { return bad ? nan : none || x == -kInf ? -kInf : fmaf(2.f, a.scale * (0.5f * x - 0.5f * r.m), -ls); };
  if (lane == 0) {
    if (a.lse) a.lse[row] = bad ? nan : none ? -kInf : fmaf(a.scale, r.m, ls);
    if (a.entropy) a.entropy[row] = bad ? nan : none ? 0.f : fmaxf(fmaf(-kLn2, r.u / r.s, ls), 0.f);
  }
  const auto answer = [&](int i, int64_t t, float x) {
    a.logprobs[row * a.n_targets + i] = t < 0 ? 0.f : t >= a.vocab ? nan : log_p(x);
  };
  if (lane < a.n_targets) answer(lane, early.token, early.x);
  for (int i = lane + 64; i < a.n_targets; i += 64) {
    const int64_t t = a.targets[row * a.n_targets + i];
    answer(i, t, t >= 0 && t < a.vocab ? value<DT>(z, (int)t) : 0.f);
  }
  if (a.n_top == 0) return;
  int id = -1;
  float x = -kInf;
  if (lane < n) {
    const uint64_t k = sorted[lane];
    id = (int)~(uint32_t)k;
    x = unorder((uint32_t)(k >> 32));
  }
  // Too few above -infinity: the lowest tokens at -infinity follow.
  for (int i0 = 0; !bad && n < a.n_top && i0 < a.vocab; i0 += 64) {
    uint64_t mask = __ballot(lane < a.vocab - i0 && value<DT>(z, i0 + lane) == -kInf);
    for (; mask && n < a.n_top; mask &= mask - 1, ++n)
      if (lane == n) id = i0 + __builtin_ctzll(mask);
  }
  if (lane < a.n_top) {
    if (a.top_ids) a.top_ids[row * a.n_top + lane] = bad ? -1 : id;
    if (a.top_logprobs) a.top_logprobs[row * a.n_top + lane] = log_p(x);
  }
}

// A wave's tile is kLoads loads.
template <int DT, int NT, int kLoads, bool kTop>
__global__ __launch_bounds__(NT) void rows_kernel(LogProbArgs a) {
  constexpr int kE = kEach<DT>, kN = kE * kLoads, kWaves = NT / 64, kTile = kPiece<DT> * kLoads;
  __shared__ __align__(16) uint64_t lists[kTop ? kWaves : 1][kTop ? kList : 1];
  __shared__ Run runs[kWaves];
  __shared__ int counts[kWaves];
  __shared__ uint32_t reached;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t row = blockIdx.x;
  const char* z = (const char*)a.logits + row * a.stride * (DT == AQMB_F32 ? 4 : 2);
  const int c0 = blockIdx.y * a.chunk, c1 = min(a.vocab - c0, a.chunk) + c0;
  const float c = a.scale * kLog2E;
  TopList top = {lists[kTop ? wave : 0], 0, a.n_top, 0};
  if constexpr (kTop && kWaves > 1) {
    if (threadIdx.x == 0) reached = order(-kInf);
    __syncthreads();
  }
  float gate = -kInf;          // a later tile's value has to be above this
  bool sorted = true;
  Asked early = {-1, 0.f};
  if (a.splits == 1 && wave == 0) early = asked<DT>(a, row);

  // The values of a load, -infinity, which weighs nothing, from the chunk's end on.
  const auto piece = [&](int64_t i) {
    constexpr uint32_t kNone = DT == AQMB_F32 ? 0xFF800000u : DT == AQMB_F16 ? 0xFC00FC00u : 0xFF80FF80u;
    if (i + kE <= c1) return *(const Raw16*)(z + i * (16 / kE));
    Raw16 raw = {{kNone, kNone, kNone, kNone}};
    for (int j = 0; i + j < c1; ++j) {         // a piece that is cut: its values one by one, each into its place
      const uint32_t w = DT == AQMB_F32 ? ((const uint32_t*)z)[i + j] : ((const uint16_t*)z)[i + j];
      const int shift = DT == AQMB_F32 ? 0 : 16 * (j % 2), word = j * 4 / kE;
      const uint32_t keep = DT == AQMB_F32 ? 0u : ~(0xFFFFu << shift);
#pragma unroll
      for (int n = 0; n < 4; ++n)
        if (n == word) raw.w[n] = (raw.w[n] & keep) | w << shift;
    }
    return raw;
  };
  Run r = {-kInf, 0.f, 0.f};
  for (int64_t t0 = c0 + (int64_t)wave * kTile; t0 < c1; t0 += kWaves * kTile) {
    float x[kN];
    Raw16 raw[kLoads];
    const auto at = [&](int l) { return t0 + (l * 64 + lane) * kE; };
    if (t0 + kTile <= c1) {
#pragma unroll
      for (int l = 0; l < kLoads; ++l) raw[l] = *(const Raw16*)(z + at(l) * (16 / kE));
    } else {
#pragma unroll
      for (int l = 0; l < kLoads; ++l) raw[l] = piece(at(l));
    }
#pragma unroll
    for (int l = 0; l < kLoads; ++l) widen<DT>(raw[l], x + kE * l);
    float m = x[0];
#pragma unroll
    for (int e = 1; e < kN; ++e) m = fmaxf(m, x[e]);
    m = fmaxf(m, -kInf);       // not NaN
    if (__ballot(m > r.m)) {
      const float to = fmaxf(r.m, m), ref = to == -kInf ? 0.f : to, t = (r.m - ref) * c;
      const float f = __builtin_amdgcn_exp2f(t);
      r.u = f * fmaf(fmaxf(t, kFar), r.s, r.u);
      r.s *= f;
      r.m = to;
    }
    const float ref = r.m == -kInf ? 0.f : r.m;
#pragma unroll
    for (int e = 0; e < kN; ++e) {
      const float t = (x[e] - ref) * c, p = __builtin_amdgcn_exp2f(t);
      r.s += p;
      r.u = fmaf(p, fmaxf(t, kFar), r.u);
    }
    if constexpr (kTop) {
      // What all waves' keys have to reach: as many of one wave's do. An equal value may still be the lower token.
      const float others = kWaves > 1 ? unorder(*(volatile uint32_t*)&reached) : kLowest;
      if (!__ballot(m > gate && m >= others)) continue;
      if (top.least == 0) top.start(order(m));
      float bound = fmaxf(fmaxf(unorder((uint32_t)(top.least >> 32)), others), kLowest);
#pragma unroll
      for (int l = 0; l < kLoads; ++l) {
        const int64_t i0 = at(l);
        const float* v = x + kE * l;
        // Which values come into question; nearly always they fit into the list.
        uint64_t masks[kE];
        int more = 0;
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          masks[e] = __ballot(v[e] >= bound);
          more += __builtin_popcountll(masks[e]);
        }
        if (more == 0) continue;
        if (top.n + more <= kList) {
#pragma unroll
          for (int e = 0; e < kE; ++e)
            if (masks[e]) top.put(key_of(v[e], (int)i0 + e), masks[e]);
        } else {
          // As among many equal values: one by one, sorting where the list is full.
#pragma unroll 1
          for (int e = 0; e < kE; ++e) {
            const float u = i0 + e < c1 ? value<DT>(z, (int)i0 + e) : -kInf;
            top.push(key_of(u, (int)i0 + e), u >= bound);
          }
        }
      }
      // Sorted once so many are there, and then when the list is half full: a bound that is a little old costs less.
      sorted = top.n >= a.n_top && (gate == -kInf || top.n > kList / 2);
      if (sorted) {
        top.sort();
        gate = unorder((uint32_t)(top.least >> 32));
        if (kWaves > 1 && lane == 0) atomicMax(&reached, (uint32_t)(top.least >> 32));
      }
    }
  }

  r = over_wave(r, c);
  if constexpr (kTop) {
    if (!sorted) top.sort();
  }
  if constexpr (kWaves > 1) {
    if (lane == 0) runs[wave] = r, counts[wave] = top.n;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) r = join(r, runs[w], c);
    if constexpr (kTop) {
#pragma unroll 1
      for (int w = 1; w < kWaves; ++w) {
        const bool in = lane < counts[w];
        top.push(in ? lists[w][lane] : 0, in);
      }
      top.sort();
    }
  }
  const int n = top.n;
  if (a.splits == 1) {
    finish<DT>(a, row, r, early, lists[0], n);
    return;
  }
  if (lane == 0) a.stats[row * a.splits + blockIdx.y] = make_float4(r.m, r.s, r.u, 0.f);
  if constexpr (kTop) {
    if (lane < a.n_top) a.keys[(row * a.splits + blockIdx.y) * a.n_top + lane] = lane < n ? lists[0][lane] : 0;
  }
}

// A wave joins a row's chunks: lane l has chunk l's sums and its sorted keys, all lanes' largest, then all second ones...
template <int DT>
__global__ __launch_bounds__(64) void join_kernel(LogProbArgs a) {
  __shared__ __align__(16) uint64_t list[kList];
  const int lane = threadIdx.x;
  const int64_t row = blockIdx.x;
  const bool on = lane < a.splits;
  const Asked early = asked<DT>(a, row);
  const uint64_t* keys = a.keys + (row * a.splits + lane) * a.n_top;
  constexpr int kAhead = 4;                    // keys of a chunk loaded at once
  uint64_t key[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j) key[j] = on && j < a.n_top ? keys[j] : 0;
  Run r = {-kInf, 0.f, 0.f};
  if (on) {
    const float4 s = a.stats[row * a.splits + lane];
    r = {s.x, s.y, s.z};
  }
  r = over_wave(r, a.scale * kLog2E);
  TopList top = {list, 0, a.n_top, 0};
  if (a.n_top) {
    top.start((uint32_t)(key[0] >> 32));
    for (int j0 = 0; j0 < a.n_top; j0 += kAhead) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) top.push(key[j], key[j] != 0);
      if (__ballot(key[kAhead - 1] != 0 && key[kAhead - 1] >= top.least) == 0) break;
#pragma unroll
      for (int j = 0; j < kAhead; ++j) key[j] = on && j0 + kAhead + j < a.n_top ? keys[j0 + kAhead + j] : 0;
    }
    top.sort();
  }
  finish<DT>(a, row, r, early, list, top.n);
}

template <int DT>
hipError_t go(const LogProbArgs& a, hipStream_t st) {
  const dim3 grid(a.rows, a.splits);
  // A wave's work has to be short where few rows wait for it: one load a tile then (the code of a tile is unrolled, and is
  // fetched for one use; one row of 32000 with 5 top values 6.4 us, with four loads 8.5). Many short rows: a wave each, no joining
  // (4000 rows of 2000: 12 us against 22 by four waves; 4096 rows of 32000 with 20 top values 103 and 118, 1024 rows 41 and 31;
  // 16 rows of 131072 in 64 parts of 4 loads of 16 bits 10.1 and 12.9, of 8 in binary32 12.6 and 12.6; 2000 rows of 8000 21.4 and 26.7;
  // 4200 of 16000 62 and 78). The bounds by their number are not the best everywhere: 1100 rows of 8000 20.2 and 18.2, 4000 of 16000 75 by
  // four waves and 60 by one, and rows without top values are up to a fifth slower by one (1100 of 8000 9.3 and 7.6, 4200 of 16000 33 and 29).
  const int64_t pieces = ((int64_t)a.chunk + kPiece<DT> - 1) / kPiece<DT>, groups = (int64_t)a.rows * a.splits;
  const int variant = pieces <= 2 ? 0 : pieces <= (groups >= 4096 ? 64 : groups >= 1024 ? 16 : 0) ? 1 : pieces <= 16 ? 2 : 3;
  if (a.n_top) {
    if (variant == 0) rows_kernel<DT, 64, 1, true><<<grid, 64, 0, st>>>(a);
    else if (variant == 1) rows_kernel<DT, 64, 4, true><<<grid, 64, 0, st>>>(a);
    else if (variant == 2) rows_kernel<DT, 256, 1, true><<<grid, 256, 0, st>>>(a);
    else rows_kernel<DT, 256, 4, true><<<grid, 256, 0, st>>>(a);
  } else {
    if (variant == 0) rows_kernel<DT, 64, 1, false><<<grid, 64, 0, st>>>(a);
    else if (variant == 1) rows_kernel<DT, 64, 4, false><<<grid, 64, 0, st>>>(a);
    else if (variant == 2) rows_kernel<DT, 256, 1, false><<<grid, 256, 0, st>>>(a);
    else rows_kernel<DT, 256, 4, false><<<grid, 256, 0, st>>>(a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  join_kernel<DT><<<a.rows, 64, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

// Rows are cut while they are few: at most one chunk per load of a wave, 64 per row (a lane each in the second launch), about
// 2048 workgroups (128 rows of 131072, 20 top values: 28 us, with 1024 32, 512 30; 300 rows of 32000 17, 21 and 16), from 512
// rows on 1024 (1024 rows of 32000: 31 us uncut, 36 in two).
LogProbPlan log_prob_plan(aqmb_dtype dtype, int rows, int vocab, int n_top) {
  const int unit = dtype == AQMB_F32 ? kPiece<AQMB_F32> : kPiece<AQMB_F16>;
  LogProbPlan p;
  int64_t splits = (rows < 512 ? 2048 : 1024) / rows;
  const int64_t most = ((int64_t)vocab + unit - 1) / unit;
  if (splits > most) splits = most;
  if (splits > 64) splits = 64;
  if (splits < 1) splits = 1;
  int64_t chunk = (vocab + splits - 1) / splits;
  chunk = (chunk + 63) / 64 * 64;                  // chunks start where the row's lines do
  p.chunk = chunk < vocab ? (int)chunk : vocab;
  p.splits = (int)(((int64_t)vocab + p.chunk - 1) / p.chunk);
  p.bytes = p.splits > 1 ? (size_t)rows * p.splits * (16 + 8 * (size_t)n_top) : 0;
  return p;
}

hipError_t launch_log_probs(const LogProbArgs& a, aqmb_dtype dtype, hipStream_t st) {
  return dtype == AQMB_F32 ? go<AQMB_F32>(a, st) : dtype == AQMB_F16 ? go<AQMB_F16>(a, st) : go<AQMB_BF16>(a, st);
}

}  // namespace aqmb
