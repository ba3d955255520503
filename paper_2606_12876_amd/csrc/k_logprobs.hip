// Log probabilities of given tokens, entropy and the largest values of every row of logits, in one pass over them.
//
//   p = 2^t, t = (x - M) scale / log 2,  s = sum p,  u = sum p t,  M the largest x
//   lse = scale M + log s,  log p_t = scale (x_t - M) - log s,  entropy = log s - log 2 u / s
//
// A lane keeps M, s and u of what it has seen and brings them to a new M once per tile. The largest n_top values are
// kept per wave as sorted 64-bit keys (the value's order, then the lower index) in LDS: values above the last of them
// are few once some tiles have passed, so that a tile mostly costs one comparison of its largest value. Few rows are cut
// into chunks, which a second launch joins. Bound by the logits' bytes for many rows, by latency for few.
#include "device.h"
#include "ops.h"
#include "wave.h"

// Products are fused with additions only where that is written: every instance of the kernels rounds alike, whatever
// outputs are asked for.
#pragma clang fp contract(off)

namespace aqmb {

namespace {

struct __attribute__((packed, aligned(2))) Raw16 { uint32_t w[4]; };

constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f, kInf = __builtin_inff();
constexpr float kFar = -1000.f;  // 2^t is 0 there and below: u's factor stays finite
constexpr int kList = 128;       // keys a wave may hold before it sorts: the top ones and a wave's 64 more

template <int DT> constexpr int kEach = DT == AQMB_F32 ? 4 : 8;     // values of a 16-byte load
constexpr int kLoads = 4;                                           // loads of a lane in a tile
template <int DT> constexpr int kTile = 64 * kEach<DT> * kLoads;    // values of a wave's tile

template <int DT>
__device__ __forceinline__ float value(const void* row, int i) {
  if constexpr (DT == AQMB_F32) return ((const float*)row)[i];
  else if constexpr (DT == AQMB_F16) return f16_to_f32(((const uint16_t*)row)[i]);
  else return bf16lo(((const uint16_t*)row)[i]);
}

struct Run { float m, s, u; };
// Both brought to the larger of their maxima; the same whichever comes first, so that all lanes get one result. Of an empty one (m = -infinity) s and u are 0.
__device__ __forceinline__ Run join(const Run& a, const Run& b, float c) {
  const float m = fmaxf(a.m, b.m), ref = m == -kInf ? 0.f : m;
  const float ta = (a.m - ref) * c, tb = (b.m - ref) * c;
  const float fa = __builtin_amdgcn_exp2f(ta), fb = __builtin_amdgcn_exp2f(tb);
  return {m, fa * a.s + fb * b.s, fa * fmaf(fmaxf(ta, kFar), a.s, a.u) + fb * fmaf(fmaxf(tb, kFar), b.s, b.u)};
}
__device__ __forceinline__ Run over_wave(Run r, float c) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int at = 4 * ((threadIdx.x % 64) ^ d);
    const auto from = [&](float x) {
      return __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(at, __builtin_bit_cast(int, x)));
    };
    r = join(r, Run{from(r.m), from(r.s), from(r.u)}, c);
  }
  return r;
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

// The list's n keys sorted, largest first, cut to `top`; the new n. Each key's place is the number of larger ones.
__device__ __forceinline__ int sort_list(uint64_t* list, int n, int top) {
  const int lane = threadIdx.x % 64;
  lds_order();
  const uint64_t a = lane < n ? list[lane] : 0, b = lane + 64 < n ? list[lane + 64] : 0;
  int pa = 0, pb = 0;
  for (int i = 0; i < n; ++i) {
    const uint64_t k = list[i];
    pa += k > a;
    pb += k > b;
  }
  lds_order();
  if (lane < n && pa < top) list[pa] = a;
  if (lane + 64 < n && pb < top) list[pb] = b;
  lds_order();
  return min(n, top);
}

// What a row has come to, by one wave: keys sorted in `sorted`, n of them.
template <int DT>
__device__ __forceinline__ void finish(const LogProbArgs& a, int64_t row, const Run& r, const uint64_t* sorted, int n) {
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
  for (int i = lane; i < a.n_targets; i += 64) {
    const int64_t t = a.targets[row * a.n_targets + i];
    a.logprobs[row * a.n_targets + i] = t < 0 ? 0.f : t >= a.vocab ? nan : log_p(value<DT>(z, (int)t));
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

template <int DT, int NT, bool kTop>
__global__ __launch_bounds__(NT) void rows_kernel(LogProbArgs a) {
  constexpr int kE = kEach<DT>, kN = kE * kLoads, kWaves = NT / 64;
  __shared__ __align__(16) uint64_t lists[kTop ? kWaves : 1][kTop ? kList : 1];
  __shared__ Run runs[kWaves];
  __shared__ int counts[kWaves];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t row = blockIdx.x;
  const char* z = (const char*)a.logits + row * a.stride * (DT == AQMB_F32 ? 4 : 2);
  const int c0 = blockIdx.y * a.chunk, c1 = min(a.vocab - c0, a.chunk) + c0;
  const float c = a.scale * kLog2E;
  uint64_t* list = lists[kTop ? wave : 0];
  int n = 0;                   // keys in the list
  uint64_t least = 0;          // a key has to reach this
  float gate = -kInf;          // a later tile's value has to be above this

  Run r = {-kInf, 0.f, 0.f};
  for (int64_t t0 = c0 + (int64_t)wave * kTile<DT>; t0 < c1; t0 += kWaves * kTile<DT>) {
    float x[kN];
    Raw16 raw[kLoads];
    if (t0 + kTile<DT> <= c1) {
#pragma unroll
      for (int l = 0; l < kLoads; ++l) raw[l] = *(const Raw16*)(z + (t0 + (l * 64 + lane) * kE) * (16 / kE));
#pragma unroll
      for (int l = 0; l < kLoads; ++l)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t w = raw[l].w[j];
          if constexpr (DT == AQMB_F32) {
            x[4 * l + j] = __builtin_bit_cast(float, w);
          } else {
            x[8 * l + 2 * j] = DT == AQMB_F16 ? f16lo(w) : bf16lo(w);
            x[8 * l + 2 * j + 1] = DT == AQMB_F16 ? f16hi(w) : bf16hi(w);
          }
        }
    } else {
#pragma unroll
      for (int e = 0; e < kN; ++e) {
        const int64_t i = t0 + (e / kE * 64 + lane) * kE + e % kE;
        x[e] = i < c1 ? value<DT>(z, (int)i) : -kInf;
      }
    }
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
      if (!__ballot(m > gate)) continue;
      if (least == 0) {
        // As many lanes as top values have a value that reaches the n_top-th largest of the lanes' largest.
        int above = 0;
#pragma unroll
        for (int l = 0; l < 64; ++l) {
          const float o = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, m), l));
          above += o > m || (o == m && l < lane);
        }
        const int at = __builtin_ctzll(__ballot(above == a.n_top - 1));
        least = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)order(m), at) << 32;
      }
#pragma unroll
      for (int e = 0; e < kN; ++e) {
        const uint64_t key = key_of(x[e], (int)(t0 + (e / kE * 64 + lane) * kE + e % kE));
        bool in = x[e] > -kInf && key >= least;
        uint64_t mask = __ballot(in);
        if (mask) {
          if (n + __builtin_popcountll(mask) > kList) {
            n = sort_list(list, n, a.n_top);
            if (n == a.n_top) {
              least = list[n - 1];
              in = in && key >= least;
              mask = __ballot(in);
            }
          }
          if (in) list[n + __builtin_popcountll(mask & ((1ull << lane) - 1))] = key;
          n += __builtin_popcountll(mask);
        }
      }
      if (n >= a.n_top) {
        n = sort_list(list, n, a.n_top);
        least = list[n - 1];
        gate = unorder((uint32_t)(least >> 32));
      }
    }
  }

  r = over_wave(r, c);
  if constexpr (kTop) n = sort_list(list, n, a.n_top);
  if constexpr (kWaves > 1) {
    if (lane == 0) runs[wave] = r, counts[wave] = n;
    __syncthreads();
    r = runs[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) r = join(r, runs[w], c);
    if constexpr (kTop) {
      // Each key's place among all waves'.
      const uint64_t key = lane < n ? list[lane] : 0;
      int place = 0, all = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const int k = counts[w];
        for (int i = 0; i < k; ++i) place += lists[w][i] > key;
        all += k;
      }
      __syncthreads();
      if (lane < n && place < a.n_top) lists[0][place] = key;
      __syncthreads();
      n = min(all, a.n_top);
    }
    if (wave != 0) return;
  }
  if (a.splits == 1) {
    finish<DT>(a, row, r, lists[0], n);
    return;
  }
  if (lane == 0) a.stats[row * a.splits + blockIdx.y] = make_float4(r.m, r.s, r.u, 0.f);
  if constexpr (kTop) {
    if (lane < a.n_top) a.keys[(row * a.splits + blockIdx.y) * a.n_top + lane] = lane < n ? lists[0][lane] : 0;
  }
}

// A wave joins a row's chunks: lane l has chunk l's sums and its keys, of which the largest is taken n_top times.
template <int DT>
__global__ __launch_bounds__(64) void join_kernel(LogProbArgs a) {
  __shared__ uint64_t sorted[64];
  const int lane = threadIdx.x;
  const int64_t row = blockIdx.x;
  const bool on = lane < a.splits;
  Run r = {-kInf, 0.f, 0.f};
  const uint64_t* keys = a.keys + (row * a.splits + lane) * a.n_top;
  uint64_t head = on && a.n_top ? keys[0] : 0;
  if (on) {
    const float4 s = a.stats[row * a.splits + lane];
    r = {s.x, s.y, s.z};
  }
  r = over_wave(r, a.scale * kLog2E);
  int taken = 0, n = 0;
  while (n < a.n_top) {
    uint32_t hi = over_lanes<64>((uint32_t)(head >> 32), max_bits);
    const uint32_t lo = over_lanes<64>((uint32_t)(head >> 32) == hi ? (uint32_t)head : 0, max_bits);
    const uint64_t most = (uint64_t)hi << 32 | lo;
    if (most == 0) break;
    if (head == most) {
      sorted[n] = head;
      ++taken;
      head = taken < a.n_top ? keys[taken] : 0;
    }
    ++n;
  }
  lds_order();
  finish<DT>(a, row, r, sorted, n);
}

template <int DT>
hipError_t go(const LogProbArgs& a, hipStream_t st) {
  const dim3 grid(a.rows, a.splits);
  const bool small = a.chunk <= kTile<DT>;
  if (a.n_top) {
    if (small) rows_kernel<DT, 64, true><<<grid, 64, 0, st>>>(a);
    else rows_kernel<DT, 256, true><<<grid, 256, 0, st>>>(a);
  } else {
    if (small) rows_kernel<DT, 64, false><<<grid, 64, 0, st>>>(a);
    else rows_kernel<DT, 256, false><<<grid, 256, 0, st>>>(a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  join_kernel<DT><<<a.rows, 64, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

LogProbPlan log_prob_plan(aqmb_dtype dtype, int rows, int vocab, int n_top) {
  const int unit = 4 * (dtype == AQMB_F32 ? kTile<AQMB_F32> : kTile<AQMB_F16>);
  LogProbPlan p;
  int64_t splits = 1024 / rows;
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
