// Sampling with temperature, top-k, top-p and min-p from given random numbers
// (wedlm_sample).
//
// One workgroup per row.  What a row keeps is a leading run of its tokens in
// falling order, so it is described by a key (the order-preserving pattern of
// a logit) and a number of ties: tokens above the key, and the first m ids at
// it.  Weights w = 2^((x - max) log2(e) / T) are fp64 values rounded to whole
// multiples of 2^-shift (shift >= 40, so that V of them fit 64 bits): sums
// are exact and the same in any order, which both the histograms' atomics and
// the comparison of running sums with u * total need.
// Passes over a row (the first from HBM, the others from the caches):
//   1. the largest logit;
//   2. with top-k: the logits that can be among the first k, into a list (the
//      parts' maxima of pass 1 bound them from below); with top-p alone: the
//      sum of all weights, and a histogram of the logits near the top.  A
//      histogram (tokens and weights) tells the bins that the ends of top-k's
//      and top-p's runs lie in.  A row whose list does not overflow is not read
//      again.  (If an end lies below the histogram, the pass is done again over
//      all that has a weight.)
//   3. otherwise the weights of the tokens that are surely kept, summed by
//      segments of consecutive ids, and the tokens of the ends' bins collected.
// The exact ends are found among the tokens of their bins: by comparing all
// with all if they are few, else by a radix search over the keys (over the row
// itself where they are too many for LDS, as in a flat row).  Last, one wave
// walks the segment that the draw falls into.
// Bounds, 1280 rows of 151936 fp32 logits: greedy 136 us (HBM, 5.7 TB/s), k = 50
// 191, k = 1000 328 (the second pass), no limit 375 (fp64 weights: 15 fp64
// operations and an LDS read a token), top-p alone 0.68 ms (the histogram's
// 64-bit LDS additions beside that).  bf16 logits: 71, 132, 247, 282 and 587
// us (8 registers of the vectors under way spill).  One row: 8 to 165 us, its
// workgroup's own time; rows are not split over workgroups.
#include "common.h"
#include "wedlm_serve.h"

using namespace wedlm;

namespace {

// (1024 threads: 762 us in place of 669 for 1280 rows with top-p alone, and 125
// in place of 155 for one row)
constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 2048;
constexpr int kSegs = 256;              // segments of a row at most

struct Args {
  const void* x;
  int64_t stride;
  const float* u;
  const int32_t* n_obs;
  const float* temp;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* token;
  float* logp;
  int B, W, V, shift;
  int seg;                // tokens per segment, whole vectors of a wave
};

// Order-preserving pattern of a logit (NaN: -inf; +inf: the largest number).
__device__ __forceinline__ uint32_t key_of(float x) {
  x = x == x ? x : kNegInf;
  x = fminf(x, 3.402823466e38f);
  const uint32_t b = __float_as_uint(x + 0.f);     // -0 counts as 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

constexpr int kNear = 4096;             // tokens near the top
constexpr int kList = 2048;             // tokens of the bins at the runs' ends
constexpr int kPairs = 256;             // of them compared all with all
constexpr int kBlocks = 2 * kList;      // blocks of a row at most
constexpr int kFine = 256;              // steps of the table of powers
// log2 units below the top that the histogram covers, at first and at last:
// 48 units down every weight is zero (shift <= 46)
constexpr float kUnits = 24.f, kAllUnits = 48.f;

// 2^(i / 256), and weights from it: t = k + i / 256 + r, |r| <= 2^-9, with
// 2^r by its series to r^4 (what is left out is below 2^-54).
struct Row {
  double max, rate;       // largest logit; log2(e) / T
  int shift;
  const double* powers;   // LDS
  // weight of a logit, in units of 2^-shift; without a branch: half of the
  // work is here
  __device__ __forceinline__ uint64_t weight(float x) const {
    // 48 units down and more every weight is zero (as is that of -inf, also
    // where the rate is zero)
    const double t =
        __builtin_fmax((static_cast<double>(x) - max) * rate, -48.0);
    constexpr double kMagic = 6755399441055744.0 / kFine;   // 1.5 * 2^52 / 256
    const double y = t + kMagic;
    const int n = static_cast<int>(__double2loint(y));       // round(256 t)
    const double r = t - (y - kMagic);
    double e = 9.618129107628477e-3;                         // ln2^4 / 24
    e = __builtin_fma(e, r, 5.550410866482158e-2);           // ln2^3 / 6
    e = __builtin_fma(e, r, 2.402265069591007e-1);           // ln2^2 / 2
    e = __builtin_fma(e, r, 6.931471805599453e-1);
    e = __builtin_fma(e, r, 1.0);
    e *= powers[n & (kFine - 1)];
    // a whole number below 2^47 by adding 2^52
    const double q = __builtin_amdgcn_ldexp(e, (n >> 8) + shift);
    return static_cast<uint64_t>(__double_as_longlong(q + 4503599627370496.0)) &
           ((1ull << 52) - 1);
  }
};

struct Lds {
  uint64_t sum[kBins];
  uint32_t count[kBins];
  uint64_t near[kNear];   // key << 32 | ~id: larger is earlier in the order
  union {
    uint64_t list[kList];
    float blocks[2 * kList];   // largest logit of each (before the list)
  };
  uint64_t weights[kPairs];
  double powers[kFine];
  uint64_t part[kWaves];
  uint64_t found_before, found_ties;
  uint32_t found, nears, listed, low, tied;
};

// A logit as it counts: NaN: -inf; +inf: the largest number.
__device__ __forceinline__ float clean(float x) {
  return fminf(fmaxf(x, kNegInf), 3.402823466e38f);
}

// Largest of a value over the wave, in lane 63: rows of 16 lanes shifted by 1,
// 2, 4 and 8, then lane 15 of each row to the next row and lane 31 to the upper
// half.
template <int CTRL>
__device__ __forceinline__ float dpp_top(float v) {
  const int x = __float_as_int(v);
  return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(x, x, CTRL, 0xf,
                                                             0xf, false)));
}
__device__ __forceinline__ float wave_top(float v) {
  v = dpp_top<0x118>(dpp_top<0x114>(dpp_top<0x112>(dpp_top<0x111>(v))));
  return dpp_top<0x143>(dpp_top<0x142>(v));
}

// Appends e of the lanes that call it to a list of `most`; false if it is
// full, with its length then beyond that.
__device__ __forceinline__ bool push(uint64_t* list, uint32_t* n, uint32_t most,
                                     uint64_t e) {
  const uint64_t m = ballot(true);
  const int lead = __ffsll(static_cast<unsigned long long>(m)) - 1;
  uint32_t at = 0;
  if (lane_id() == lead)
    at = atomicAdd(n, static_cast<uint32_t>(__popcll(m)));
  at = __shfl(at, lead) + __popcll(m & ((1ull << lane_id()) - 1));
  if (at < most) list[at] = e;
  return at < most;
}

__device__ __forceinline__ uint64_t entry(float x, int id) {
  return static_cast<uint64_t>(key_of(x)) << 32 |
         static_cast<uint32_t>(~static_cast<uint32_t>(id));
}

// Sum over the workgroup, to all threads.
__device__ __forceinline__ uint64_t group_sum(uint64_t v, uint64_t* part) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1)
    v += __shfl_xor(static_cast<unsigned long long>(v), off);
  __syncthreads();
  if (lane_id() == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  uint64_t all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) all += part[w];
  return all;
}

// Exclusive sums over the workgroup; `total` to all threads.
__device__ __forceinline__ uint64_t group_scan(uint64_t v, uint64_t* part,
                                               uint64_t& total) {
  const int wave = threadIdx.x / kWave, lane = lane_id();
  uint64_t s = v;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const uint64_t o = __shfl_up(static_cast<unsigned long long>(s), off);
    if (lane >= off) s += o;
  }
  __syncthreads();
  if (lane == kWave - 1) part[wave] = s;
  __syncthreads();
  uint64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const uint64_t t = part[w];
    before += w < wave ? t : 0;
    all += t;
  }
  total = all;
  return before + s - v;
}

// The first bin, in the order of `bin_at` (place 0 .. kBins-1 -> bin), at
// which the running sum of `value` reaches `want` (>= 1); `before` gets the
// sum ahead of it.  kBins if the sum of all is less.
template <typename F, typename G>
__device__ __forceinline__ uint32_t find_bin(Lds& l, F value, G bin_at,
                                             uint64_t want, uint64_t& before) {
  constexpr int N = kBins / kThreads;
  const int p0 = N * static_cast<int>(threadIdx.x);
  uint64_t v[N], own = 0;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v[k] = value(bin_at(p0 + k));
    own += v[k];
  }
  uint64_t total;
  uint64_t at = group_scan(own, l.part, total);
  if (threadIdx.x == 0 && total < want) {
    l.found = kBins;
    l.found_before = total;
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if (at < want && at + v[k] >= want) {
      l.found = bin_at(p0 + k);
      l.found_before = at;
    }
    at += v[k];
  }
  __syncthreads();
  before = l.found_before;
  return l.found;
}

// The logits of a row: `head` of them before the first 16-byte boundary, then
// vectors.
template <bool HALF>
struct Logits {
  static constexpr int VEC = HALF ? 8 : 4;
  const void* x;
  int V, head;

  __device__ __forceinline__ float one(int i) const {
    if constexpr (HALF) return bf16_to_f32(static_cast<const uint16_t*>(x)[i]);
    else return static_cast<const float*>(x)[i];
  }
  __device__ __forceinline__ void many(int i, float (&f)[VEC]) const {
    if constexpr (HALF) {
      const u16x8_t v = *reinterpret_cast<const u16x8_t*>(
          static_cast<const uint16_t*>(x) + i);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = bf16_to_f32(v[k]);
    } else {
      const floatx4_t v = *reinterpret_cast<const floatx4_t*>(
          static_cast<const float*>(x) + i);
#pragma unroll
      for (int k = 0; k < 4; ++k) f[k] = v[k];
    }
  }
  // f(logits, first id) of all tokens, over the workgroup: vectors, the next
  // AHEAD under way, and single tokens at the ends
  template <int AHEAD, typename F>
  __device__ __forceinline__ void each(F f) const {
    const int tid = threadIdx.x;
    if (tid < head) {
      const float s[1] = {one(tid)};
      f(s, tid);
    }
    constexpr int kStep = kThreads * VEC;
    int i = head + tid * VEC;
    if (i + VEC <= V) {
      const int last = i + (V - VEC - i) / kStep * kStep;
      float v[AHEAD + 1][VEC];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) many(min(i + u * kStep, last), v[u]);
      for (; i <= last; i += kStep) {
        many(min(i + AHEAD * kStep, last), v[AHEAD]);
        f(v[0], i);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
          for (int k = 0; k < VEC; ++k) v[u][k] = v[u + 1][k];
      }
    }
    for (int k = i; k < V && k < i + VEC; ++k) {
      const float s[1] = {one(k)};
      f(s, k);
    }
  }
  // Rounds of the workgroup's whole vectors, and the rounds of one block: a
  // block is a wave's vectors of `fold` rounds in a row, as many blocks as fit.
  __device__ __forceinline__ int rounds() const {
    return (V - head) / VEC / kThreads +
           ((V - head) / VEC % kThreads != 0 ? 1 : 0);
  }
  __device__ __forceinline__ int fold() const {
    return (rounds() * kWaves + kBlocks - 1) / kBlocks;
  }
  // The largest logits that this thread meets, by their place in a vector, and
  // if wanted of each block (blocks[block round * kWaves + wave]); four vectors
  // under way.  What is not in whole vectors counts in m alone.
  template <bool BLOCKS>
  __device__ __forceinline__ void largest(float (&m)[VEC], float* blocks) const {
    const int tid = threadIdx.x, n = rounds(), f = fold();
#pragma unroll
    for (int k = 0; k < VEC; ++k) m[k] = kNegInf;
    if (tid < head) m[0] = fmaxf(m[0], one(tid));
    constexpr int kStep = kThreads * VEC;
    float top = kNegInf;
    int left = f, block = tid / kWave;
    auto round = [&](const float (&v)[VEC], bool whole) {
      float t = kNegInf;
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        m[k] = fmaxf(m[k], whole ? v[k] : kNegInf);
        t = fmaxf(t, v[k]);
      }
      top = fmaxf(top, whole ? t : kNegInf);
      if (BLOCKS && --left == 0) {
        top = wave_top(top);
        if (lane_id() == kWave - 1) blocks[block] = top;
        top = kNegInf;
        left = f;
        block += kWaves;
      }
    };
    int i = head + tid * VEC, j = 0;
    for (; j + 4 <= n && i - tid * VEC + 4 * kStep <= V; j += 4, i += 4 * kStep) {
      float v[4][VEC];
#pragma unroll
      for (int u = 0; u < 4; ++u) many(i + u * kStep, v[u]);
      if (BLOCKS && f == 1) {
        // (four reductions side by side)
        float t[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          t[u] = kNegInf;
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            m[k] = fmaxf(m[k], v[u][k]);
            t[u] = fmaxf(t[u], v[u][k]);
          }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) t[u] = wave_top(t[u]);
        if (lane_id() == kWave - 1)
#pragma unroll
          for (int u = 0; u < 4; ++u) blocks[block + u * kWaves] = t[u];
        block += 4 * kWaves;
        continue;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) round(v[u], true);
    }
    for (; j < n; ++j, i += kStep) {
      const bool whole = i + VEC <= V;
      float v[VEC];
#pragma unroll
      for (int k = 0; k < VEC; ++k) v[k] = kNegInf;
      if (whole) many(i, v);
      round(v, whole);
    }
    if (BLOCKS && left < f) {
      top = wave_top(top);
      if (lane_id() == kWave - 1) blocks[block] = top;
    }
    // the last, not whole, vector is the one after all whole ones
    const int rest = head + (V - head) / VEC * VEC + tid;
    if (rest < V) m[0] = fmaxf(m[0], one(rest));
  }
  // f(logits, first id) of the blocks that want(largest) says, each by the wave
  // that has it, and of the tokens that are in no whole vector
  template <typename W, typename F>
  __device__ __forceinline__ void each_block(const float* blocks, W want,
                                             F f) const {
    const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave;
    const int n = rounds(), fo = fold();
    const int mine = (n + fo - 1) / fo;        // block rounds
    for (int b0 = 0; b0 < mine; b0 += kWave) {
      uint64_t todo = ballot(b0 + lane < mine &&
                             want(blocks[(b0 + lane) * kWaves + wave]));
      while (todo) {
        const int b = b0 + __ffsll(static_cast<unsigned long long>(todo)) - 1;
        todo &= todo - 1;
        for (int j = b * fo; j < min((b + 1) * fo, n); ++j) {
          const int i = head + (j * kThreads + tid) * VEC;
          if (i + VEC <= V) {
            float v[VEC];
            many(i, v);
            f(v, i);
          }
        }
      }
    }
    const int rest = head + (V - head) / VEC * VEC + tid;
    if (tid < head || rest < V) {
      if (tid < head) {
        const float s[1] = {one(tid)};
        f(s, tid);
      }
      if (rest < V) {
        const float s[1] = {one(rest)};
        f(s, rest);
      }
    }
  }
};

// f of each of N values
template <int N, typename F>
__device__ __forceinline__ void one_by_one(const float (&v)[N], int id, F f) {
#pragma unroll
  for (int k = 0; k < N; ++k) f(v[k], id + k);
}

// Digits of a radix search: bits [down, up) of the key.
__device__ __forceinline__ int digit_up(int level) {
  return level == 0 ? 32 : level == 1 ? 21 : 10;
}
__device__ __forceinline__ int digit_down(int level) {
  return level == 0 ? 21 : level == 1 ? 10 : 0;
}
__device__ __forceinline__ bool in_prefix(uint32_t key, uint32_t prefix,
                                          int level) {
  return level == 0 || key >> digit_up(level) == prefix >> digit_up(level);
}
__device__ __forceinline__ int digit_of(uint32_t key, int level) {
  return (key >> digit_down(level)) &
         ((1u << (digit_up(level) - digit_down(level))) - 1);
}

// Key of the want-th largest of the tokens that each(f) visits (f(key)), and
// how many of its ties are among the first `want`.
template <typename E>
__device__ __forceinline__ void kth_key(Lds& l, E each, uint64_t want,
                                        uint32_t& key, uint32_t& ties) {
  uint32_t prefix = 0;
  for (int level = 0; level < 3; ++level) {
    __syncthreads();
    for (int j = threadIdx.x; j < kBins; j += kThreads) l.count[j] = 0;
    __syncthreads();
    each([&](uint32_t k) {
      if (in_prefix(k, prefix, level)) atomicAdd(&l.count[digit_of(k, level)], 1u);
    });
    __syncthreads();
    uint64_t before;
    prefix |= find_bin(
                  l, [&](int j) { return static_cast<uint64_t>(l.count[j]); },
                  [](int p) { return kBins - 1 - p; }, want, before)
              << digit_down(level);
    want -= before;
  }
  key = prefix;
  ties = static_cast<uint32_t>(want);
}

// Key at which the weights of the tokens above kkey, with the first kties ties
// at it, reach `want` in falling order, and how many of its ties that takes.
template <typename E>
__device__ __forceinline__ void pth_key(Lds& l, const Row& r, E each,
                                        uint32_t kkey, uint32_t kties,
                                        uint64_t want, uint32_t& key,
                                        uint32_t& ties) {
  uint32_t prefix = 0;
  for (int level = 0; level < 3; ++level) {
    __syncthreads();
    for (int j = threadIdx.x; j < kBins; j += kThreads) l.sum[j] = 0;
    __syncthreads();
    each([&](uint32_t k) {
      if (k > kkey && in_prefix(k, prefix, level)) {
        const uint64_t q = r.weight(of_key(k));
        if (q)
          atomicAdd(reinterpret_cast<unsigned long long*>(
                        &l.sum[digit_of(k, level)]),
                    static_cast<unsigned long long>(q));
      }
    });
    __syncthreads();
    if (threadIdx.x == 0 && kkey != 0 && in_prefix(kkey, prefix, level))
      l.sum[digit_of(kkey, level)] += kties * r.weight(of_key(kkey));
    __syncthreads();
    uint64_t before;
    prefix |= find_bin(l, [&](int j) { return l.sum[j]; },
                       [](int p) { return kBins - 1 - p; }, want, before)
              << digit_down(level);
    want -= before;
  }
  key = prefix;
  const uint64_t q = r.weight(of_key(key));
  ties = static_cast<uint32_t>((want + q - 1) / q);
}

// The least whole number >= p * total, one at least (0 <= p < 1).
__device__ __forceinline__ uint64_t share(double p, uint64_t total) {
  const uint64_t f = static_cast<uint64_t>(ldexp(p, 63)) << 1;
  const uint64_t s = __umul64hi(total, f) + (total * f != 0 ? 1 : 0);
  return s < 1 ? 1 : s;
}

// (registers for two workgroups a CU: one's barriers and short searches run
// under the other's passes)
template <bool HALF>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(4))) void sample_kernel(Args a) {
  __shared__ Lds l;
  // neighbours take rows of different sequences: settings, and so the rows'
  // times, go by sequence
  const int row = blockIdx.x, b = row / a.W, i = row - b * a.W;
  if (a.n_obs && i < a.n_obs[b]) return;
  Logits<HALF> x;
  constexpr int VEC = Logits<HALF>::VEC;
  if constexpr (HALF)
    x.x = static_cast<const uint16_t*>(a.x) + row * a.stride;
  else
    x.x = static_cast<const float*>(a.x) + row * a.stride;
  const int V = a.V, tid = threadIdx.x, lane = lane_id();
  const int wave = tid / kWave;
  x.V = V;
  x.head = min(V, static_cast<int>((-reinterpret_cast<uintptr_t>(x.x) & 15) /
                                   (16 / VEC)));

  // ---- the largest logit
  if (tid < kFine) l.powers[tid] = exp2(tid / static_cast<double>(kFine));
  float some[VEC];        // the largest of kThreads * VEC parts of the row
  const float T = a.temp ? a.temp[b] : 1.f;
  const int k_raw = a.top_k ? a.top_k[b] : 0;
  // with few k the blocks' maxima too (1280 rows of 151936, k = 50: 189 us with
  // them, 281 without; other rows' first pass takes up to 7 us longer with them)
  const int blocks = (x.rounds() + x.fold() - 1) / max(x.fold(), 1) * kWaves;
  const bool few = T > 0.f && k_raw > 0 && k_raw < V && k_raw <= blocks / 4;
  if (few) x.template largest<true>(some, l.blocks);
  else x.template largest<false>(some, l.blocks);
  float fmax_ = some[0];
#pragma unroll
  for (int k = 1; k < VEC; ++k) fmax_ = fmaxf(fmax_, some[k]);
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1)
    fmax_ = fmaxf(fmax_, __shfl_xor(fmax_, off));
  if (tid == 0) {
    l.nears = 0;
    l.listed = 0;
    l.low = 0xffffffffu;
    l.tied = 0;
  }
  if (lane == 0) l.part[wave] = __float_as_uint(fmax_);
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w)
    fmax_ = fmaxf(fmax_, __uint_as_float(static_cast<uint32_t>(l.part[w])));
  fmax_ = clean(fmax_);
  if (!(T > 0.f) || fmax_ == kNegInf) {
    // its first id: among the parts that it is the maximum of, a thread per
    // vector, and the ends; over the whole row if it is that of many
    uint32_t first = 0xffffffffu;
#pragma unroll
    for (int k = 0; k < VEC; ++k)
      if (clean(some[k]) == fmax_)
        push(l.list, &l.listed, kPairs, static_cast<uint64_t>(tid * VEC + k));
    __syncthreads();
    const int n = static_cast<int>(l.listed);
    auto look = [&](int v) {
      if (v >= 0 && v < V && clean(x.one(v)) == fmax_)
        first = min(first, static_cast<uint32_t>(v));
    };
    if (n <= kPairs) {
      for (int j = 0; j < n; ++j)
        for (int v = x.head + static_cast<int>(l.list[j]) + tid * kThreads * VEC;
             v < V; v += kThreads * kThreads * VEC)
          look(v);
      if (tid < VEC) {
        if (tid < x.head) look(tid);
        look(V - 1 - tid);
      }
    } else {
      x.template each<1>([&](const auto& f, int v) {
        one_by_one(f, v, [&](float, int id) { look(id); });
      });
    }
    if (first != 0xffffffffu) atomicMin(&l.low, first);
    __syncthreads();
    if (tid == 0) {
      a.token[row] = static_cast<int>(l.low);
      if (a.logp) a.logp[row] = 0.f;
    }
    return;
  }
  Row r;
  r.max = fmax_;
  r.rate = 1.4426950408889634 / static_cast<double>(T);
  r.shift = a.shift;
  r.powers = l.powers;
  bool use_k = k_raw > 0 && k_raw < V;
  const float p = a.top_p ? a.top_p[b] : 1.f;
  bool use_p = p < 1.f;
  const double pd = p > 0.f ? static_cast<double>(p) : 0.0;
  const float least = a.min_p ? a.min_p[b] : 0.f;
  uint64_t qmin = 1;
  if (least > 0.f) {
    const double m = least < 1.f ? static_cast<double>(least) : 1.0;
    const uint64_t q = static_cast<uint64_t>(rint(ldexp(m, r.shift)));
    qmin = q > 1 ? q : 1;
  }

  // ---- the bins of the runs' ends: bins lo .. hi and kb, those below lo are
  // kept whole
  int lo = kBins, hi = kBins - 1, kb = -1;
  uint64_t k_left = 0, k_above = 0;     // tokens of bin kb; weights above it
  uint64_t p_above = 0;                 // weights above bin lo
  float rate = 0.f;
  // (fmax_ - f) * rate / 2: falls with the logit, so bins are in the order of
  // the keys; -inf has none.  Half of each, since the difference of two fp32
  // numbers can pass the largest one: a token would have a weight and no bin
  // where T is that large too.
  const float half = 0.5f * fmax_;
  auto place = [&](float f) { return __builtin_fmaf(-0.5f, f, half) * rate; };
  auto rate_of = [&](float units) {
    return static_cast<float>(fmin(r.rate * (kBins / units), 1e30) * 2.0);
  };
  auto bin_of = [&](uint32_t key) {
    return static_cast<int>(fminf(place(of_key(key)), 1e6f));
  };
  auto same = [](int j) { return j; };
  auto counts = [&](int j) { return static_cast<uint64_t>(l.count[j]); };
  auto sums = [&](int j) { return l.sum[j]; };
  auto clear = [&]() {
    for (int j = tid; j < kBins; j += kThreads) {
      l.sum[j] = 0;
      l.count[j] = 0;
    }
    if (tid == 0) l.nears = 0;
    __syncthreads();
  };
  // From the bins' counts and weights (`all`: this thread's part of the weight
  // of all tokens): true if an end lies below the bins; never with `last`, so
  // that the passes end whatever the bins hold.
  auto locate = [&](uint64_t all, bool last) {
    if (use_k) {
      uint64_t before;
      const uint32_t f =
          find_bin(l, counts, same, static_cast<uint64_t>(k_raw), before);
      if (f < kBins) {
        kb = static_cast<int>(f);
        k_left = k_raw - before;
      } else if (last) {
        use_k = false;                  // fewer than k have a weight: no limit
      } else {
        return true;
      }
    }
    if (use_p) {
      // what top-k leaves weighs at least the bins above kb, at most kb too
      uint64_t most;
      if (kb < 0) {
        most = group_sum(all, l.part);
        k_above = most;
      } else {
        uint64_t part = 0;
        for (int j = tid; j <= kb; j += kThreads) part += l.sum[j];
        most = group_sum(part, l.part);
        k_above = most - l.sum[kb];
      }
      const uint32_t f = find_bin(l, sums, same, share(pd, k_above), p_above);
      if (f < kBins) {
        lo = hi = static_cast<int>(f);
        if (kb >= 0) {
          uint64_t before;
          hi = static_cast<int>(
              find_bin(l, sums, same, share(pd, most), before));
        }
        return false;
      }
      if (!last) return true;
      use_p = false;                    // what has no bin then has no weight
    }
    if (kb >= 0) lo = hi = kb;
    return false;
  };
  bool placed = false;
  if (use_k && k_raw <= kThreads * VEC / 2) {
    // The k-th largest of the parts' maxima is not above the k-th largest
    // logit, and mostly near it: what is above its bin is collected.  With few
    // k the parts are the blocks, and only those with something are read again.
    rate = rate_of(kAllUnits);
    clear();
    auto mark = [&](float f) {
      const float at = place(clean(f));
      if (at < static_cast<float>(kBins))
        atomicAdd(&l.count[static_cast<int>(at)], 1u);
    };
    if (few) {
      for (int j = tid; j < blocks; j += kThreads) mark(l.blocks[j]);
    } else {
#pragma unroll
      for (int k = 0; k < VEC; ++k) mark(some[k]);
    }
    __syncthreads();
    uint64_t before;
    const uint32_t f =
        find_bin(l, counts, same, static_cast<uint64_t>(k_raw), before);
    if (f < kBins) {
      const float most = static_cast<float>(f + 1);
      bool room = true;
      auto take = [&](const auto& g, int v) {
        // (one question for a vector: few have any)
        constexpr int N = sizeof(g) / sizeof(float);
        float top = kNegInf;
#pragma unroll
        for (int k = 0; k < N; ++k) top = fmaxf(top, g[k]);
        if (!(place(clean(top)) < most) || !room) return;
        one_by_one(g, v, [&](float h, int id) {
          if (place(clean(h)) < most && room)
            room = push(l.near, &l.nears, kNear, entry(h, id));
        });
      };
      if (few)
        x.each_block(l.blocks,
                     [&](float top) { return place(clean(top)) < most; }, take);
      else
        x.template each<4>(take);
      __syncthreads();
      const uint32_t n = l.nears;
      if (n <= kNear) {
        __syncthreads();
        clear();
        for (uint32_t j = tid; j < n; j += kThreads) {
          const uint32_t k = static_cast<uint32_t>(l.near[j] >> 32);
          const int bin = bin_of(k);
          atomicAdd(&l.count[bin], 1u);
          if (use_p)
            atomicAdd(reinterpret_cast<unsigned long long*>(&l.sum[bin]),
                      static_cast<unsigned long long>(r.weight(of_key(k))));
        }
        if (tid == 0) l.nears = n;
        __syncthreads();
        locate(0, true);
        placed = true;
      }
    }
    __syncthreads();
  }
  for (float units = kUnits; !placed && (use_k || use_p); units = kAllUnits) {
    rate = rate_of(units);
    clear();
    uint64_t all = 0;
    bool room = true;                   // in the list, as far as this wave saw
    x.template each<2>([&](const auto& f, int v) {
      constexpr int N = sizeof(f) / sizeof(float);
      // weights of a vector side by side: each is a chain of fp64 operations
      // and an LDS read
      uint64_t q[N] = {};
      if (use_p) {
#pragma unroll
        for (int k = 0; k < N; ++k) q[k] = r.weight(clean(f[k]));
#pragma unroll
        for (int k = 0; k < N; ++k) all += q[k];
      }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float at = place(clean(f[k]));
        if (at < static_cast<float>(kBins)) {
          const int bin = static_cast<int>(at);
          if (use_k) atomicAdd(&l.count[bin], 1u);
          if (use_p)
            atomicAdd(reinterpret_cast<unsigned long long*>(&l.sum[bin]),
                      static_cast<unsigned long long>(q[k]));
          if (room) room = push(l.near, &l.nears, kNear, entry(f[k], v + k));
        }
      }
    });
    __syncthreads();
    placed = !locate(all, units == kAllUnits);
    __syncthreads();
  }

  // ---- sums of each segment: what is above the ends' bins; those bins' tokens
  // into the list.  Segment s is seg tokens from head + s * seg on, the first
  // has the head too.
  const int seg = a.seg;
  const int nseg = max(1, (V - x.head + seg - 1) / seg);
  uint32_t tkey = 0, ties = 0;
  const bool ends = use_k || use_p;
  auto in_list = [&](int bin) { return (bin >= lo && bin <= hi) || bin == kb; };
  auto segment_of = [&](int v) { return max(v - x.head, 0) / seg; };
  auto id_of = [](uint64_t e) {
    return static_cast<int>(~static_cast<uint32_t>(e));
  };
  if (ends && l.nears <= kNear) {
    // all that can be kept is in LDS
    if (tid < kSegs) l.sum[tid] = 0;
    __syncthreads();
    for (uint32_t j = tid; j < l.nears; j += kThreads) {
      const uint64_t e = l.near[j];
      const uint32_t k = static_cast<uint32_t>(e >> 32);
      const int bin = bin_of(k);
      if (in_list(bin)) push(l.list, &l.listed, kList, e);
      if (bin >= lo) continue;
      const uint64_t q = r.weight(of_key(k));
      if (q >= qmin)
        atomicAdd(reinterpret_cast<unsigned long long*>(
                      &l.sum[segment_of(id_of(e))]),
                  static_cast<unsigned long long>(q));
    }
  } else {
    for (int s = wave; s < nseg; s += kWaves) {
      uint64_t sum = 0;
      auto take = [&](const auto& f, int v) {
        constexpr int N = sizeof(f) / sizeof(float);
        bool whole[N], any = !ends;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          whole[k] = true;
          if (ends) {
            const float at = place(clean(f[k]));
            whole[k] = at < static_cast<float>(lo);
            any = any || whole[k];
            if (!whole[k] && at < static_cast<float>(kBins) &&
                in_list(static_cast<int>(at)))
              push(l.list, &l.listed, kList, entry(f[k], v + k));
          }
        }
        if (!any) return;
        uint64_t q[N];
#pragma unroll
        for (int k = 0; k < N; ++k) q[k] = r.weight(clean(f[k]));
#pragma unroll
        for (int k = 0; k < N; ++k)
          sum += whole[k] && (qmin == 1 || q[k] >= qmin) ? q[k] : 0;
      };
      if (s == 0 && lane < x.head) {
        const float f[1] = {x.one(lane)};
        take(f, lane);
      }
      const int end = min(V, x.head + (s + 1) * seg);
      int v = x.head + s * seg + lane * VEC;
      for (; v + VEC <= end; v += kWave * VEC) {
        float f[VEC];
        x.many(v, f);
        take(f, v);
      }
      for (int k = v; k < end && k < v + VEC; ++k) {
        const float f[1] = {x.one(k)};
        take(f, k);
      }
      if (ballot(sum != 0)) {
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1)
          sum += __shfl_xor(static_cast<unsigned long long>(sum), off);
      }
      if (lane == 0) l.sum[s] = sum;
    }
  }
  __syncthreads();

  if (ends) {
    const int n = static_cast<int>(l.listed);
    const bool small = n <= kList;
    // the sums by segment wait in registers while the searches use the bins
    const uint64_t mine = tid < nseg ? l.sum[tid] : 0;
    if (n <= kPairs) {
      // a thread per token, which compares itself with all of them
      uint64_t e = 0, q = 0;
      bool kept = tid < n;
      if (kept) {
        e = l.list[tid];
        const uint32_t k = static_cast<uint32_t>(e >> 32);
        q = r.weight(of_key(k));
        if (kb >= 0 && bin_of(k) == kb) {
          uint64_t rank = 0;
          for (int j = 0; j < n; ++j)
            rank += l.list[j] > e &&
                            bin_of(static_cast<uint32_t>(l.list[j] >> 32)) == kb
                        ? 1 : 0;
          kept = rank < k_left;
        }
      }
      if (use_p) {
        const bool at_kb =
            kept && kb >= 0 && bin_of(static_cast<uint32_t>(e >> 32)) == kb;
        const uint64_t total =
            k_above + (kb >= 0 ? group_sum(at_kb ? q : 0, l.part) : 0);
        if (tid < n) l.weights[tid] = kept ? q : 0;
        __syncthreads();
        if (kept) {
          uint64_t before = 0;
          for (int j = 0; j < n; ++j) before += l.list[j] > e ? l.weights[j] : 0;
          kept = before < share(pd, total) - p_above;
        }
      }
      // the last kept key and its kept ties
      if (kept) atomicMin(&l.low, static_cast<uint32_t>(e >> 32));
      __syncthreads();
      tkey = l.low;
      if (kept && static_cast<uint32_t>(e >> 32) == tkey) atomicAdd(&l.tied, 1u);
      __syncthreads();
      ties = l.tied;
    } else {
      auto list_keys = [&](auto f) {
        for (int j = tid; j < n; j += kThreads)
          f(static_cast<uint32_t>(l.list[j] >> 32));
      };
      auto row_keys = [&](auto f) {
        x.template each<1>([&](const auto& g, int v) {
          one_by_one(g, v, [&](float h, int) { f(key_of(h)); });
        });
      };
      uint32_t kkey = 0, kties = 0;
      if (kb >= 0) {
        if (small)
          kth_key(l, [&](auto f) {
            list_keys([&](uint32_t k) { if (bin_of(k) == kb) f(k); });
          }, k_left, kkey, kties);
        else
          kth_key(l, row_keys, static_cast<uint64_t>(k_raw), kkey, kties);
        tkey = kkey;
        ties = kties;
      }
      if (use_p) {
        // the weight of all that top-k left
        uint64_t total = 0;
        if (kb >= 0) {
          auto add = [&](uint32_t k) {
            if (k > kkey && bin_of(k) == kb) total += r.weight(of_key(k));
          };
          if (small) list_keys(add);
          else row_keys(add);
          total = group_sum(total, l.part) + kties * r.weight(of_key(kkey));
        }
        total += k_above;
        const uint64_t want = share(pd, total);
        if (small)
          pth_key(l, r, list_keys, kkey, kties, want - p_above, tkey, ties);
        else
          pth_key(l, r, row_keys, kkey, kties, want, tkey, ties);
      }
    }
    // the kept tokens of the ends' bins, and the ties of each segment
    __syncthreads();
    if (tid < kSegs) {
      l.sum[tid] = mine;
      l.count[tid] = 0;
    }
    __syncthreads();
    auto keep = [&](uint32_t k, int v) {
      if (k < tkey || !in_list(bin_of(k))) return;
      if (k == tkey) {
        atomicAdd(&l.count[segment_of(v)], 1u);
        return;
      }
      const uint64_t q = r.weight(of_key(k));
      if (q >= qmin)
        atomicAdd(reinterpret_cast<unsigned long long*>(&l.sum[segment_of(v)]),
                  static_cast<unsigned long long>(q));
    };
    if (small) {
      for (int j = tid; j < n; j += kThreads)
        keep(static_cast<uint32_t>(l.list[j] >> 32), id_of(l.list[j]));
    } else {
      x.template each<1>([&](const auto& f, int v) {
        one_by_one(f, v, [&](float g, int id) { keep(key_of(g), id); });
      });
    }
    __syncthreads();
  }

  // ---- the draw
  uint64_t qt = ends ? r.weight(of_key(tkey)) : 0;
  qt = qt >= qmin ? qt : 0;
  uint64_t total;
  const uint32_t tied = ends && tid < nseg ? l.count[tid] : 0;
  const uint64_t ties_before = group_scan(tied, l.part, total);
  const uint64_t left = ties > ties_before ? ties - ties_before : 0;
  const uint64_t own = (tid < nseg ? l.sum[tid] : 0) +
                       qt * (left < tied ? left : tied);
  const uint64_t before = group_scan(own, l.part, total);
  float u = a.u[row];
  u = u > 0.f ? (u < 1.f ? u : 0.99999994f) : 0.f;
  const uint64_t goal =
      __umul64hi(total, static_cast<uint64_t>(ldexp(static_cast<double>(u), 63))
                            << 1);
  if (before <= goal && before + own > goal) {
    l.found = tid;
    l.found_before = before;
    l.found_ties = ties_before;
  }
  __syncthreads();
  if (wave != 0) return;
  // ---- the segment that holds the drawn token, one wave, a run of ids a lane
  const int s = l.found;
  const int begin = s == 0 ? 0 : x.head + s * seg;
  const int end = min(V, x.head + (s + 1) * seg);
  const int per = (end - begin + kWave - 1) / kWave;
  const int v0 = min(begin + lane * per, end), v1 = min(v0 + per, end);
  uint64_t sum = 0;
  uint32_t mine = 0;
  for (int v = v0; v < v1; ++v) {
    const uint32_t k = key_of(x.one(v));
    mine += ends && k == tkey ? 1 : 0;
    const uint64_t q = k > tkey ? r.weight(of_key(k)) : 0;
    sum += q >= qmin ? q : 0;
  }
  uint64_t seen = mine;                 // ties up to this lane's last
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const uint64_t o = __shfl_up(static_cast<unsigned long long>(seen), off);
    if (lane >= off) seen += o;
  }
  seen += l.found_ties - mine;          // ties before its first
  uint64_t rest = ties > seen ? ties - seen : 0;
  sum += qt * (rest < mine ? rest : mine);
  uint64_t run = sum;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const uint64_t o = __shfl_up(static_cast<unsigned long long>(run), off);
    if (lane >= off) run += o;
  }
  run += l.found_before - sum;          // weights before its first
  if (!(run <= goal && run + sum > goal)) return;
  for (int v = v0; v < v1; ++v) {
    const uint32_t k = key_of(x.one(v));
    uint64_t q = 0;
    if (k > tkey) {
      q = r.weight(of_key(k));
      q = q >= qmin ? q : 0;
    } else if (ends && k == tkey && rest > 0) {
      q = qt;
      --rest;
    }
    run += q;
    if (run > goal) {
      a.token[row] = v;
      if (a.logp)
        a.logp[row] = static_cast<float>(
            (static_cast<double>(of_key(k)) - r.max) / static_cast<double>(T) -
            log(ldexp(static_cast<double>(total), -r.shift)));
      return;
    }
  }
}

}  // namespace

extern "C" int wedlm_sample(const void* logits, int32_t logits_type,
                            int64_t row_stride, const float* u,
                            const int32_t* n_obs, const float* temperature,
                            const int32_t* top_k, const float* top_p,
                            const float* min_p, int32_t B, int32_t W,
                            int32_t V, int32_t* token, float* logp,
                            void* stream) {
  if (!logits || !u || !token) return WEDLM_E_ARG;
  if (logits_type != WEDLM_SAMPLE_F32 && logits_type != WEDLM_SAMPLE_BF16)
    return WEDLM_E_ARG;
  if (B < 1 || W < 1 || V < 1 || V > (1 << 22) || row_stride < V)
    return WEDLM_E_SHAPE;
  const int64_t rows = static_cast<int64_t>(B) * W;
  if (rows >= (1ll << 22)) return WEDLM_E_SHAPE;   // one launch's threads
  Args a{};
  a.x = logits; a.stride = row_stride; a.u = u; a.n_obs = n_obs;
  a.temp = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p;
  a.token = token; a.logp = logp; a.B = B; a.W = W; a.V = V;
  // V weights of at most 2^shift each stay below 2^63
  int bits = 0;
  while ((1 << bits) < V) ++bits;
  a.shift = 62 - bits < 46 ? 62 - bits : 46;
  a.seg = logits_type == WEDLM_SAMPLE_BF16 ? 512 : 256;
  while ((V + a.seg - 1) / a.seg > kSegs) a.seg *= 2;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (logits_type == WEDLM_SAMPLE_BF16)
    hipLaunchKernelGGL(sample_kernel<true>, dim3(static_cast<unsigned>(rows)),
                       dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL(sample_kernel<false>, dim3(static_cast<unsigned>(rows)),
                       dim3(kThreads), 0, st, a);
  WEDLM_LAUNCH_CHECK();
  return WEDLM_OK;
}
