// Sampling with temperature, top-k, top-p and min-p from given random numbers
// (wedlm_sample).
//
// One workgroup per row.  What a row keeps is a leading run of its tokens in
// falling order, so it is described by a key (the order-preserving pattern of
// a logit) and a number of ties: tokens above the key, and the first m ids at
// it.  top-k's key is found by counts, top-p's by sums of weights, each by a
// radix search over the key's 32 bits (11, 11 and 10 at a time).  Then the
// kept weights are summed by segments of consecutive ids, and the drawn
// segment is walked.
// Weights w = 2^((x - max) log2(e) / T) are fp64 values rounded to whole
// multiples of 2^-shift (shift >= 41, so that V of them fit 64 bits): sums
// are exact and the same in any order, which both the histogram's atomics and
// the comparison of running sums with u * total need.
#include "common.h"
#include "wedlm_serve.h"

using namespace wedlm;

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 2048;
constexpr int kSegs = 1024;             // segments of a row at most

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
  int W, V, shift;
  int seg;                // tokens per segment, a multiple of 256
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

template <bool HALF>
__device__ __forceinline__ float load(const void* x, int64_t i) {
  if constexpr (HALF) return bf16_to_f32(static_cast<const uint16_t*>(x)[i]);
  else return static_cast<const float*>(x)[i];
}

struct Row {
  double max, rate;       // largest logit; log2(e) / T
  int shift;
  // weight of a key, in units of 2^-shift
  __device__ __forceinline__ uint64_t weight(uint32_t key) const {
    const double t = (static_cast<double>(of_key(key)) - max) * rate;
    if (!(t > -static_cast<double>(shift) - 2)) return 0;
    return static_cast<uint64_t>(rint(ldexp(exp2(t), shift)));
  }
};

struct Lds {
  uint64_t sum[kBins];
  uint32_t count[kBins];
  uint64_t part[kWaves];
  uint64_t found_before, found_ties;
  uint32_t found;
};

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

// The bin, from the highest down, at which the sum of `value` over the bins
// reaches `want` (>= 1, at most the sum of all); `before` gets the sum of the
// bins above it.
template <typename F>
__device__ __forceinline__ uint32_t find_bin(Lds& l, F value, uint64_t want,
                                             uint64_t& before) {
  const int b1 = kBins - 1 - 2 * static_cast<int>(threadIdx.x);   // and b1 - 1
  const uint64_t hi = value(b1), lo = value(b1 - 1);
  uint64_t total;
  const uint64_t at = group_scan(hi + lo, l.part, total);
  if (at < want && at + hi >= want) {
    l.found = b1;
    l.found_before = at;
  } else if (at + hi < want && at + hi + lo >= want) {
    l.found = b1 - 1;
    l.found_before = at + hi;
  }
  __syncthreads();
  before = l.found_before;
  return l.found;
}

template <bool HALF>
__global__ __launch_bounds__(kThreads) void sample_kernel(Args a) {
  __shared__ Lds l;
  const int row = blockIdx.x, b = row / a.W, i = row - b * a.W;
  if (a.n_obs && i < a.n_obs[b]) return;
  const void* x;
  if constexpr (HALF)
    x = static_cast<const uint16_t*>(a.x) + row * a.stride;
  else
    x = static_cast<const float*>(a.x) + row * a.stride;
  const int V = a.V, tid = threadIdx.x, lane = lane_id();
  const int wave = tid / kWave;

  // ---- the largest logit and its first id
  uint64_t best = 0;
  for (int v = tid; v < V; v += kThreads) {
    const uint64_t k = static_cast<uint64_t>(key_of(load<HALF>(x, v))) << 32 |
                       static_cast<uint32_t>(~v);
    best = k > best ? k : best;
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const uint64_t o = __shfl_xor(static_cast<unsigned long long>(best), off);
    best = o > best ? o : best;
  }
  if (lane == 0) l.part[wave] = best;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) best = l.part[w] > best ? l.part[w] : best;
  __syncthreads();
  const uint32_t top = static_cast<uint32_t>(best >> 32);
  const int first = static_cast<int>(~static_cast<uint32_t>(best));
  const float T = a.temp ? a.temp[b] : 1.f;
  if (!(T > 0.f) || of_key(top) == kNegInf) {
    if (tid == 0) {
      a.token[row] = first;
      if (a.logp) a.logp[row] = 0.f;
    }
    return;
  }
  Row r;
  r.max = of_key(top);
  r.rate = 1.4426950408889634 / static_cast<double>(T);
  r.shift = a.shift;
  const int k_raw = a.top_k ? a.top_k[b] : 0;
  const float p = a.top_p ? a.top_p[b] : 1.f;
  const float least = a.min_p ? a.min_p[b] : 0.f;

  // ---- top-k: tokens with keys above tkey, and the first ties at it
  uint32_t tkey = 0;
  uint32_t ties = 0xffffffffu;
  if (k_raw > 0 && k_raw < V) {
    uint32_t prefix = 0;
    uint64_t want = k_raw;
    for (int level = 0; level < 3; ++level) {
      const int down = level == 0 ? 21 : level == 1 ? 10 : 0;
      const int up = level == 0 ? 32 : level == 1 ? 21 : 10;
      for (int j = tid; j < kBins; j += kThreads) l.count[j] = 0;
      __syncthreads();
      for (int v = tid; v < V; v += kThreads) {
        const uint32_t k = key_of(load<HALF>(x, v));
        if (level == 0 || k >> up == prefix >> up)
          atomicAdd(&l.count[(k >> down) & ((1u << (up - down)) - 1)], 1u);
      }
      __syncthreads();
      uint64_t before;
      const uint32_t bin = find_bin(
          l, [&](int j) { return static_cast<uint64_t>(l.count[j]); }, want,
          before);
      prefix |= bin << down;
      want -= before;
      __syncthreads();
    }
    tkey = prefix;
    ties = static_cast<uint32_t>(want);
  }

  // ---- top-p, over what top-k left
  if (p < 1.f) {
    const uint32_t kkey = tkey, kties = ties;
    uint32_t prefix = 0;
    uint64_t want = 0;
    for (int level = 0; level < 3; ++level) {
      const int down = level == 0 ? 21 : level == 1 ? 10 : 0;
      const int up = level == 0 ? 32 : level == 1 ? 21 : 10;
      for (int j = tid; j < kBins; j += kThreads) {
        l.sum[j] = 0;
        l.count[j] = 0;
      }
      __syncthreads();
      for (int v = tid; v < V; v += kThreads) {
        const uint32_t k = key_of(load<HALF>(x, v));
        if (k > kkey && (level == 0 || k >> up == prefix >> up)) {
          const uint64_t q = r.weight(k);
          if (q) {
            atomicAdd(reinterpret_cast<unsigned long long*>(
                          &l.sum[(k >> down) & ((1u << (up - down)) - 1)]),
                      static_cast<unsigned long long>(q));
          }
        }
      }
      __syncthreads();
      // the ties that top-k kept (without top-k kkey is below every key)
      if (tid == 0 && kties != 0xffffffffu &&
          (level == 0 || kkey >> up == prefix >> up))
        l.sum[(kkey >> down) & ((1u << (up - down)) - 1)] +=
            kties * r.weight(kkey);
      __syncthreads();
      if (level == 0) {
        uint64_t total;
        group_scan(l.sum[2 * tid] + l.sum[2 * tid + 1], l.part, total);
        // the least whole number >= p * total, one at least
        const double ps = p > 0.f ? static_cast<double>(p) : 0.0;
        const uint64_t pf = static_cast<uint64_t>(ldexp(ps, 63)) << 1;
        want = __umul64hi(total, pf) + (total * pf != 0 ? 1 : 0);
        want = want < 1 ? 1 : want;
      }
      uint64_t before;
      const uint32_t bin =
          find_bin(l, [&](int j) { return l.sum[j]; }, want, before);
      prefix |= bin << down;
      want -= before;
      __syncthreads();
    }
    tkey = prefix;
    const uint64_t q = r.weight(tkey);
    ties = static_cast<uint32_t>((want + q - 1) / q);
  }

  // ---- min-p
  uint64_t qmin = 1;
  if (least > 0.f) {
    const double m = least < 1.f ? static_cast<double>(least) : 1.0;
    const uint64_t q = static_cast<uint64_t>(rint(ldexp(m, r.shift)));
    qmin = q > 1 ? q : 1;
  }

  // ---- sums and ties of each segment
  const int nseg = (V + a.seg - 1) / a.seg;
  for (int s = wave; s < nseg; s += kWaves) {
    const int end = min(V, (s + 1) * a.seg);
    uint64_t sum = 0;
    uint32_t at = 0;
    for (int v = s * a.seg + lane; v < end; v += kWave) {
      const uint32_t k = key_of(load<HALF>(x, v));
      if (k > tkey) {
        const uint64_t q = r.weight(k);
        sum += q >= qmin ? q : 0;
      }
      at += k == tkey ? 1 : 0;
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
      sum += __shfl_xor(static_cast<unsigned long long>(sum), off);
      at += __shfl_xor(at, off);
    }
    if (lane == 0) {
      l.sum[s] = sum;
      l.count[s] = at;
    }
  }
  __syncthreads();
  uint64_t qt = r.weight(tkey);
  qt = qt >= qmin ? qt : 0;
  uint64_t total;
  const uint32_t mine = tid < nseg ? l.count[tid] : 0;
  const uint64_t ties_before = group_scan(mine, l.part, total);
  const uint64_t left = ties > ties_before ? ties - ties_before : 0;
  const uint64_t own = (tid < nseg ? l.sum[tid] : 0) +
                       qt * (left < mine ? left : mine);
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
  // ---- the segment that holds the drawn token, one wave
  uint64_t run = l.found_before, seen = l.found_ties;
  const int s = l.found;
  const int end = min(V, (s + 1) * a.seg);
  for (int base = s * a.seg; base < end; base += kWave) {
    const int v = base + lane;
    const uint32_t k = v < end ? key_of(load<HALF>(x, v)) : 0;
    const bool tie = v < end && k == tkey;
    const uint64_t tm = ballot(tie);
    const uint64_t rank = seen + __popcll(tm & ((1ull << lane) - 1));
    uint64_t q = 0;
    if (v < end && (k > tkey || (tie && rank < ties))) q = r.weight(k);
    q = q >= qmin ? q : 0;
    uint64_t c = q;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      const uint64_t o = __shfl_up(static_cast<unsigned long long>(c), off);
      if (lane >= off) c += o;
    }
    const uint64_t hit = ballot(run + c > goal);
    if (hit) {
      if (lane == __ffsll(static_cast<unsigned long long>(hit)) - 1) {
        a.token[row] = v;
        if (a.logp)
          a.logp[row] = static_cast<float>(
              (static_cast<double>(of_key(k)) - r.max) /
                  static_cast<double>(T) -
              log(ldexp(static_cast<double>(total), -r.shift)));
      }
      return;
    }
    run += __shfl(static_cast<unsigned long long>(c), kWave - 1);
    seen += __popcll(tm);
  }
}

}  // namespace

extern "C" size_t wedlm_sample_workspace_size(int32_t B, int32_t W,
                                              int32_t V) {
  (void)B; (void)W; (void)V;
  return 0;
}

extern "C" int wedlm_sample(const void* logits, int32_t logits_type,
                            int64_t row_stride, const float* u,
                            const int32_t* n_obs, const float* temperature,
                            const int32_t* top_k, const float* top_p,
                            const float* min_p, int32_t B, int32_t W,
                            int32_t V, int32_t* token, float* logp,
                            void* workspace, size_t workspace_bytes,
                            void* stream) {
  (void)workspace; (void)workspace_bytes;
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
  a.token = token; a.logp = logp; a.W = W; a.V = V;
  // V weights of at most 2^shift each stay below 2^63
  int bits = 0;
  while ((1 << bits) < V) ++bits;
  a.shift = 62 - bits < 46 ? 62 - bits : 46;
  a.seg = 256;
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
