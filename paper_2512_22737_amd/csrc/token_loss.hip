// The masked-token loss of the training objective with the gradient of its
// logits.  Row r with target t and weight w (logits l, m the largest; R the sum
// over all others, Z = R + e^{l_t - m}):
//   loss = w (ln Z + (m - l_t)), ln Z = ln(1 + R) if l_t = m
//   dl_v = w e^{l_v - m} / Z for v != t,  dl_t = -w R / Z
// Nothing cancels, so that a token predicted with p_t near 1 keeps the digits
// of 1 - p_t; the target is kept out of the sum from the start.
// One workgroup per row.  Every thread keeps the first H 16-byte chunks that
// it reads in registers: maximum, sum and gradient all come from there, so that
// these logits are read once.  What does not fit (fp32 rows beyond 77824) is
// reduced with a running maximum and read again for the gradient.  Few long
// rows are split over workgroups: one kernel for the slices' maxima and sums,
// one that joins them and forms the gradient.
// Bound by HBM: logits read once, gradients written once (past the caches: a
// large gradient does not stay there, the row's rest does).  4096 x 151936
// fp32 1.03 ms, 4.8 TB/s, where a large copy reaches 5.1 (one element at a
// time in two passes 1.85 ms); 1000 x 32003 bf16, half of the rows without
// loss, 24 us; 32 x 1024 8 us, one launch.
#include "common.h"
#include "wedlm_train.h"

#include <algorithm>

using namespace wedlm;

namespace {

constexpr float kLog2e = 1.4426950408889634f;
// Workgroups of few long rows: threads, chunks a thread holds
constexpr int kSmallThreads = 256, kSmallHeld = 16;
constexpr int kSmallChunks = kSmallThreads * kSmallHeld;

struct LossArgs {
  const void* logits;     // [R, stride] fp32 or bf16
  const int32_t* target;  // [R]
  const float* weight;    // [R] or null
  float* loss;            // [R]
  void* dlogits;          // [R, stride] or null
  float2* part;           // [R, slices + 1]: maximum, sum; the target's logit
  int64_t stride;
  int R, V, slices, slice_len;
};

// Running maximum and sum of e^{x - m}.
struct MaxSum {
  float m, s;
};

__device__ __forceinline__ float exp_below(float x, float m) {
  return __builtin_amdgcn_exp2f((x - m) * kLog2e);
}

// The same to the bit whichever way round: the one with the larger maximum
// enters as it is.  (With both scaled, one product would be rounded and the
// other fused into the sum, by its place.)
__device__ __forceinline__ MaxSum merge(MaxSum a, MaxSum b) {
  const bool first = a.m >= b.m;
  const MaxSum hi{first ? a.m : b.m, first ? a.s : b.s};
  const MaxSum lo{first ? b.m : a.m, first ? b.s : a.s};
  if (lo.m == kNegInf) return hi;
  return {hi.m, __builtin_fmaf(lo.s, exp_below(lo.m, hi.m), hi.s)};
}

// One element type: values of a 16-byte chunk and of a single element.
template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static constexpr int n = 4;
  typedef floatx4_t chunk;
  __device__ static float get(const chunk& c, int e) { return c[e]; }
  __device__ static void set(chunk& c, int e, float v) { c[e] = v; }
  __device__ static float get(const float* p) { return *p; }
  __device__ static void set(float* p, float v) { *p = v; }
};
template <>
struct Elem<uint16_t> {
  static constexpr int n = 8;
  typedef u16x8_t chunk;
  __device__ static float get(const chunk& c, int e) { return bf16_to_f32(c[e]); }
  __device__ static void set(chunk& c, int e, float v) { c[e] = to_bf16(v); }
  __device__ static float get(const uint16_t* p) { return bf16_to_f32(*p); }
  __device__ static void set(uint16_t* p, float v) { *p = to_bf16(v); }
};

// A stretch of a row: elements up to the first 16-byte boundary, whole
// chunks, and the rest; the single elements (fewer than 16) are numbered on.
template <typename T>
struct Span {
  int head, chunks, singles;
  __device__ __forceinline__ Span(const T* p, int n) {
    constexpr int E = Elem<T>::n;
    const int off = static_cast<int>(reinterpret_cast<uintptr_t>(p) / sizeof(T)) &
                    (E - 1);
    head = min(off ? E - off : 0, n);
    chunks = (n - head) / E;
    singles = n - chunks * E;
  }
  __device__ __forceinline__ int single(int i) const {
    return i < head ? i : i + chunks * Elem<T>::n;
  }
};

// Reduction over the workgroup, the same value in every thread.
template <int NT, typename Op>
__device__ __forceinline__ float reduce(float v, float* lds, Op op) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = op(v, __shfl_xor(v, off));
  if (lane_id() == 0) lds[threadIdx.x / kWave] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int i = 1; i < NT / kWave; ++i) v = op(v, lds[i]);
  return v;
}

__device__ __forceinline__ bool no_loss(const LossArgs& a, int r, int& t,
                                        float& w) {
  t = a.target[r];
  w = a.weight ? a.weight[r] : 1.f;
  return t < 0 || t >= a.V || w == 0.f;
}

// What a row's loss and gradient take from its maximum m, the sum of the
// others r and the target's logit lt.
struct RowStats {
  float loss;
  float ref, k, hit;      // dl_v = e^{l_v - ref} k, dl_t = hit
  __device__ __forceinline__ RowStats(float w, float m, float r, float lt) {
    if (m == kNegInf) {   // nothing but -inf: no probabilities, gradient 0
      loss = w * -kNegInf;
      ref = k = hit = 0.f;
      return;
    }
    const float z = r + exp_below(lt, m);
    loss = w * (lt == m ? log1pf(r) : logf(z) + (m - lt));
    ref = m;
    k = w / z;
    hit = -w * (r / z);
  }
};

// The chunk without the target (element e of it, if in 0 .. n-1).
template <typename T>
__device__ __forceinline__ void drop(typename Elem<T>::chunk& x, int e) {
#pragma unroll
  for (int i = 0; i < Elem<T>::n; ++i)
    if (i == e) Elem<T>::set(x, i, kNegInf);
}

// Zeros over a stretch of a row of dlogits.
template <typename T, int NT>
__device__ __forceinline__ void clear(T* p, int n) {
  const Span<T> sp(p, n);
  typedef typename Elem<T>::chunk C;
  C* body = reinterpret_cast<C*>(p + sp.head);
  for (int c = threadIdx.x; c < sp.chunks; c += NT) body[c] = C{};
  if (static_cast<int>(threadIdx.x) < sp.singles)
    p[sp.single(threadIdx.x)] = static_cast<T>(0);
}

// Logits and gradients at the same offset from a 16-byte boundary: rows of
// both have the same chunks.
template <typename T, int NT, int H>
__global__ __launch_bounds__(NT) void token_loss_kernel(LossArgs a) {
  typedef Elem<T> E;
  typedef typename E::chunk C;
  const int r = blockIdx.x;
  const T* row = static_cast<const T*>(a.logits) + r * a.stride;
  T* drow = a.dlogits ? static_cast<T*>(a.dlogits) + r * a.stride : nullptr;
  int t;
  float w;
  if (no_loss(a, r, t, w)) {
    if (threadIdx.x == 0) a.loss[r] = 0.f;
    if (drow) clear<T, NT>(drow, a.V);
    return;
  }
  __shared__ float lds[2][NT / kWave];
  const Span<T> sp(row, a.V);
  const C* body = reinterpret_cast<const C*>(row + sp.head);
  const int tid = threadIdx.x;
  // the target's logit is read before any gradient is written over it
  const float lt = E::get(row + t);
  const int tb = t - sp.head;            // the target, from the first chunk
  const int tc = tb >= 0 ? tb / E::n : -1;
  C held[H];
  float one = kNegInf, m = lt;
#pragma unroll
  for (int i = 0; i < H; ++i)
    if (tid + i * NT < sp.chunks) held[i] = body[tid + i * NT];
  const bool single = tid < sp.singles && sp.single(tid) != t;
  if (single) one = E::get(row + sp.single(tid));
  m = fmaxf(m, one);
#pragma unroll
  for (int i = 0; i < H; ++i)
    if (tid + i * NT < sp.chunks) {
      if (tid + i * NT == tc) drop<T>(held[i], tb - tc * E::n);
#pragma unroll
      for (int e = 0; e < E::n; ++e) m = fmaxf(m, E::get(held[i], e));
    }
  // the rest, four chunks under way at a time (past the end: the last again)
  constexpr int U = 4;
  MaxSum rest{kNegInf, 0.f};
  for (int c0 = tid + H * NT; c0 < sp.chunks; c0 += U * NT) {
    C x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = body[min(c0 + u * NT, sp.chunks - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * NT;
      if (c >= sp.chunks) break;
      if (c == tc) drop<T>(x[u], tb - tc * E::n);
      float cm = E::get(x[u], 0);
#pragma unroll
      for (int e = 1; e < E::n; ++e) cm = fmaxf(cm, E::get(x[u], e));
      if (cm > rest.m) {
        rest.s *= exp_below(rest.m, cm);
        rest.m = cm;
      }
      if (rest.m != kNegInf) {
#pragma unroll
        for (int e = 0; e < E::n; ++e)
          rest.s += exp_below(E::get(x[u], e), rest.m);
      }
    }
  }
  m = reduce<NT>(fmaxf(m, rest.m), lds[0],
                 [](float x, float y) { return fmaxf(x, y); });
  const float ref = m == kNegInf ? 0.f : m;
  float s = rest.m == kNegInf ? 0.f : rest.s * exp_below(rest.m, ref);
  if (single) s += exp_below(one, ref);
#pragma unroll
  for (int i = 0; i < H; ++i)
    if (tid + i * NT < sp.chunks) {
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < E::n; ++e) x += exp_below(E::get(held[i], e), ref);
      s += x;
    }
  s = reduce<NT>(s, lds[1], [](float x, float y) { return x + y; });
  const RowStats q(w, m, s, lt);
  if (tid == 0) a.loss[r] = q.loss;
  if (!drow) return;
  C* dbody = reinterpret_cast<C*>(drow + sp.head);
  auto grad = [&](const C& x, int c) {
    C d;
#pragma unroll
    for (int e = 0; e < E::n; ++e)
      E::set(d, e, tb == c * E::n + e ? q.hit
                                      : exp_below(E::get(x, e), q.ref) * q.k);
    __builtin_nontemporal_store(d, dbody + c);
  };
#pragma unroll
  for (int i = 0; i < H; ++i)
    if (tid + i * NT < sp.chunks) grad(held[i], tid + i * NT);
  for (int c0 = tid + H * NT; c0 < sp.chunks; c0 += U * NT) {
    C x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = body[min(c0 + u * NT, sp.chunks - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c0 + u * NT < sp.chunks) grad(x[u], c0 + u * NT);
  }
  if (tid < sp.singles)
    E::set(drow + sp.single(tid),
           single ? exp_below(one, q.ref) * q.k : q.hit);
}

// Maximum and sum of one slice, without the target.
template <typename T>
__global__ __launch_bounds__(kSmallThreads) void slice_kernel(LossArgs a) {
  typedef Elem<T> E;
  typedef typename E::chunk C;
  const int r = blockIdx.y, sl = blockIdx.x;
  int t;
  float w;
  if (no_loss(a, r, t, w)) return;
  __shared__ float lds[2][kSmallThreads / kWave];
  const int v0 = sl * a.slice_len;
  const int n = min(a.slice_len, a.V - v0);
  const T* p = static_cast<const T*>(a.logits) + r * a.stride + v0;
  const Span<T> sp(p, n);
  const C* body = reinterpret_cast<const C*>(p + sp.head);
  const int tid = threadIdx.x;
  C held[kSmallHeld];
  const int tb = t - v0 - sp.head;
  const int tc = tb >= 0 ? tb / E::n : -1;
  float one = kNegInf, m = kNegInf, s = 0.f;
#pragma unroll
  for (int i = 0; i < kSmallHeld; ++i)
    if (tid + i * kSmallThreads < sp.chunks) held[i] = body[tid + i * kSmallThreads];
  const bool single = tid < sp.singles && v0 + sp.single(tid) != t;
  if (single) m = one = E::get(p + sp.single(tid));
#pragma unroll
  for (int i = 0; i < kSmallHeld; ++i)
    if (tid + i * kSmallThreads < sp.chunks) {
      if (tid + i * kSmallThreads == tc) drop<T>(held[i], tb - tc * E::n);
#pragma unroll
      for (int e = 0; e < E::n; ++e) m = fmaxf(m, E::get(held[i], e));
    }
  m = reduce<kSmallThreads>(m, lds[0],
                            [](float x, float y) { return fmaxf(x, y); });
  const float ref = m == kNegInf ? 0.f : m;
  if (single) s += exp_below(one, ref);
#pragma unroll
  for (int i = 0; i < kSmallHeld; ++i)
    if (tid + i * kSmallThreads < sp.chunks) {
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < E::n; ++e) x += exp_below(E::get(held[i], e), ref);
      s += x;
    }
  s = reduce<kSmallThreads>(s, lds[1], [](float x, float y) { return x + y; });
  if (tid == 0) {
    float2* part = a.part + static_cast<int64_t>(r) * (a.slices + 1);
    part[sl] = make_float2(m, s);
    if (t >= v0 && t < v0 + n)
      part[a.slices] = make_float2(E::get(p + t - v0), 0.f);
  }
}

// Gradient of one slice, the slices joined in order; the loss too where the
// slice holds the target.  Every slice needs the target's logit, which
// slice_kernel has left behind the slices' sums: here it may be overwritten.
template <typename T>
__global__ __launch_bounds__(kSmallThreads) void slice_grad_kernel(LossArgs a) {
  typedef Elem<T> E;
  typedef typename E::chunk C;
  const int r = blockIdx.y, sl = blockIdx.x;
  const int v0 = sl * a.slice_len;
  const int n = min(a.slice_len, a.V - v0);
  const T* p = static_cast<const T*>(a.logits) + r * a.stride + v0;
  T* dp = a.dlogits ? static_cast<T*>(a.dlogits) + r * a.stride + v0 : nullptr;
  int t;
  float w;
  if (no_loss(a, r, t, w)) {
    if (sl == 0 && threadIdx.x == 0) a.loss[r] = 0.f;
    if (dp) clear<T, kSmallThreads>(dp, n);
    return;
  }
  const int tid = threadIdx.x;
  const bool mine = t >= v0 && t < v0 + n;
  if (!dp && !mine) return;
  const float2* part = a.part + static_cast<int64_t>(r) * (a.slices + 1);
  // (every lane ends with the same value: merge() does not ask for an order)
  MaxSum x{kNegInf, 0.f};
  for (int i = lane_id(); i < a.slices; i += kWave)
    x = merge(x, MaxSum{part[i].x, part[i].y});
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1)
    x = merge(x, MaxSum{__shfl_xor(x.m, off), __shfl_xor(x.s, off)});
  const float lt = part[a.slices].x;
  const float m = fmaxf(x.m, lt);
  const RowStats q(w, m, x.m == kNegInf ? 0.f : x.s * exp_below(x.m, m), lt);
  if (mine && tid == 0) a.loss[r] = q.loss;
  if (!dp) return;
  const Span<T> sp(p, n);
  const C* body = reinterpret_cast<const C*>(p + sp.head);
  C* dbody = reinterpret_cast<C*>(dp + sp.head);
  const int tb = t - v0 - sp.head;
#pragma unroll 4
  for (int c = tid; c < sp.chunks; c += kSmallThreads) {
    const C l = body[c];
    C d;
#pragma unroll
    for (int e = 0; e < E::n; ++e)
      E::set(d, e, tb == c * E::n + e ? q.hit
                                      : exp_below(E::get(l, e), q.ref) * q.k);
    dbody[c] = d;
  }
  if (tid < sp.singles) {
    const int v = sp.single(tid);
    E::set(dp + v, v + v0 == t ? q.hit
                               : exp_below(E::get(p + v), q.ref) * q.k);
  }
}

// Logits and gradients at different offsets from 16-byte boundaries: element
// by element, a running maximum and sum, then the gradient.  (Unsigned: the
// column after a row's last one may pass 2^31 - 1.)
template <typename T>
__global__ __launch_bounds__(kSmallThreads) void token_loss_plain_kernel(
    LossArgs a) {
  typedef Elem<T> E;
  const int r = blockIdx.x;
  const T* row = static_cast<const T*>(a.logits) + r * a.stride;
  T* drow = static_cast<T*>(a.dlogits) + r * a.stride;
  const uint32_t tid = threadIdx.x, V = static_cast<uint32_t>(a.V);
  int t;
  float w;
  if (no_loss(a, r, t, w)) {
    if (tid == 0) a.loss[r] = 0.f;
    clear<T, kSmallThreads>(drow, a.V);
    return;
  }
  __shared__ float lds[2][kSmallThreads / kWave];
  const float lt = E::get(row + t);
  const uint32_t target = static_cast<uint32_t>(t);      // (0 .. V-1)
  MaxSum x{kNegInf, 0.f};
  for (uint32_t v = tid; v < V; v += kSmallThreads) {
    const float l = v == target ? kNegInf : E::get(row + v);
    if (l > x.m) {
      x.s *= exp_below(x.m, l);
      x.m = l;
    }
    if (x.m != kNegInf) x.s += exp_below(l, x.m);
  }
  const float m = reduce<kSmallThreads>(
      fmaxf(x.m, lt), lds[0], [](float y, float z) { return fmaxf(y, z); });
  const float s = reduce<kSmallThreads>(
      x.m == kNegInf ? 0.f : x.s * exp_below(x.m, m), lds[1],
      [](float y, float z) { return y + z; });
  const RowStats q(w, m, s, lt);
  if (tid == 0) a.loss[r] = q.loss;
  for (uint32_t v = tid; v < V; v += kSmallThreads)
    E::set(drow + v,
           v == target ? q.hit : exp_below(E::get(row + v), q.ref) * q.k);
}

// Elements of a row's slices, or V (one slice).  Rows of more than 16384 chunks
// (262144 bytes) are cut when they are fewer than 128, so that there are about
// 512 workgroups, of 1024 chunks each at least.  In us, whole rows and slices:
// 8 x 151936 fp32 22.9, 9.7, bf16 22.6, 9.5; 64 x 151936 25.4, 22.6 and 23.0,
// 16.4; 128 x 151936 bf16 25.4, 26.0; 200 x 151936 51.6, 59 and 29.7, 35.6;
// 64 x 32000 fp32 8.8, 10.4.
int slice_len(int R, int V, int per_chunk) {
  const int64_t chunks = V / per_chunk;
  if (R >= 128 || chunks <= 4 * kSmallChunks) return V;
  int64_t c = (chunks * R / 512 + kSmallThreads - 1) / kSmallThreads;
  c = c < 4 ? 4 : c > kSmallHeld ? kSmallHeld : c;
  return static_cast<int>(c) * kSmallThreads * per_chunk;
}

int row_slices(int R, int V, int per_chunk) {
  const int len = slice_len(R, V, per_chunk);
  return V / len + (V % len != 0);
}

// One workgroup per row, in stretches of rows: a launch has fewer than 2^32
// threads.
constexpr int kRowsPerLaunch = 1 << 21;

template <typename T>
int launch_rows(void (*kernel)(LossArgs), int threads, const LossArgs& a,
                hipStream_t st) {
  for (int64_t r = 0; r < a.R; r += kRowsPerLaunch) {
    LossArgs b = a;
    b.logits = static_cast<const T*>(a.logits) + r * a.stride;
    b.target = a.target + r;
    b.weight = a.weight ? a.weight + r : nullptr;
    b.loss = a.loss + r;
    b.dlogits = a.dlogits ? static_cast<T*>(a.dlogits) + r * a.stride : nullptr;
    const int64_t rows = std::min<int64_t>(a.R - r, kRowsPerLaunch);
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(rows)), dim3(threads),
                       0, st, b);
    WEDLM_LAUNCH_CHECK();
  }
  return WEDLM_OK;
}

template <typename T>
int launch(const LossArgs& a0, hipStream_t st) {
  LossArgs a = a0;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.logits);
  const uintptr_t y = reinterpret_cast<uintptr_t>(a.dlogits);
  if (y && (x ^ y) % 16 != 0)
    return launch_rows<T>(token_loss_plain_kernel<T>, kSmallThreads, a, st);
  a.slices = row_slices(a.R, a.V, Elem<T>::n);
  a.slice_len = slice_len(a.R, a.V, Elem<T>::n);
  if (a.slices > 1) {
    hipLaunchKernelGGL(slice_kernel<T>, dim3(a.slices, a.R),
                       dim3(kSmallThreads), 0, st, a);
    WEDLM_LAUNCH_CHECK();
    hipLaunchKernelGGL(slice_grad_kernel<T>, dim3(a.slices, a.R),
                       dim3(kSmallThreads), 0, st, a);
    WEDLM_LAUNCH_CHECK();
    return WEDLM_OK;
  }
  // 256 threads as long as they hold the row: 1000 x 8000 fp32 10.3 us against
  // 20.8 with 1024; four chunks each where those do (4000 x 1000 9.6, 15.3).
  // Up to a row per CU 1024 are as many as the row has use for: 256 x 32000 bf16
  // 12.9 with 256, 9.6 with 1024; 384 x 32000 14.8, 17.1
  const int chunks = a.V / Elem<T>::n;
  if (chunks <= kSmallThreads * 4)
    return launch_rows<T>(token_loss_kernel<T, kSmallThreads, 4>,
                          kSmallThreads, a, st);
  if (chunks <= kSmallChunks && a.R > 256)
    return launch_rows<T>(token_loss_kernel<T, kSmallThreads, kSmallHeld>,
                          kSmallThreads, a, st);
  return launch_rows<T>(token_loss_kernel<T, 1024, 19>, 1024, a, st);
}

}  // namespace

extern "C" size_t wedlm_token_loss_workspace_size(int32_t R, int32_t V) {
  if (R < 1 || V < 1) return 0;
  const int n = std::max(row_slices(R, V, Elem<float>::n),
                         row_slices(R, V, Elem<uint16_t>::n));
  return n > 1 ? static_cast<size_t>(R) * (n + 1) * sizeof(float2) : 0;
}

extern "C" int wedlm_token_loss(const void* logits, int32_t logits_type,
                                int64_t row_stride, const int32_t* target,
                                const float* weight, int32_t R, int32_t V,
                                float* loss, void* dlogits, void* workspace,
                                size_t workspace_bytes, void* stream) {
  if (!logits || !target || !loss) return WEDLM_E_ARG;
  if (logits_type != WEDLM_LOGITS_F32 && logits_type != WEDLM_LOGITS_BF16)
    return WEDLM_E_ARG;
  if (R < 1 || V < 1 || row_stride < V) return WEDLM_E_SHAPE;
  const size_t need = wedlm_token_loss_workspace_size(R, V);
  // (a float2 for every slice)
  if (need && reinterpret_cast<uintptr_t>(workspace) % sizeof(float2) != 0)
    return WEDLM_E_ARG;
  if (need && (!workspace || workspace_bytes < need)) return WEDLM_E_WORKSPACE;
  LossArgs a{};
  a.logits = logits;
  a.target = target;
  a.weight = weight;
  a.loss = loss;
  a.dlogits = dlogits;
  a.part = static_cast<float2*>(workspace);
  a.stride = row_stride;
  a.R = R;
  a.V = V;
  hipStream_t st = static_cast<hipStream_t>(stream);
  return logits_type == WEDLM_LOGITS_F32
             ? launch<float>(a, st)
             : launch<uint16_t>(a, st);
}
