// The masked-token loss of the training objective with the gradient of its
// logits.  Row r with target t and weight w (logits l, Z = sum_v e^{l_v - m},
// m the largest logit):
//   loss = w (ln Z - (l_t - m))      dl_v = w (e^{l_v - m} / Z - [v = t])
// One workgroup per row: a pass with a running maximum and sum per thread,
// then one that forms the gradient from logits that are still in a cache.
// Bound by HBM: logits read once, gradients written once.
#include "common.h"
#include "wedlm_train.h"

using namespace wedlm;

namespace {

constexpr int kThreads = 512;
constexpr float kLog2e = 1.4426950408889634f;

struct LossArgs {
  const void* logits;     // [R, stride] fp32 or bf16
  const int32_t* target;  // [R]
  const float* weight;    // [R] or null
  float* loss;            // [R]
  void* dlogits;          // [R, stride] or null
  int64_t stride;
  int R, V;
};

// Running maximum and sum of e^{x - m}.
struct MaxSum {
  float m, s;
};

__device__ __forceinline__ float exp_below(float x, float m) {
  return __builtin_amdgcn_exp2f((x - m) * kLog2e);
}

__device__ __forceinline__ MaxSum merge(MaxSum a, MaxSum b) {
  const float m = fmaxf(a.m, b.m);
  if (m == kNegInf) return {m, 0.f};
  return {m, a.s * exp_below(a.m, m) + b.s * exp_below(b.m, m)};
}

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t* p) {
  return bf16_to_f32(*p);
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t* p, float v) {
  *p = f32_to_bf16(v);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void token_loss_kernel(LossArgs a) {
  const int r = blockIdx.x;
  const T* row = static_cast<const T*>(a.logits) + r * a.stride;
  T* drow = a.dlogits ? static_cast<T*>(a.dlogits) + r * a.stride : nullptr;
  const int t = a.target[r];
  const float w = a.weight ? a.weight[r] : 1.f;
  if (t < 0 || t >= a.V || w == 0.f) {
    if (threadIdx.x == 0) a.loss[r] = 0.f;
    if (drow)
      for (int v = threadIdx.x; v < a.V; v += kThreads) store1(drow + v, 0.f);
    return;
  }
  MaxSum x{kNegInf, 0.f};
  for (int v = threadIdx.x; v < a.V; v += kThreads) {
    const float l = load1(row + v);
    if (l == kNegInf) continue;
    if (l > x.m) {
      x.s = x.s * exp_below(x.m, l) + 1.f;
      x.m = l;
    } else {
      x.s += exp_below(l, x.m);
    }
  }
  __shared__ MaxSum part[kThreads / kWave];
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1)
    x = merge(x, MaxSum{__shfl_xor(x.m, off), __shfl_xor(x.s, off)});
  if (lane_id() == 0) part[threadIdx.x / kWave] = x;
  // the target's logit is read before any gradient is written over it
  const float lt = load1(row + t);
  __syncthreads();
  x = part[0];
#pragma unroll
  for (int i = 1; i < kThreads / kWave; ++i) x = merge(x, part[i]);
  if (threadIdx.x == 0)
    a.loss[r] = w * (x.m == kNegInf ? -kNegInf : logf(x.s) - (lt - x.m));
  if (!drow) return;
  const float k = x.m == kNegInf ? 0.f : w / x.s;
  for (int v = threadIdx.x; v < a.V; v += kThreads) {
    const float l = load1(row + v);
    float d = l == kNegInf ? 0.f : exp_below(l, x.m) * k;
    if (v == t && x.m != kNegInf) d -= w;
    store1(drow + v, d);
  }
}

}  // namespace

extern "C" size_t wedlm_token_loss_workspace_size(int32_t R, int32_t V) {
  return 0;
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
  if (need && (!workspace || workspace_bytes < need)) return WEDLM_E_WORKSPACE;
  LossArgs a{logits, target, weight, loss, dlogits, row_stride, R, V};
  hipLaunchKernelGGL(logits_type == WEDLM_LOGITS_F32
                         ? token_loss_kernel<float>
                         : token_loss_kernel<uint16_t>,
                     dim3(R), dim3(kThreads), 0,
                     static_cast<hipStream_t>(stream), a);
  WEDLM_LAUNCH_CHECK();
  return WEDLM_OK;
}
