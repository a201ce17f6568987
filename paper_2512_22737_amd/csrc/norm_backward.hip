// Backward passes of the decoder's norms.
//
// RMSNorm, y = x r g with r = 1 / sqrt(mean(x^2) + eps), per row:
//   dg = sum over rows of dy x r          u = dy g
//   dx = r (u - x r mean(u x r))  [+ the gradient that came past the norm]
// Per-head q/k norm with RoPE: the gradient is first rotated back (by minus
// the row's angles), then each head is such a norm over its D values.
#include "common.h"
#include "wedlm_train.h"

using namespace wedlm;

namespace {

constexpr int kThreads = 256;
constexpr int kParts = 512;       // partial gain gradients of a call

// Sum over the wave.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// One workgroup walks the rows t = blockIdx, blockIdx + grid, ...; a thread
// owns the float4 chunks c = tid + 256 i of every row and, with them, their
// part of dg.
template <int CPT>
__global__ __launch_bounds__(kThreads) void rmsnorm_backward_kernel(
    const float* __restrict__ x, const uint16_t* __restrict__ g,
    const uint16_t* __restrict__ dy, const float* dres, int M, int Hd,
    float eps, float* dx, float* __restrict__ part) {
  const int nc = Hd / 4;
  __shared__ float sums[2][2][kThreads / kWave];
  floatx4_t dg[CPT], gg[CPT];
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    dg[i] = floatx4_t{};
    const int c = threadIdx.x + i * kThreads;
    if (c < nc) {
      const u16x4_t v = *reinterpret_cast<const u16x4_t*>(g + c * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) gg[i][e] = bf16_to_f32(v[e]);
    }
  }
  int turn = 0;
  for (int t = blockIdx.x; t < M; t += gridDim.x, turn ^= 1) {
    const int64_t row = static_cast<int64_t>(t) * Hd;
    floatx4_t v[CPT], d[CPT];
    float ss = 0.f, dot = 0.f;
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int c = threadIdx.x + i * kThreads;
      if (c >= nc) continue;
      v[i] = *reinterpret_cast<const floatx4_t*>(x + row + c * 4);
      const u16x4_t b = *reinterpret_cast<const u16x4_t*>(dy + row + c * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        d[i][e] = bf16_to_f32(b[e]);
        ss += v[i][e] * v[i][e];
        dot += d[i][e] * gg[i][e] * v[i][e];
      }
    }
    ss = wave_sum(ss);
    dot = wave_sum(dot);
    if (lane_id() == 0) {
      sums[turn][0][threadIdx.x / kWave] = ss;
      sums[turn][1][threadIdx.x / kWave] = dot;
    }
    __syncthreads();
    ss = dot = 0.f;
#pragma unroll
    for (int i = 0; i < kThreads / kWave; ++i) {
      ss += sums[turn][0][i];
      dot += sums[turn][1][i];
    }
    const float r = 1.0f / sqrtf(ss / static_cast<float>(Hd) + eps);
    const float k = dot * r / static_cast<float>(Hd) * r;
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int c = threadIdx.x + i * kThreads;
      if (c >= nc) continue;
      floatx4_t o;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        dg[i][e] += d[i][e] * (v[i][e] * r);
        o[e] = r * (d[i][e] * gg[i][e] - v[i][e] * k);
      }
      if (dres) {
        const floatx4_t b =
            *reinterpret_cast<const floatx4_t*>(dres + row + c * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += b[e];
      }
      *reinterpret_cast<floatx4_t*>(dx + row + c * 4) = o;
    }
  }
  if (!part) return;
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    const int c = threadIdx.x + i * kThreads;
    if (c < nc)
      *reinterpret_cast<floatx4_t*>(part + static_cast<int64_t>(blockIdx.x) * Hd +
                                    c * 4) = dg[i];
  }
}

// Rows longer than the registers hold (Hd > 16384): the chunks are read twice
// and every workgroup adds to its own row of partials.
__global__ __launch_bounds__(kThreads) void rmsnorm_backward_long_kernel(
    const float* __restrict__ x, const uint16_t* __restrict__ g,
    const uint16_t* __restrict__ dy, const float* dres, int M, int Hd,
    float eps, float* dx, float* __restrict__ part) {
  const int nc = Hd / 4;
  __shared__ float sums[2][2][kThreads / kWave];
  int turn = 0;
  for (int t = blockIdx.x; t < M; t += gridDim.x, turn ^= 1) {
    const int64_t row = static_cast<int64_t>(t) * Hd;
    float ss = 0.f, dot = 0.f;
    for (int c = threadIdx.x; c < nc; c += kThreads) {
      const floatx4_t v = *reinterpret_cast<const floatx4_t*>(x + row + c * 4);
      const u16x4_t b = *reinterpret_cast<const u16x4_t*>(dy + row + c * 4);
      const u16x4_t w = *reinterpret_cast<const u16x4_t*>(g + c * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        ss += v[e] * v[e];
        dot += bf16_to_f32(b[e]) * bf16_to_f32(w[e]) * v[e];
      }
    }
    ss = wave_sum(ss);
    dot = wave_sum(dot);
    if (lane_id() == 0) {
      sums[turn][0][threadIdx.x / kWave] = ss;
      sums[turn][1][threadIdx.x / kWave] = dot;
    }
    __syncthreads();
    ss = dot = 0.f;
#pragma unroll
    for (int i = 0; i < kThreads / kWave; ++i) {
      ss += sums[turn][0][i];
      dot += sums[turn][1][i];
    }
    const float r = 1.0f / sqrtf(ss / static_cast<float>(Hd) + eps);
    const float k = dot * r / static_cast<float>(Hd) * r;
    float* prow = part ? part + static_cast<int64_t>(blockIdx.x) * Hd : nullptr;
    for (int c = threadIdx.x; c < nc; c += kThreads) {
      const floatx4_t v = *reinterpret_cast<const floatx4_t*>(x + row + c * 4);
      const u16x4_t b = *reinterpret_cast<const u16x4_t*>(dy + row + c * 4);
      const u16x4_t w = *reinterpret_cast<const u16x4_t*>(g + c * 4);
      floatx4_t o, s = {};
      if (dres) s = *reinterpret_cast<const floatx4_t*>(dres + row + c * 4);
      floatx4_t p = {};
      if (prow && t != static_cast<int>(blockIdx.x))
        p = *reinterpret_cast<const floatx4_t*>(prow + c * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float d = bf16_to_f32(b[e]);
        p[e] += d * (v[e] * r);
        o[e] = s[e] + r * (d * bf16_to_f32(w[e]) - v[e] * k);
      }
      if (prow) *reinterpret_cast<floatx4_t*>(prow + c * 4) = p;
      *reinterpret_cast<floatx4_t*>(dx + row + c * 4) = o;
    }
  }
}

// Columns of part [parts, n0 + n1] summed in a fixed order into out0 [n0] and
// out1 [n1] (either may be null): 64 columns per workgroup, its four waves
// take every fourth part.
__global__ __launch_bounds__(kThreads) void sum_parts_kernel(
    const float* __restrict__ part, int parts, int n0, int n1,
    float* __restrict__ out0, float* __restrict__ out1) {
  const int n = n0 + n1;
  const int c = blockIdx.x * kWave + lane_id();
  const int w = threadIdx.x / kWave;
  __shared__ float s[kThreads / kWave][kWave];
  float v = 0.f;
  if (c < n)
    for (int p = w; p < parts; p += kThreads / kWave)
      v += part[static_cast<int64_t>(p) * n + c];
  s[w][lane_id()] = v;
  __syncthreads();
  float* out = c < n0 ? out0 : out1;
  if (w == 0 && c < n && out)
    out[c < n0 ? c : c - n0] = (s[0][lane_id()] + s[1][lane_id()]) +
                               (s[2][lane_id()] + s[3][lane_id()]);
}

// q/k norm with RoPE: one workgroup walks rows; an item is 8 rotation pairs
// of one head, the D/16 items of a head sit on neighbouring lanes.  A thread
// meets the same pairs j0 .. j0+7 of D in every item (the strides are
// multiples of a head's items), so the gains' gradients stay in its
// registers until the end.
constexpr int kMaxHalf = 64;

__global__ __launch_bounds__(kThreads) void qk_norm_rope_backward_kernel(
    const uint16_t* __restrict__ qkv, const uint16_t* __restrict__ gq,
    const uint16_t* __restrict__ gk, const int32_t* __restrict__ pos_ids,
    const uint16_t* __restrict__ dq, const uint16_t* __restrict__ dk,
    const uint16_t* __restrict__ dv, int M, int Hq, int Hkv, int D,
    double theta, float eps, uint16_t* __restrict__ dqkv,
    float* __restrict__ part) {
  const int half = D / 2, per_head = half / 8;
  const int n_items = (Hq + Hkv) * per_head, nv = Hkv * D / 8;
  const int H = Hq + 2 * Hkv;
  const int j0 = threadIdx.x % per_head * 8;
  __shared__ float s_cos[kMaxHalf], s_sin[kMaxHalf];
  __shared__ float s_dg[kThreads / kWave][2][2 * kMaxHalf];
  float dga[2][8] = {}, dgb[2][8] = {};
  double omega = 0.0;
  if (threadIdx.x < half)
    omega = pow(theta, -2.0 * static_cast<double>(threadIdx.x) / D);
  for (int t = blockIdx.x; t < M; t += gridDim.x) {
    __syncthreads();
    if (threadIdx.x < half) {
      double sn, cs;
      sincos(static_cast<double>(pos_ids[t]) * omega, &sn, &cs);
      s_cos[threadIdx.x] = static_cast<float>(cs);
      s_sin[threadIdx.x] = static_cast<float>(sn);
    }
    __syncthreads();
    const int64_t row = static_cast<int64_t>(t) * H * D;
    for (int base = 0; base < n_items + nv; base += kThreads) {
      const int it = base + threadIdx.x;
      if (it >= n_items) {
        if (it < n_items + nv)
          *reinterpret_cast<u16x8_t*>(dqkv + row + (Hq + Hkv) * D +
                                      (it - n_items) * 8) =
              *reinterpret_cast<const u16x8_t*>(
                  dv + static_cast<int64_t>(t) * Hkv * D + (it - n_items) * 8);
        continue;
      }
      const int head = it / per_head;
      const bool isq = head < Hq;
      const uint16_t* xp = qkv + row + head * D + j0;
      const uint16_t* dp =
          (isq ? dq + (static_cast<int64_t>(t) * Hq + head) * D
               : dk + (static_cast<int64_t>(t) * Hkv + head - Hq) * D) + j0;
      const uint16_t* gp = (isq ? gq : gk) + j0;
      const u16x8_t xl = *reinterpret_cast<const u16x8_t*>(xp);
      const u16x8_t xh = *reinterpret_cast<const u16x8_t*>(xp + half);
      const u16x8_t dl = *reinterpret_cast<const u16x8_t*>(dp);
      const u16x8_t dh = *reinterpret_cast<const u16x8_t*>(dp + half);
      const u16x8_t gl = *reinterpret_cast<const u16x8_t*>(gp);
      const u16x8_t gh = *reinterpret_cast<const u16x8_t*>(gp + half);
      float a[8], b[8], za[8], zb[8], ss = 0.f, dot = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        a[e] = bf16_to_f32(xl[e]);
        b[e] = bf16_to_f32(xh[e]);
        const float lo = bf16_to_f32(dl[e]), hi = bf16_to_f32(dh[e]);
        const float cs = s_cos[j0 + e], sn = s_sin[j0 + e];
        za[e] = lo * cs + hi * sn;
        zb[e] = hi * cs - lo * sn;
        ss += a[e] * a[e] + b[e] * b[e];
        dot += za[e] * bf16_to_f32(gl[e]) * a[e] +
               zb[e] * bf16_to_f32(gh[e]) * b[e];
      }
      for (int off = 1; off < per_head; off <<= 1) {
        ss += __shfl_xor(ss, off);
        dot += __shfl_xor(dot, off);
      }
      const float r = 1.0f / sqrtf(ss / static_cast<float>(D) + eps);
      const float k = dot * r / static_cast<float>(D) * r;
      u16x8_t ol, oh;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dga[isq ? 0 : 1][e] += za[e] * (a[e] * r);
        dgb[isq ? 0 : 1][e] += zb[e] * (b[e] * r);
        ol[e] = f32_to_bf16(r * (za[e] * bf16_to_f32(gl[e]) - a[e] * k));
        oh[e] = f32_to_bf16(r * (zb[e] * bf16_to_f32(gh[e]) - b[e] * k));
      }
      *reinterpret_cast<u16x8_t*>(dqkv + row + head * D + j0) = ol;
      *reinterpret_cast<u16x8_t*>(dqkv + row + head * D + j0 + half) = oh;
    }
  }
  if (!part) return;
  // lanes of equal j0, then the waves
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float va = dga[s][e], vb = dgb[s][e];
      for (int off = per_head; off < kWave; off <<= 1) {
        va += __shfl_xor(va, off);
        vb += __shfl_xor(vb, off);
      }
      if (lane_id() < per_head) {
        s_dg[threadIdx.x / kWave][s][j0 + e] = va;
        s_dg[threadIdx.x / kWave][s][half + j0 + e] = vb;
      }
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
    const int s = i / D, d = i % D;
    part[static_cast<int64_t>(blockIdx.x) * 2 * D + i] =
        (s_dg[0][s][d] + s_dg[1][s][d]) + (s_dg[2][s][d] + s_dg[3][s][d]);
  }
}

int norm_parts(int M) { return M < kParts ? M : kParts; }

int sum_parts(const float* part, int parts, int n0, int n1, float* out0,
              float* out1, hipStream_t st) {
  hipLaunchKernelGGL(sum_parts_kernel, dim3((n0 + n1 + kWave - 1) / kWave),
                     dim3(kThreads), 0, st, part, parts, n0, n1, out0, out1);
  WEDLM_LAUNCH_CHECK();
  return WEDLM_OK;
}

bool qk_ok(int M, int Hq, int Hkv, int D) {
  return M >= 1 && Hq >= 1 && Hkv >= 1 && (D == 64 || D == 128) &&
         (static_cast<int64_t>(Hq) + 2 * Hkv) * D <= 0x7fffffff / 8;
}

}  // namespace

extern "C" size_t wedlm_rmsnorm_backward_workspace_size(int32_t M, int32_t Hd) {
  if (M < 1 || Hd < 4 || Hd % 4 != 0) return 0;
  return static_cast<size_t>(norm_parts(M)) * Hd * sizeof(float);
}

extern "C" int wedlm_rmsnorm_backward(const float* x, const uint16_t* gain,
                                      const uint16_t* dy, const float* dres,
                                      int32_t M, int32_t Hd, float eps,
                                      float* dx, float* dgain, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  if (!x || !gain || !dy || !dx || !(eps > 0.f)) return WEDLM_E_ARG;
  if (M < 1 || Hd < 4 || Hd % 4 != 0) return WEDLM_E_SHAPE;
  if (dgain && (!workspace ||
                workspace_bytes < wedlm_rmsnorm_backward_workspace_size(M, Hd)))
    return WEDLM_E_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  float* part = dgain ? static_cast<float*>(workspace) : nullptr;
  const int parts = norm_parts(M), nc = Hd / 4;
  auto k = nc <= kThreads       ? rmsnorm_backward_kernel<1>
           : nc <= 2 * kThreads ? rmsnorm_backward_kernel<2>
           : nc <= 4 * kThreads ? rmsnorm_backward_kernel<4>
           : nc <= 8 * kThreads ? rmsnorm_backward_kernel<8>
           : nc <= 16 * kThreads ? rmsnorm_backward_kernel<16>
                                 : rmsnorm_backward_long_kernel;
  hipLaunchKernelGGL(k, dim3(parts), dim3(kThreads), 0, st, x, gain, dy, dres,
                     M, Hd, eps, dx, part);
  WEDLM_LAUNCH_CHECK();
  return dgain ? sum_parts(part, parts, Hd, 0, dgain, nullptr, st) : WEDLM_OK;
}

extern "C" size_t wedlm_qk_norm_rope_backward_workspace_size(int32_t M,
                                                             int32_t Hq,
                                                             int32_t Hkv,
                                                             int32_t D) {
  if (!qk_ok(M, Hq, Hkv, D)) return 0;
  return static_cast<size_t>(norm_parts(M)) * 2 * D * sizeof(float);
}

extern "C" int wedlm_qk_norm_rope_backward(
    const uint16_t* qkv, const uint16_t* q_gain, const uint16_t* k_gain,
    const int32_t* pos_ids, const uint16_t* dq, const uint16_t* dk,
    const uint16_t* dv, int32_t M, int32_t Hq, int32_t Hkv, int32_t D,
    double rope_theta, float eps, uint16_t* dqkv, float* dq_gain,
    float* dk_gain, void* workspace, size_t workspace_bytes, void* stream) {
  if (!qkv || !q_gain || !k_gain || !pos_ids || !dq || !dk || !dv || !dqkv)
    return WEDLM_E_ARG;
  if (!(rope_theta > 1.0) || !(eps > 0.f)) return WEDLM_E_ARG;
  if (!qk_ok(M, Hq, Hkv, D)) return WEDLM_E_SHAPE;
  const bool gains = dq_gain || dk_gain;
  if (gains && (!workspace ||
                workspace_bytes <
                    wedlm_qk_norm_rope_backward_workspace_size(M, Hq, Hkv, D)))
    return WEDLM_E_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  float* part = gains ? static_cast<float*>(workspace) : nullptr;
  const int parts = norm_parts(M);
  hipLaunchKernelGGL(qk_norm_rope_backward_kernel, dim3(parts), dim3(kThreads),
                     0, st, qkv, q_gain, k_gain, pos_ids, dq, dk, dv, M, Hq,
                     Hkv, D, rope_theta, eps, dqkv, part);
  WEDLM_LAUNCH_CHECK();
  return gains ? sum_parts(part, parts, D, D, dq_gain, dk_gain, st) : WEDLM_OK;
}
