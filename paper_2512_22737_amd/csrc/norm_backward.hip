// Backward passes of the decoder's norms.
//
// RMSNorm, y = x r g with r = 1 / sqrt(mean(x^2) + eps), per row:
//   dg = sum over rows of dy x r          u = dy g
//   dx = r (u - x r mean(u x r))  [+ the gradient that came past the norm]
// Per-head q/k norm with RoPE: the gradient is first rotated back (by minus
// the row's angles), then each head is such a norm over its D values.
//
// Bound by HBM: every array is passed over once, rows stay in registers between
// their sums and their gradients.  RMSNorm 32768 x 4096 338-346 us, 5.5 TB/s
// (a large copy reaches 5.1), 8193 x 2560 without a residual gradient 47 us,
// 4.4 TB/s; q/k norm with RoPE of 32768 rows of 32/8 heads of 128 229 us,
// 4.9 TB/s.  Few rows are bound by the two launches, 8 to 12 us.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "common.h"
#include "wedlm_train.h"

using namespace wedlm;

namespace {

constexpr int kThreads = 256;
// Workgroups of the q/k kernel, at most: four per CU (32768 rows of 16/2 heads
// of 64 54 us; 512 workgroups 73, 2048 59)
constexpr int kQkParts = 1024;

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
  // (unsigned: t may pass 2^31 - 1 once)
  for (uint32_t t = blockIdx.x; t < static_cast<uint32_t>(M);
       t += gridDim.x, turn ^= 1) {
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
  // (unsigned: t may pass 2^31 - 1 once)
  for (uint32_t t = blockIdx.x; t < static_cast<uint32_t>(M);
       t += gridDim.x, turn ^= 1) {
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
      if (prow && t != blockIdx.x)
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
// out1 [n1] (either may be null): C columns per workgroup, 1024 / C threads to a
// column, eight loads under way each: with 64 columns 1024 parts are eight
// round trips to memory.
constexpr int kSumThreads = 1024;

template <int C>
__global__ __launch_bounds__(kSumThreads) void sum_parts_kernel(
    const float* __restrict__ part, int parts, int n0, int n1,
    float* __restrict__ out0, float* __restrict__ out1) {
  constexpr int W = kSumThreads / C;
  const int n = n0 + n1, col = threadIdx.x % C;
  const int c = blockIdx.x * C + col;
  __shared__ float s[kSumThreads / kWave][C];
  float v = 0.f;
  if (c < n) {
    int p = threadIdx.x / C;
    for (; p + 7 * W < parts; p += 8 * W) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        x[i] = part[static_cast<int64_t>(p + i * W) * n + c];
      v += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    }
#pragma unroll 4
    for (; p < parts; p += W) v += part[static_cast<int64_t>(p) * n + c];
  }
#pragma unroll
  for (int off = C; off < kWave; off <<= 1) v += __shfl_xor(v, off);
  if (lane_id() < C) s[threadIdx.x / kWave][col] = v;
  __syncthreads();
  float* out = c < n0 ? out0 : out1;
  if (threadIdx.x < C && c < n && out) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kSumThreads / kWave; ++i) t += s[i][col];
    out[c < n0 ? c : c - n0] = t;
  }
}

// q/k norm with RoPE: one workgroup walks groups of R rows; an item is 8
// rotation pairs of one head of one row, the D/16 items of a head sit on
// neighbouring lanes.  A thread meets the same pairs j0 .. j0+7 of D in every
// item (the strides are multiples of a head's items), so the gains' gradients
// stay in its registers until the end.  Several rows at once give every
// thread an angle (64 bits: positions are far) and items to hide the loads.
constexpr int kMaxHalf = 64;

struct QkArgs {
  const uint16_t* qkv;
  const uint16_t* gq;
  const uint16_t* gk;
  const int32_t* pos;
  const uint16_t* dq;
  const uint16_t* dk;
  const uint16_t* dv;
  uint16_t* dqkv;
  float* part;            // [grid, 2, D] or null
  int M, Hq, Hkv, D;
  float eps;
  double omega[kMaxHalf]; // theta^(-2j/D)
};

template <int R>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_backward_kernel(
    QkArgs a) {
  const int half = a.D / 2, per_head = half / 8;
  const int n_items = (a.Hq + a.Hkv) * per_head, nv = a.Hkv * a.D / 8;
  const int H = a.Hq + 2 * a.Hkv;
  const int j0 = threadIdx.x % per_head * 8;
  __shared__ float s_cos[R][kMaxHalf], s_sin[R][kMaxHalf];
  __shared__ float s_dg[kThreads / kWave][2][2 * kMaxHalf];
  float dga[2][8] = {}, dgb[2][8] = {};
  for (int t0 = blockIdx.x * R; t0 < a.M; t0 += gridDim.x * R) {
    const int rows = min(R, a.M - t0);
    __syncthreads();
    for (int i = threadIdx.x; i < R * half; i += kThreads) {
      const int j = i % half, t = min(t0 + i / half, a.M - 1);
      double sn, cs;
      sincos(static_cast<double>(a.pos[t]) * a.omega[j], &sn, &cs);
      s_cos[i / half][j] = static_cast<float>(cs);
      s_sin[i / half][j] = static_cast<float>(sn);
    }
    // the rows' v are one stretch of dv
    for (int i = threadIdx.x; i < rows * nv; i += kThreads) {
      const int t = i / nv;
      *reinterpret_cast<u16x8_t*>(
          a.dqkv + (static_cast<int64_t>(t0 + t) * H + a.Hq + a.Hkv) * a.D +
          (i - t * nv) * 8) =
          *reinterpret_cast<const u16x8_t*>(
              a.dv + static_cast<int64_t>(t0) * a.Hkv * a.D + i * 8);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * n_items; i += kThreads) {
      const int tr = i / n_items, head = (i - tr * n_items) / per_head;
      const int64_t t = t0 + tr;
      const bool isq = head < a.Hq;
      const int64_t o = (t * H + head) * a.D + j0;
      const uint16_t* dp = (isq ? a.dq + (t * a.Hq + head) * a.D
                                : a.dk + (t * a.Hkv + head - a.Hq) * a.D) + j0;
      const uint16_t* gp = (isq ? a.gq : a.gk) + j0;
      const u16x8_t xl = *reinterpret_cast<const u16x8_t*>(a.qkv + o);
      const u16x8_t xh = *reinterpret_cast<const u16x8_t*>(a.qkv + o + half);
      const u16x8_t dl = *reinterpret_cast<const u16x8_t*>(dp);
      const u16x8_t dh = *reinterpret_cast<const u16x8_t*>(dp + half);
      const u16x8_t gl = *reinterpret_cast<const u16x8_t*>(gp);
      const u16x8_t gh = *reinterpret_cast<const u16x8_t*>(gp + half);
      float x[8], y[8], za[8], zb[8], ss = 0.f, dot = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = bf16_to_f32(xl[e]);
        y[e] = bf16_to_f32(xh[e]);
        const float lo = bf16_to_f32(dl[e]), hi = bf16_to_f32(dh[e]);
        const float cs = s_cos[tr][j0 + e], sn = s_sin[tr][j0 + e];
        za[e] = lo * cs + hi * sn;
        zb[e] = hi * cs - lo * sn;
        ss += x[e] * x[e] + y[e] * y[e];
        dot += za[e] * bf16_to_f32(gl[e]) * x[e] +
               zb[e] * bf16_to_f32(gh[e]) * y[e];
      }
      for (int off = 1; off < per_head; off <<= 1) {
        ss += __shfl_xor(ss, off);
        dot += __shfl_xor(dot, off);
      }
      const float r = 1.0f / sqrtf(ss / static_cast<float>(a.D) + a.eps);
      const float k = dot * r / static_cast<float>(a.D) * r;
      u16x8_t ol, oh;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float ga = za[e] * (x[e] * r), gb = zb[e] * (y[e] * r);
        dga[0][e] += isq ? ga : 0.f;
        dgb[0][e] += isq ? gb : 0.f;
        dga[1][e] += isq ? 0.f : ga;
        dgb[1][e] += isq ? 0.f : gb;
        ol[e] = to_bf16(r * (za[e] * bf16_to_f32(gl[e]) - x[e] * k));
        oh[e] = to_bf16(r * (zb[e] * bf16_to_f32(gh[e]) - y[e] * k));
      }
      *reinterpret_cast<u16x8_t*>(a.dqkv + o) = ol;
      *reinterpret_cast<u16x8_t*>(a.dqkv + o + half) = oh;
    }
  }
  if (!a.part) return;
  // lanes of equal j0 (all values a step at a time: the kernel on 512 rows of
  // 4/2 heads of 64 7.7 us, one value after the other 10.4), then the waves
  for (int off = per_head; off < kWave; off <<= 1)
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dga[s][e] += __shfl_xor(dga[s][e], off);
        dgb[s][e] += __shfl_xor(dgb[s][e], off);
      }
  if (lane_id() < per_head)
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s_dg[threadIdx.x / kWave][s][j0 + e] = dga[s][e];
        s_dg[threadIdx.x / kWave][s][half + j0 + e] = dgb[s][e];
      }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.D; i += kThreads) {
    const int s = i / a.D, d = i % a.D;
    a.part[static_cast<int64_t>(blockIdx.x) * 2 * a.D + i] =
        (s_dg[0][s][d] + s_dg[1][s][d]) + (s_dg[2][s][d] + s_dg[3][s][d]);
  }
}

bool aligned(std::initializer_list<const void*> ps, int bytes) {
  for (const void* p : ps)
    if (reinterpret_cast<uintptr_t>(p) % bytes != 0) return false;
  return true;
}

bool norm_ok(int M, int Hd) {
  return M >= 1 && Hd >= 4 && Hd <= 1 << 20 && Hd % 4 == 0;
}
// Workgroups of the RMSNorm kernel, each with its part of the gain's gradient:
// four per CU for many rows of up to 4096 (32768 x 4096 249 us in a graph; 512
// workgroups 279, 2048 276), two for longer ones, whose registers hold no more
// (4096 x 8192 78 us; 2048 workgroups 103), and two rows each where they are
// few, for fewer parts to add up (1024 x 4096 15.5 us; a row each 18.7; 512 x
// 16384 31.9, 40.5; 2048 x 1024 10.3 with 512 workgroups, 11.2 with 1024).  All
// without a residual gradient; with one 32768 x 4096 takes 338 us.
int norm_parts(int M, int Hd) {
  const int most = M < 4096 || Hd > 4096 ? 512 : 1024;
  return std::min({M, most, std::max(256, M - M / 2)});
}

// Rows that a workgroup of the q/k kernel takes at once.  Four, so that its
// threads have work (512 rows of 4/2 heads of 64, 24 items each, 7.8 us; one
// row 9.0), but one where four have more items than threads and there is not a
// workgroup per CU (512 rows of 32/8 heads of 128, 320 items, 10.7 us; four
// 13.4; 1024 rows 18.7, 15.5; 32768 rows 282, 229).  Eight of few items, two
// workgroups per CU (4096 rows of 4/2 heads of 64 10.4 us; four 14.0; 32768 of
// 16/2 49.6, 54.5; 8192 of 32/8 heads of 128 59.7, 57.5).
int qk_rows(int M, int items) {
  if (items <= 96 && M >= 8 * 512) return 8;
  return M >= 4 * 256 || 4 * items <= kThreads ? 4 : 1;
}
int qk_items(int Hq, int Hkv, int D) { return (Hq + Hkv) * (D / 16); }
int qk_parts(int M, int items) {
  return std::min((M - 1) / qk_rows(M, items) + 1, kQkParts);
}

// 64 columns per workgroup read 256 bytes together (1024 parts of 4096 5.6 us;
// 16 columns 7.2); few columns would leave most CUs idle (2048 parts of 256
// 11.8 us; 16 columns 8.4).
int sum_parts(const float* part, int parts, int n0, int n1, float* out0,
              float* out1, hipStream_t st) {
  const int n = n0 + n1, cols = n <= 256 ? 16 : 64;
  hipLaunchKernelGGL(cols == 16 ? sum_parts_kernel<16> : sum_parts_kernel<64>,
                     dim3((n + cols - 1) / cols), dim3(kSumThreads), 0, st,
                     part, parts, n0, n1, out0, out1);
  WEDLM_LAUNCH_CHECK();
  return WEDLM_OK;
}

bool qk_ok(int M, int Hq, int Hkv, int D) {
  return M >= 1 && Hq >= 1 && Hkv >= 1 && (D == 64 || D == 128) &&
         (Hq + 2ll * Hkv) * D <= 0x7fffffff / 8;
}

}  // namespace

extern "C" size_t wedlm_rmsnorm_backward_workspace_size(int32_t M, int32_t Hd) {
  if (!norm_ok(M, Hd)) return 0;
  return static_cast<size_t>(norm_parts(M, Hd)) * Hd * sizeof(float);
}

extern "C" int wedlm_rmsnorm_backward(const float* x, const uint16_t* gain,
                                      const uint16_t* dy, const float* dres,
                                      int32_t M, int32_t Hd, float eps,
                                      float* dx, float* dgain, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  if (!x || !gain || !dy || !dx || !(eps > 0.f)) return WEDLM_E_ARG;
  if (!aligned({x, dres, dx, workspace}, 16) || !aligned({gain, dy}, 8))
    return WEDLM_E_ARG;
  if (!norm_ok(M, Hd)) return WEDLM_E_SHAPE;
  if (dgain && (!workspace ||
                workspace_bytes < wedlm_rmsnorm_backward_workspace_size(M, Hd)))
    return WEDLM_E_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  float* part = dgain ? static_cast<float*>(workspace) : nullptr;
  const int parts = norm_parts(M, Hd), nc = Hd / 4;
  auto k = nc <= kThreads        ? rmsnorm_backward_kernel<1>
           : nc <= 2 * kThreads  ? rmsnorm_backward_kernel<2>
           : nc <= 3 * kThreads  ? rmsnorm_backward_kernel<3>
           : nc <= 4 * kThreads  ? rmsnorm_backward_kernel<4>
           : nc <= 8 * kThreads  ? rmsnorm_backward_kernel<8>
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
  return static_cast<size_t>(qk_parts(M, qk_items(Hq, Hkv, D))) * 2 * D *
         sizeof(float);
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
  if (!aligned({qkv, q_gain, k_gain, dq, dk, dv, dqkv}, 16)) return WEDLM_E_ARG;
  if (!qk_ok(M, Hq, Hkv, D)) return WEDLM_E_SHAPE;
  const bool gains = dq_gain || dk_gain;
  if (gains && !aligned({workspace}, alignof(float))) return WEDLM_E_ARG;
  if (gains && (!workspace ||
                workspace_bytes <
                    wedlm_qk_norm_rope_backward_workspace_size(M, Hq, Hkv, D)))
    return WEDLM_E_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  float* part = gains ? static_cast<float*>(workspace) : nullptr;
  QkArgs a{qkv, q_gain, k_gain, pos_ids, dq, dk, dv, dqkv, part, M, Hq, Hkv,
           D, eps, {}};
  // theta^(-2 j / D) as products of two powers, not one power each: they cost
  // the host as much as a launch.  Three roundings: off by 3 2^-53 at most beside
  // pow()'s own error (found: 1.3 2^-52)
  double low[8], high[kMaxHalf / 8];
  for (int j = 0; j < 8; ++j) low[j] = std::pow(rope_theta, -2.0 * j / D);
  for (int j = 0; j < D / 16; ++j) high[j] = std::pow(rope_theta, -16.0 * j / D);
  for (int j = 0; j < D / 2; ++j) a.omega[j] = high[j / 8] * low[j % 8];
  const int items = qk_items(Hq, Hkv, D), parts = qk_parts(M, items);
  const int rows = qk_rows(M, items);
  auto k = rows == 8   ? qk_norm_rope_backward_kernel<8>
           : rows == 4 ? qk_norm_rope_backward_kernel<4>
                       : qk_norm_rope_backward_kernel<1>;
  hipLaunchKernelGGL(k, dim3(parts), dim3(kThreads), 0, st, a);
  WEDLM_LAUNCH_CHECK();
  return gains ? sum_parts(part, parts, D, D, dq_gain, dk_gain, st) : WEDLM_OK;
}
