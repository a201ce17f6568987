// The window attention over a paged cache of e4m3 codes with one power-of-two
// scale per page and kv head (wedlm_window_attn_cache8).
//
// Query rows of one kv head are packed as in the bf16 kernel (row r = i*G + j
// is window row i, query head kvh*G + j); a wave owns 32 of them and walks
// 32-key tiles (two pages).  S^T = K Q^T and O^T += V^T P^T run on
// v_mfma_f32_32x32x16_bf16: e4m3 values are exact in bf16, so the codes are
// converted on the way into the products and nothing else is rounded than
// over a bf16 cache.
// Orders.  A lane's 16 bytes of a key row are 16 values of d: the K and Q
// operands take d in that order (products do not care), so a lane reads whole
// 16-byte pieces.  Score rows are the keys in the order that leaves lane
// half hf with the 16 keys of page hf: its K scale is then one factor per
// lane, folded into the softmax's, and its 16 weights meet the 16 bytes of a
// V^T row of that page, whose scale the conversion applies.
// Softmax, split of the prefix and its merge are those of the bf16 kernel.
#include "common.h"
#include "wedlm_serve.h"

using namespace wedlm;

namespace {

constexpr int kTileKeys = 32;       // keys per tile (two 16-token pages)
// A prefix split holds at least this many tiles.
constexpr int kMinSplitTiles = 8;
constexpr float kLn2 = 0.69314718055994530942f;

struct Args {
  const uint16_t* q;      // [B, W, Hq, D]
  const uint16_t* kw;     // [B, W, Hkv, D]
  const uint16_t* vw;
  const uint8_t* k8;      // [P, Hkv, 16, D]
  const uint8_t* v8;      // [P, Hkv, D, 16]
  const uint8_t* ke;      // [P, Hkv]
  const uint8_t* ve;
  const int32_t* bt;      // [B, max_pages]
  const int32_t* plen;    // [B]
  uint16_t* out;          // [B, W, Hq, D]
  float* lse;             // [B, W, Hq] or null
  int32_t* status;        // [B] or null
  uint16_t* ws_o;         // [B, Hkv, rows_pad, nsplit, D]
  float2* ws_ml;          // [B, Hkv, rows_pad, nsplit]
  int num_pages, B, W, Hq, Hkv, G, max_pages, max_prefix, nsplit, qgroups,
      rows_pad;
  float scale_log2;       // softmax_scale * log2(e)
};

struct Plan {
  int nw, qgroups, rows_pad, nsplit;
  size_t ws_bytes;
};

Plan make_plan(int B, int W, int Hq, int Hkv, int D, int max_prefix) {
  Plan p{};
  const int rows = W * (Hq / Hkv);
  const int blocks = (rows + 31) / 32;
  p.nw = blocks < 8 ? blocks : 8;
  p.qgroups = (blocks + p.nw - 1) / p.nw;
  p.rows_pad = p.qgroups * p.nw * 32;
  const int tiles = (max_prefix + kTileKeys - 1) / kTileKeys;
  const int64_t waves = static_cast<int64_t>(B) * Hkv * p.qgroups * p.nw;
  // about eight waves a CU
  int64_t n = (2048 + waves - 1) / waves;
  const int most = tiles / kMinSplitTiles;
  if (n > most) n = most;
  if (n < 1) n = 1;
  p.nsplit = static_cast<int>(n);
  if (p.nsplit > 1) {
    const size_t r = static_cast<size_t>(B) * Hkv * p.rows_pad * p.nsplit;
    p.ws_bytes = ((r * D * sizeof(uint16_t) + 255) & ~static_cast<size_t>(255)) +
                 r * sizeof(float2);
  }
  return p;
}

__device__ __forceinline__ bool len_ok(const Args& a, int c) {
  return c >= 0 && c <= a.max_prefix &&
         static_cast<int64_t>(c) <= static_cast<int64_t>(a.max_pages) * kPage;
}

// Split of one sequence's prefix of c positions over the launch's nsplit
// slots: as many splits as keep kMinSplitTiles tiles each (one for an empty
// prefix), each of the same whole number of tiles.  From the sequence's own c,
// so that a max_prefix_len far above it leaves no split empty.
struct SeqSplit {
  int n, len;             // splits in use, positions per split
};

__device__ __forceinline__ SeqSplit seq_split(int c, int nsplit) {
  const int tiles = c / kTileKeys + (c % kTileKeys != 0 ? 1 : 0);
  const int n = max(1, min(tiles / kMinSplitTiles, nsplit));
  const int per = max(1, (tiles + n - 1) / n);
  SeqSplit r;
  r.len = per * kTileKeys;
  r.n = c > 0 ? (tiles + per - 1) / per : 1;
  return r;
}

// Values of x in this lane and in the lane 32 away.
__device__ __forceinline__ void xor32_pair(float x, float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x),
                                                  __float_as_uint(x), false,
                                                  false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}

// Eight e4m3 codes as bf16, times a power of two.
__device__ __forceinline__ bf16x8_t widen(uint32_t lo, uint32_t hi,
                                          float scale) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 2^(e - 127) of a scale's exponent (1 .. 254).
__device__ __forceinline__ float scale_of(int e) {
  return __uint_as_float(static_cast<uint32_t>(e) << 23);
}

template <int D>
__global__ __launch_bounds__(8 * kWave)
void window_attn8_kernel(Args a) {
  constexpr int NJ = D / 32;          // 16-byte pieces of a key row per half
  constexpr int NK = D / 16;          // k-steps of the score MFMA
  constexpr int NM = D / 32;          // 32-row blocks of O^T

  int wg = blockIdx.x;
  const int split = wg % a.nsplit;
  wg /= a.nsplit;
  const int qg = wg % a.qgroups;
  wg /= a.qgroups;
  const int kvh = wg % a.Hkv;
  const int b = wg / a.Hkv;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int nw = blockDim.x / kWave;
  const int lane = lane_id();
  const int col = lane & 31, hf = lane >> 5;
  const int rows = a.W * a.G;
  const int rb = (qg * nw + wave) * 32;

  const int c = a.plen[b];
  if (!len_ok(a, c)) {
    if (a.status && threadIdx.x == 0 && split == 0 && qg == 0 && kvh == 0)
      atomicOr(a.status + b, WEDLM_SEQ_BAD_LEN);
    return;
  }
  const SeqSplit ss = seq_split(c, a.nsplit);
  if (split >= ss.n || rb >= rows) return;
  const int k0 = split * ss.len;
  const int k1 = min(c, k0 + ss.len);
  const bool last = split == ss.n - 1;

  // ---- queries
  const int r = rb + col;
  const bool rvalid = r < rows;
  const int qi = rvalid ? r / a.G : 0;
  const int qh = kvh * a.G + (rvalid ? r % a.G : 0);
  const uint16_t* qp =
      a.q + ((static_cast<int64_t>(b) * a.W + qi) * a.Hq + qh) * D;
  bf16x8_t qf[NK];
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i)
      qf[2 * j + i] = __builtin_bit_cast(
          bf16x8_t,
          *reinterpret_cast<const u16x8_t*>(qp + 32 * j + 16 * hf + 8 * i));

  floatx16_t o[NM];
#pragma unroll
  for (int m = 0; m < NM; ++m)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[m][e] = 0.f;
  float m2 = kNegInf, l_run = 0.f;

  // MFMA output row m holds the scores of this key of the tile
  const int key = 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3);

  auto rescale = [&](float alpha) {
    l_run *= alpha;
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[m][e] *= alpha;
  };
  // one tile's weights and products; x: scores in log2 units
  auto finish = [&](float (&x)[16], const bf16x8_t (&vf)[2][NM], bool first) {
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, x[e]);
    float x0, x1;
    xor32_pair(mx, x0, x1);
    mx = fmaxf(x0, x1);
    if (ballot(mx > m2)) {
      const float m_new = fmaxf(m2, mx);
      rescale(m2 == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m2 - m_new));
      m2 = m_new;
    }
    const float mc = m2 == kNegInf ? 0.f : m2;
    bf16x8_t pf[2];
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float p = __builtin_amdgcn_exp2f(x[e] - mc);
      sum += p;
      pf[e >> 3][e & 7] = static_cast<__bf16>(p);
    }
    l_run += sum;
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
      for (int m = 0; m < NM; ++m)
        o[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[h2][m], pf[h2], o[m],
                                                       0, 0, 0);
  };

  // ---- the prefix
  const int32_t* btb = a.bt + static_cast<int64_t>(b) * a.max_pages;
  bool pages_ok = true;
  for (int base = k0; base < k1; base += kTileKeys) {
    int id[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int p = base / kPage + h;
      id[h] = base + h * kPage < k1 ? btb[p] : 0;
      const bool ok = id[h] >= 0 && id[h] < a.num_pages;
      pages_ok = pages_ok && ok;
      id[h] = ok ? id[h] : 0;
    }
    const int64_t kpage =
        static_cast<int64_t>(id[(col >> 2) & 1]) * a.Hkv + kvh;
    const int64_t vpage = static_cast<int64_t>(id[hf]) * a.Hkv + kvh;
    u32x4_t kr[NJ], vr[NM];
    const uint8_t* kp = a.k8 + (kpage * kPage + (key & 15)) * D + 16 * hf;
    const uint8_t* vp = a.v8 + (vpage * D + col) * kPage;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      kr[j] = *reinterpret_cast<const u32x4_t*>(kp + 32 * j);
#pragma unroll
    for (int m = 0; m < NM; ++m)
      vr[m] = *reinterpret_cast<const u32x4_t*>(vp + 32 * m * kPage);
    // keys of this lane's page that are in the prefix
    const int n = min(max(k1 - base - 16 * hf, 0), kPage);
    // (a page without any may hold any scale)
    const float ks = n > 0 ? scale_of(a.ke[vpage]) : 1.f;
    const float vs = n > 0 ? scale_of(a.ve[vpage]) : 1.f;
    floatx16_t s = {};
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            widen(kr[j][2 * i], kr[j][2 * i + 1], 1.f), qf[2 * j + i], s, 0, 0,
            0);
    float x[16];
    const float f = a.scale_log2 * ks;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = e < n ? s[e] * f : kNegInf;
    // codes behind the prefix count as zero
    uint32_t mask[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int k = min(max(n - 4 * w, 0), 4);
      mask[w] = k == 4 ? ~0u : (1u << (8 * k)) - 1;
    }
    bf16x8_t vf[2][NM];
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
      for (int m = 0; m < NM; ++m)
        vf[h2][m] = widen(vr[m][2 * h2] & mask[2 * h2],
                          vr[m][2 * h2 + 1] & mask[2 * h2 + 1], vs);
    finish(x, vf, false);
  }

  // ---- the window, with the last split
  if (last) {
    const int64_t wrow = static_cast<int64_t>(b) * a.W;
    for (int base = 0; base < a.W; base += kTileKeys) {
      const int kk = base + key;
      const uint16_t* kp = a.kw + ((wrow + min(kk, a.W - 1)) * a.Hkv + kvh) * D;
      floatx16_t s = {};
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              __builtin_bit_cast(bf16x8_t,
                                 *reinterpret_cast<const u16x8_t*>(
                                     kp + 32 * j + 16 * hf + 8 * i)),
              qf[2 * j + i], s, 0, 0, 0);
      float x[16];
      const int at = base + 16 * hf;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        x[e] = at + e <= qi ? s[e] * a.scale_log2 : kNegInf;
      bf16x8_t vf[2][NM];
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
        for (int m = 0; m < NM; ++m) {
          u16x8_t v;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int kv = at + 8 * h2 + e;
            v[e] = kv < a.W ? a.vw[((wrow + kv) * a.Hkv + kvh) * D + 32 * m +
                                   col]
                            : static_cast<uint16_t>(0);
          }
          vf[h2][m] = __builtin_bit_cast(bf16x8_t, v);
        }
      finish(x, vf, false);
    }
  }

  if (!pages_ok && a.status && lane == 0)
    atomicOr(a.status + b, WEDLM_SEQ_BAD_PAGE);

  float l0, l1;
  xor32_pair(l_run, l0, l1);
  const float l_tot = l0 + l1;
  if (!rvalid) return;
  const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
  const int64_t part =
      ((static_cast<int64_t>(b) * a.Hkv + kvh) * a.rows_pad + r) * a.nsplit +
      split;
  const int64_t orow = (static_cast<int64_t>(b) * a.W + qi) * a.Hq + qh;
  uint16_t* op = a.nsplit == 1 ? a.out + orow * D : a.ws_o + part * D;
#pragma unroll
  for (int m = 0; m < NM; ++m)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const u16x4_t v = {to_bf16(o[m][4 * g] * inv),
                         to_bf16(o[m][4 * g + 1] * inv),
                         to_bf16(o[m][4 * g + 2] * inv),
                         to_bf16(o[m][4 * g + 3] * inv)};
      *reinterpret_cast<u16x4_t*>(op + m * 32 + g * 8 + hf * 4) = v;
    }
  if (hf == 0) {
    if (a.nsplit > 1)
      a.ws_ml[part] = make_float2(m2, l_tot);
    else if (a.lse)
      a.lse[orow] = (m2 + __log2f(l_tot)) * kLn2;
  }
}

// Merge of the splits' outputs: O = sum_s 2^(m_s - M) l_s O_s / sum_s
// 2^(m_s - M) l_s, O_s normalised by l_s.  D/8 threads a row, 16 bytes of a
// split each; a row's threads take its splits in order.
constexpr int kMergeThreads = 256;

template <int D>
__global__ __launch_bounds__(kMergeThreads) void merge8_kernel(Args a) {
  constexpr int TPR = D / 8;
  const int rows = a.W * a.G;
  const int64_t gr = (static_cast<int64_t>(blockIdx.x) * kMergeThreads +
                      threadIdx.x) / TPR;
  if (gr >= static_cast<int64_t>(a.B) * a.Hkv * rows) return;
  const int r = static_cast<int>(gr % rows);
  const int64_t bk = gr / rows;
  const int kvh = static_cast<int>(bk % a.Hkv), b = static_cast<int>(bk / a.Hkv);
  const int d = (threadIdx.x % TPR) * 8;
  const int c = a.plen[b];
  if (!len_ok(a, c)) return;
  const int n = seq_split(c, a.nsplit).n;
  const int64_t part = (bk * a.rows_pad + r) * a.nsplit;
  const float2* ml = a.ws_ml + part;
  const uint16_t* op = a.ws_o + part * D + d;
  float M = kNegInf;
  for (int s = 0; s < n; ++s) M = fmaxf(M, ml[s].x);
  const float base = M == kNegInf ? 0.f : M;
  float L = 0.f, acc[8] = {};
#pragma unroll 4
  for (int s = 0; s < n; ++s) {
    const float w = __builtin_amdgcn_exp2f(ml[s].x - base) * ml[s].y;
    const u16x8_t v =
        *reinterpret_cast<const u16x8_t*>(op + static_cast<int64_t>(s) * D);
    L += w;
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[k] += w * bf16_to_f32(v[k]);
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;
  u16x8_t v;
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = to_bf16(acc[k] * inv);
  const int64_t orow = (static_cast<int64_t>(b) * a.W + r / a.G) * a.Hq +
                       kvh * a.G + r % a.G;
  *reinterpret_cast<u16x8_t*>(a.out + orow * D + d) = v;
  if (a.lse && d == 0) a.lse[orow] = (M + __log2f(L)) * kLn2;
}

bool shape_ok(int B, int W, int Hq, int Hkv, int D, int max_prefix) {
  if (!(B >= 1 && W >= 1 && W <= WEDLM_MAX_WINDOW && Hkv >= 1 && Hq >= Hkv &&
        Hq % Hkv == 0 && (D == 64 || D == 128) && max_prefix >= 0))
    return false;
  // rows, padded to whole workgroups, and their workgroups fit 31 bits
  const int64_t rows = static_cast<int64_t>(W) * (Hq / Hkv) + 255;
  return rows < (1ll << 31) / Hkv && rows * Hkv < (1ll << 31) / B;
}

bool aligned(const void* p, size_t n) {
  return reinterpret_cast<uintptr_t>(p) % n == 0;
}

}  // namespace

extern "C" size_t wedlm_window_attn_cache8_workspace_size(
    int32_t B, int32_t W, int32_t Hq, int32_t Hkv, int32_t D,
    int32_t max_prefix_len) {
  if (!shape_ok(B, W, Hq, Hkv, D, max_prefix_len)) return 0;
  return make_plan(B, W, Hq, Hkv, D, max_prefix_len).ws_bytes;
}

extern "C" int wedlm_window_attn_cache8(
    const uint16_t* q_phys, const uint16_t* k_phys, const uint16_t* v_phys,
    const uint8_t* k8, const uint8_t* v8, const uint8_t* k_exp,
    const uint8_t* v_exp, int64_t num_pages, const int32_t* block_table,
    int32_t max_pages, const int32_t* prefix_len, int32_t B, int32_t W,
    int32_t Hq, int32_t Hkv, int32_t D, int32_t max_prefix_len,
    float softmax_scale, uint16_t* out, float* lse, int32_t* status,
    void* workspace, size_t workspace_bytes, void* stream) {
  if (!q_phys || !k_phys || !v_phys || !block_table || !prefix_len || !out)
    return WEDLM_E_ARG;
  if (!shape_ok(B, W, Hq, Hkv, D, max_prefix_len)) return WEDLM_E_SHAPE;
  if (max_prefix_len > 0 && (!k8 || !v8 || !k_exp || !v_exp || num_pages < 1 ||
                             max_pages < 1))
    return WEDLM_E_ARG;
  if (num_pages >= (1ll << 31)) return WEDLM_E_SHAPE;
  if (!(softmax_scale > 0.f) || !(softmax_scale < 1e30f)) return WEDLM_E_ARG;
  if (!aligned(q_phys, 16) || !aligned(k_phys, 16) || !aligned(v_phys, 16) ||
      !aligned(k8, 16) || !aligned(v8, 16) || !aligned(out, 16))
    return WEDLM_E_ARG;
  const Plan p = make_plan(B, W, Hq, Hkv, D, max_prefix_len);
  if (workspace_bytes < p.ws_bytes || (p.ws_bytes && !workspace))
    return WEDLM_E_WORKSPACE;
  if (p.ws_bytes && !aligned(workspace, 256)) return WEDLM_E_ARG;
  Args a{};
  a.q = q_phys; a.kw = k_phys; a.vw = v_phys; a.k8 = k8; a.v8 = v8;
  a.ke = k_exp; a.ve = v_exp; a.bt = block_table; a.plen = prefix_len;
  a.out = out; a.lse = lse; a.status = status;
  a.num_pages = static_cast<int>(num_pages);
  a.B = B; a.W = W; a.Hq = Hq; a.Hkv = Hkv; a.G = Hq / Hkv;
  a.max_pages = max_pages; a.max_prefix = max_prefix_len;
  a.nsplit = p.nsplit; a.qgroups = p.qgroups; a.rows_pad = p.rows_pad;
  a.scale_log2 = softmax_scale * 1.4426950408889634f;
  if (p.nsplit > 1) {
    const size_t n = static_cast<size_t>(B) * Hkv * p.rows_pad * p.nsplit;
    char* base = static_cast<char*>(workspace);
    a.ws_o = reinterpret_cast<uint16_t*>(base);
    a.ws_ml = reinterpret_cast<float2*>(
        base + ((n * D * sizeof(uint16_t) + 255) & ~static_cast<size_t>(255)));
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t grid = static_cast<int64_t>(p.nsplit) * B * Hkv * p.qgroups;
  if (D == 128)
    hipLaunchKernelGGL(window_attn8_kernel<128>,
                       dim3(static_cast<unsigned>(grid)), dim3(p.nw * kWave),
                       0, st, a);
  else
    hipLaunchKernelGGL(window_attn8_kernel<64>,
                       dim3(static_cast<unsigned>(grid)), dim3(p.nw * kWave),
                       0, st, a);
  WEDLM_LAUNCH_CHECK();
  if (p.nsplit > 1) {
    const int64_t threads = static_cast<int64_t>(B) * W * Hq * (D / 8);
    const dim3 mg(static_cast<unsigned>((threads + kMergeThreads - 1) /
                                        kMergeThreads));
    if (D == 128)
      hipLaunchKernelGGL(merge8_kernel<128>, mg, dim3(kMergeThreads), 0, st, a);
    else
      hipLaunchKernelGGL(merge8_kernel<64>, mg, dim3(kMergeThreads), 0, st, a);
    WEDLM_LAUNCH_CHECK();
  }
  return WEDLM_OK;
}
