// Rows appended to the 8-bit paged cache: e4m3 codes, one power-of-two scale
// per page and kv head (wedlm_cache8_append, wedlm_commit_cache8).
//
// One wave per (layer, sequence, kv head) and page, or window.  The rows' largest finite
// magnitude is an integer maximum over the bf16 patterns without their sign;
// the exponent is read off that pattern, so the scale is exact and does not
// depend on any rounding.  x * 2^(127 - e) is exact in fp32 and rounded once,
// to e4m3.
// Bound by HBM where rows are many (4 x 1024 rows of 8 layers, 8 heads of 128:
// 169 MB in 33 us, 5.1 TB/s); by latency where a step commits a few tokens (16 x
// 4 rows of 36 layers: 12 us): the chain is start/count, block table with the
// rows, the page's old V bytes with its exponents, K's old codes where the
// scale grows, stores; from the block table on once more for a run that crosses
// into the next page.
#include "common.h"
#include "internal.h"
#include "wedlm_serve.h"

using namespace wedlm;

namespace {

constexpr int kWavesPerGroup = 4;

struct AppendArgs {
  const uint16_t* k;      // [L, B, T, Hkv, D]
  const uint16_t* v;
  const int32_t* start;   // [B]
  const int32_t* count;   // [B]
  const int32_t* bt;      // [B, max_pages]
  uint8_t* k8;            // [L, P, Hkv, 16, D]
  uint8_t* v8;            // [L, P, Hkv, D, 16]
  uint8_t* ke;            // [L, P, Hkv]
  uint8_t* ve;
  int32_t* status;        // [B] or null
  int64_t num_pages;
  int L, B, T, Hkv, max_pages;
  int spans;              // pages that a sequence's rows can touch
  int run, runs;          // pages of a wave; waves for them
  uint32_t units;         // waves
  int behind;             // start is the position behind the last row
};

// Smallest exponent >= 1 whose 448 * 2^(e - 127) holds the bf16 magnitude a
// (a finite pattern without its sign): 448 = 1.75 * 2^8.
__device__ __forceinline__ int need_exp(int a) {
  const int e = (a >> 7) - 8 + ((a & 0x7f) > 0x60 ? 1 : 0);
  return max(e, 1);
}

// Largest finite magnitude of eight bf16 values, with m.
__device__ __forceinline__ int mag_max(u16x8_t x, int m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int a = x[i] & 0x7fff;
    m = max(m, a < 0x7f80 ? a : 0);
  }
  return m;
}

__device__ __forceinline__ int wave_max_int(int v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = max(v, __shfl_xor(v, off));
  return v;
}

// Two e4m3 codes (in the low half) of a * 2^s, b * 2^s; what is not finite
// becomes NaN (the format has no infinity).
__device__ __forceinline__ uint32_t pack2(float a, float b, int s) {
  const float nan = __builtin_nanf("");
  a = __builtin_fabsf(a) < __builtin_huge_valf() ? a : nan;
  b = __builtin_fabsf(b) < __builtin_huge_valf() ? b : nan;
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(
             __builtin_amdgcn_ldexpf(a, s), __builtin_amdgcn_ldexpf(b, s), 0,
             false)) & 0xffffu;
}

__device__ __forceinline__ uint2 pack8(u16x8_t x, int s) {
  uint2 r;
  r.x = pack2(bf16_to_f32(x[0]), bf16_to_f32(x[1]), s) |
        pack2(bf16_to_f32(x[2]), bf16_to_f32(x[3]), s) << 16;
  r.y = pack2(bf16_to_f32(x[4]), bf16_to_f32(x[5]), s) |
        pack2(bf16_to_f32(x[6]), bf16_to_f32(x[7]), s) << 16;
  return r;
}

// Four codes at another scale: value * 2^s, rounded again.
__device__ __forceinline__ uint32_t again4(uint32_t c, int s) {
  return pack2(__builtin_amdgcn_cvt_f32_fp8(c, 0),
               __builtin_amdgcn_cvt_f32_fp8(c, 1), s) |
         pack2(__builtin_amdgcn_cvt_f32_fp8(c, 2),
               __builtin_amdgcn_cvt_f32_fp8(c, 3), s) << 16;
}

// Bytes lo .. hi-1 of a 16-byte vector, as masks of its words.
__device__ __forceinline__ uint32_t byte_mask(int word, int lo, int hi) {
  const int a = min(max(lo - 4 * word, 0), 4), b = min(max(hi - 4 * word, 0), 4);
  const uint32_t below_b = b == 4 ? ~0u : (1u << (8 * b)) - 1;
  const uint32_t below_a = a == 4 ? ~0u : (1u << (8 * a)) - 1;
  return below_b & ~below_a;
}

// The four words of a 4 x 4 transpose of bytes: byte j of word i is byte i of
// word j.
__device__ __forceinline__ void transpose4(uint32_t (&w)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400);
  const uint32_t b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400);
  const uint32_t c = __builtin_amdgcn_perm(w[1], w[0], 0x07030602);
  const uint32_t d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
  w[0] = __builtin_amdgcn_perm(b, a, 0x05040100);
  w[1] = __builtin_amdgcn_perm(b, a, 0x07060302);
  w[2] = __builtin_amdgcn_perm(d, c, 0x05040100);
  w[3] = __builtin_amdgcn_perm(d, c, 0x07060302);
}

// 16-byte row dd of V^T in LDS: its eight neighbours' order is changed from one
// group of eight to the next, so that lanes that write row k of their groups
// meet different banks.
__device__ __forceinline__ int vt_row(int dd) { return dd ^ (dd >> 3 & 7); }

// The page `span` of sequence b's rows, layer l, head h: one wave.
template <int D>
__device__ __forceinline__ void append_page(const AppendArgs& a, int l, int b,
                                            int h, int span, int n, int64_t s0,
                                            uint8_t* vt) {
  constexpr int LPR = D / 8;            // lanes per row, 8 values each
  constexpr int NI = kPage * LPR / kWave;   // rows of a lane: NI r .. NI r+NI-1
  const int lane = lane_id();
  const int64_t page0 = (s0 / kPage + span) * kPage;     // its first position
  const int r0 = static_cast<int>(max(s0 - page0, static_cast<int64_t>(0)));
  const int r1 = static_cast<int>(
      min(s0 + n - page0, static_cast<int64_t>(kPage)));
  if (r1 <= r0) return;
  const bool tell = a.status && l == 0 && h == 0 && lane == 0;
  const int64_t entry = page0 / kPage;
  if (entry >= a.max_pages) {
    if (tell) atomicOr(a.status + b, WEDLM_SEQ_CAPACITY);
    return;
  }
  // ---- the new rows, under the table's round trip
  const int row = lane / LPR * NI, d = (lane % LPR) * 8;
  u16x8_t xk[NI], xv[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const u16x8_t z = {0, 0, 0, 0, 0, 0, 0, 0};
    xk[i] = xv[i] = z;
    if (row + i >= r0 && row + i < r1) {
      const int64_t src =
          (((static_cast<int64_t>(l) * a.B + b) * a.T + (page0 + row + i - s0)) *
               a.Hkv + h) * D + d;
      xk[i] = *reinterpret_cast<const u16x8_t*>(a.k + src);
      xv[i] = *reinterpret_cast<const u16x8_t*>(a.v + src);
    }
  }
  const int64_t id = a.bt[static_cast<int64_t>(b) * a.max_pages + entry];
  if (id < 0 || id >= a.num_pages) {
    if (tell) atomicOr(a.status + b, WEDLM_SEQ_BAD_PAGE);
    return;
  }
  const int64_t ph = (l * a.num_pages + id) * a.Hkv + h;
  uint8_t* kp = a.k8 + ph * (kPage * D);
  uint8_t* vp = a.v8 + ph * (kPage * D);
  // what the page holds, where not all 16 rows are new
  constexpr int NV = D / kWave;
  u32x4_t old[NV];
  if (r1 - r0 < kPage) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      old[i] = *reinterpret_cast<const u32x4_t*>(vp + (i * kWave + lane) * kPage);
  }
  int ek0 = 0, ev0 = 0;
  if (r0 > 0) {
    ek0 = a.ke[ph];
    ev0 = a.ve[ph];
  }
  int mk = 0, mv = 0;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    mk = mag_max(xk[i], mk);
    mv = mag_max(xv[i], mv);
  }
  int ek = need_exp(wave_max_int(mk)), ev = need_exp(wave_max_int(mv));
  if (r0 > 0) {
    ek = max(ek, ek0);
    ev = max(ev, ev0);
  }
  if (lane == 0) {
    a.ke[ph] = static_cast<uint8_t>(ek);
    a.ve[ph] = static_cast<uint8_t>(ev);
  }

  // ---- keys: rows are contiguous
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int r = row + i;
    uint2* dst = reinterpret_cast<uint2*>(kp + r * D + d);
    if (r >= r0 && r < r1) {
      *dst = pack8(xk[i], 127 - ek);
    } else if (r < r0 && ek > ek0) {
      uint2 c = *dst;
      c.x = again4(c.x, ek0 - ek);
      c.y = again4(c.y, ek0 - ek);
      *dst = c;
    }
  }

  // ---- values: transposed, a lane's rows as one word (or half of one) of each
  // of its 8 d, through LDS to whole 16-byte rows of the page, merged with what
  // it holds
  uint2 c[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) c[i] = pack8(xv[i], 127 - ev);
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    uint32_t w[4] = {};
#pragma unroll
    for (int i = 0; i < NI; ++i) w[i] = half ? c[i].y : c[i].x;
    transpose4(w);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint8_t* at = vt + vt_row(d + 4 * half + k) * kPage + row;
      if constexpr (NI == 4) *reinterpret_cast<uint32_t*>(at) = w[k];
      else *reinterpret_cast<uint16_t*>(at) = static_cast<uint16_t>(w[k]);
    }
  }
  // the wave's own LDS writes are complete before its reads (in order)
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int dd = i * kWave + lane;
    u32x4_t v = *reinterpret_cast<const u32x4_t*>(vt + vt_row(dd) * kPage);
    if (r1 - r0 < kPage) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t fresh = byte_mask(q, r0, r1);
        uint32_t o = old[i][q];
        if (r0 > 0 && ev > ev0) {
          const uint32_t before = byte_mask(q, 0, r0);
          o = (again4(o, ev0 - ev) & before) | (o & ~before);
        }
        v[q] = (v[q] & fresh) | (o & ~fresh);
      }
    }
    *reinterpret_cast<u32x4_t*>(vp + dd * kPage) = v;
  }
  __builtin_amdgcn_wave_barrier();
}

// One wave per (sequence, layer, run of pages, kv head), kv heads fastest.
template <int D>
__global__ __launch_bounds__(kWavesPerGroup * kWave) void append8_kernel(
    AppendArgs a) {
  // a page's V^T, bytes, per wave
  __shared__ __attribute__((aligned(16))) uint8_t vt[kWavesPerGroup][D * kPage];
  const int wave = threadIdx.x / kWave;
  const uint32_t unit = blockIdx.x * kWavesPerGroup + wave;
  if (unit >= a.units) return;
  const int h = unit % a.Hkv;
  uint32_t w = unit / a.Hkv;
  const int run = w % a.runs;
  w /= a.runs;
  const int l = w % a.L, b = w / a.L;
  const int n = a.count[b];
  int64_t s0 = a.start[b];
  if (a.behind) s0 -= n;
  if (n < 0 || n > a.T || s0 < 0) {
    if (a.status && l == 0 && h == 0 && run == 0 && lane_id() == 0)
      atomicOr(a.status + b, WEDLM_SEQ_BAD_LEN);
    return;
  }
  const int end = min((run + 1) * a.run, a.spans);
  for (int span = run * a.run; span < end; ++span)
    append_page<D>(a, l, b, h, span, n, s0, vt[wave]);
}

bool aligned(const void* p, size_t n) {
  return reinterpret_cast<uintptr_t>(p) % n == 0;
}

// The sizes' checks of both entry points.
int append_shape(int64_t L, int64_t B, int64_t T, int64_t Hkv, int32_t D,
                 int64_t num_pages, int32_t max_pages, int64_t* units) {
  if (L < 1 || B < 1 || T < 1 || Hkv < 1 || (D != 64 && D != 128) ||
      num_pages < 1 || num_pages >= (1ll << 31) || max_pages < 1)
    return WEDLM_E_SHAPE;
  const int64_t spans = (T + kPage - 1) / kPage + 1;
  // a launch has fewer than 2^32 threads
  int64_t u = L;
  for (const int64_t f : {B, Hkv, spans}) {
    if (u > (1ll << 26) / f) return WEDLM_E_SHAPE;
    u *= f;
  }
  if (u >= (1ll << 26)) return WEDLM_E_SHAPE;
  *units = u;
  return WEDLM_OK;
}

int launch_append(AppendArgs& a, int D, int64_t units, hipStream_t st) {
  a.spans = (a.T + kPage - 1) / kPage + 1;
  // A window's rows (at most five pages, mostly one that gets a few rows) are
  // one wave's: fewer waves that find nothing to do (16 x 4 rows of 36 layers:
  // 12.0 us; with a wave a page and bytes stored one by one 18.6).  Longer ones
  // take a wave a page.
  a.run = a.T <= WEDLM_MAX_WINDOW ? a.spans : 1;
  a.runs = (a.spans + a.run - 1) / a.run;
  units = units / a.spans * a.runs;
  a.units = static_cast<uint32_t>(units);
  const dim3 grid(static_cast<unsigned>((units + kWavesPerGroup - 1) /
                                        kWavesPerGroup));
  if (D == 128)
    hipLaunchKernelGGL(append8_kernel<128>, grid,
                       dim3(kWavesPerGroup * kWave), 0, st, a);
  else
    hipLaunchKernelGGL(append8_kernel<64>, grid, dim3(kWavesPerGroup * kWave),
                       0, st, a);
  WEDLM_LAUNCH_CHECK();
  return WEDLM_OK;
}

}  // namespace

extern "C" int wedlm_cache8_append(
    const uint16_t* k, const uint16_t* v, const int32_t* start,
    const int32_t* count, int32_t n_layers, int32_t B, int32_t T, int32_t Hkv,
    int32_t D, uint8_t* k8, uint8_t* v8, uint8_t* k_exp, uint8_t* v_exp,
    int64_t num_pages, const int32_t* block_table, int32_t max_pages,
    int32_t* status, void* stream) {
  if (!k || !v || !start || !count || !k8 || !v8 || !k_exp || !v_exp ||
      !block_table)
    return WEDLM_E_ARG;
  int64_t units = 0;
  const int e = append_shape(n_layers, B, T, Hkv, D, num_pages, max_pages,
                             &units);
  if (e != WEDLM_OK) return e;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k8, 16) ||
      !aligned(v8, 16))
    return WEDLM_E_ARG;
  AppendArgs a{};
  a.k = k; a.v = v; a.start = start; a.count = count; a.bt = block_table;
  a.k8 = k8; a.v8 = v8; a.ke = k_exp; a.ve = v_exp; a.status = status;
  a.num_pages = num_pages; a.L = n_layers; a.B = B; a.T = T; a.Hkv = Hkv;
  a.max_pages = max_pages;
  return launch_append(a, D, units, static_cast<hipStream_t>(stream));
}

// The window's update first (it finds the committed run and checks that its
// positions have pages), then the rows of the run, which ends at the new
// win_start.
extern "C" int wedlm_commit_cache8(
    int32_t* win_tok, int32_t* win_start, const int32_t* argmax,
    const float* entropy, double tau, double lambda, const uint16_t* k_win,
    const uint16_t* v_win, uint8_t* k8, uint8_t* v8, uint8_t* k_exp,
    uint8_t* v_exp, int64_t num_pages, const int32_t* block_table,
    int32_t max_pages, int32_t B, int32_t W, int32_t Hkv, int32_t D,
    int32_t n_layers, int32_t* n_commit, int32_t* committed_tok,
    int32_t* committed_slot, uint8_t* selected, int32_t* status, int32_t rule,
    void* stream) {
  if (!k_win || !v_win || !k8 || !v8 || !k_exp || !v_exp) return WEDLM_E_ARG;
  if (W > WEDLM_MAX_WINDOW) return WEDLM_E_SHAPE;
  int64_t units = 0;
  int e = append_shape(n_layers, B, W, Hkv, D, num_pages, max_pages, &units);
  if (e != WEDLM_OK) return e;
  if (!aligned(k_win, 16) || !aligned(v_win, 16) || !aligned(k8, 16) ||
      !aligned(v8, 16))
    return WEDLM_E_ARG;
  e = commit_window(win_tok, win_start, argmax, entropy, tau, lambda,
                    num_pages, block_table, max_pages, B, W, n_commit,
                    committed_tok, committed_slot, selected, status, rule,
                    stream);
  if (e != WEDLM_OK) return e;
  AppendArgs a{};
  a.k = k_win; a.v = v_win; a.start = win_start; a.count = n_commit;
  a.bt = block_table;
  a.k8 = k8; a.v8 = v8; a.ke = k_exp; a.ve = v_exp;
  a.num_pages = num_pages; a.L = n_layers; a.B = B; a.T = W; a.Hkv = Hkv;
  a.max_pages = max_pages; a.behind = 1;
  return launch_append(a, D, units, static_cast<hipStream_t>(stream));
}
