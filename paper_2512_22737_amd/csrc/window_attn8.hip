// The window attention over a paged cache of e4m3 codes with one power-of-two
// scale per page and kv head (wedlm_window_attn_cache8).
//
// Work: a workgroup takes (sequence, kv head, query group, prefix split).
// Query rows of one kv head are packed as in the bf16 kernel (row r = i*G + j
// is window row i, query head kvh*G + j); a wave owns 32 of them.  Up to 32
// rows four waves share them and take every fourth 32-key tile, up to 64 two
// do; more rows go to up to eight waves that all read every tile.  S^T = K Q^T and O^T += V^T P^T
// run on v_mfma_f32_32x32x16_bf16: e4m3 values are exact in bf16, so the codes
// are converted on the way into the products and nothing else is rounded than
// over a bf16 cache.
// Orders.  A lane's 16 bytes of a key row are 16 values of d: the K and Q
// operands take d in that order (products do not care), so a lane reads whole
// 16-byte pieces.  Score rows are the keys in the order that leaves lane
// half hf with the 16 keys of page hf: its K scale is then one factor per
// lane, folded into the softmax's, and its 16 weights meet the 16 bytes of a
// V^T row of that page, whose scale the conversion applies.
// Loads go straight from HBM into LDS.  Waves that share keys: 64 keys (four
// pages) are a step, 16 KB with D = 128, in a ring of four steps, three ahead;
// one barrier a step.  Waves with keys of their own: a ring of two tiles each,
// no barrier.  The split's page ids and exponents are staged in LDS first.
// Softmax: log2 domain, no maximum per tile (the reference maximum is the
// first tile's and is raised when a sum passes 2^64).  P enters its product in
// bf16, which is exact enough beside the bf16 result (error against 64 bits
// 0.0023 of the norm, 0.0017 of it the result's own rounding); the splits' sums
// are merged in fp32.
// Bounds.  Up to 32 rows a kv head: HBM (64 prefixes of 512 to 4096, 32/8 heads
// of 128, W = 1: 59 + 4 us, 4.8 TB/s).  More: the vector work of a tile (64
// conversions, 16 exponentials, about 150 instructions) beside its 16 products
// with two waves a SIMD in order: W = 32 124 + 9 us (0.62 PFLOP/s), 8 x 32768 W
// = 64 302 + 7 us (0.9 PFLOP/s).
#include "common.h"
#include "wedlm_serve.h"

using namespace wedlm;

namespace {

constexpr int kTileKeys = 32;       // keys per tile (two 16-token pages)
// A prefix split but a sequence's last one, which has what is left, holds at
// least this many tiles, and at most 2048 pages (their ids are staged in LDS).
constexpr int kMinSplitTiles = 8;
constexpr int kMaxSplitPages = 2048;
constexpr int kMaxSplitTiles = kMaxSplitPages / 2;
// A launch has this many times the workgroups that its splits should come to:
// a sequence can have that many times its share of them.
// (Those that are not in use come last and end at once.)
constexpr int kSpare = 4;
constexpr int kStepPages = 4;       // pages of a step
constexpr int kSlots = 4;           // steps in the ring, kSlots - 1 ahead
// A column's running sum may reach this before its reference max is raised
// (every term 2^(s - m) is then at most 2^64, far inside fp32).
constexpr float kSumLimit = 18446744073709551616.0f;  // 2^64
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
  float* ws_o;            // [B, Hkv, rows_pad, nsplit, D]: a split's sums of
                          // p v, not normalised (bf16 would round once more)
  float2* ws_ml;          // [B, Hkv, rows_pad, nsplit]
  int32_t* ws_n;          // [B] splits in use (0: a bad length)
  int num_pages, B, W, Hq, Hkv, G, max_pages, max_prefix, nsplit, qgroups,
      rows_pad;
  int want;               // workgroups that the splits should come to
  float scale_log2;       // softmax_scale * log2(e)
};

// Tiles of a prefix (up to 2^31 - 1 positions).
__host__ __device__ __forceinline__ int tiles_of(int c) {
  return c / kTileKeys + (c % kTileKeys != 0 ? 1 : 0);
}

struct Plan {
  int nw, kw;             // waves, of which kw share the rows and split the keys
  int qgroups, rows_pad, nsplit, want;
  size_t ws_bytes;
};

// Byte offsets of a workspace's parts (see Args): the sums, from 0, the
// (m, l) pairs, the splits in use.
struct Layout {
  size_t ml, n, bytes;
  Layout(int B, int Hkv, const Plan& p, int D) {
    const size_t rows = static_cast<size_t>(B) * Hkv * p.rows_pad * p.nsplit;
    ml = rows * D * sizeof(float);
    n = ml + rows * sizeof(float2);
    bytes = n + static_cast<size_t>(B) * sizeof(int32_t);
  }
};

Plan make_plan(int B, int W, int Hq, int Hkv, int D, int max_prefix) {
  Plan p{};
  const int rows = W * (Hq / Hkv);
  p.kw = rows <= 32 ? 4 : rows <= 64 ? 2 : 1;
  p.nw = rows <= 128 ? 4 : 8;
  const int per = 32 * p.nw / p.kw;
  p.qgroups = (rows + per - 1) / per;
  p.rows_pad = p.qgroups * per;
  // two workgroups of four waves are on a CU, or one of eight (64 x 4096, W =
  // 32, one run each: aimed at 256 135 us, 512 134, 1024 140, 2048 177; 8 x
  // 32768, W = 64: 304, 320, 351, 429)
  p.want = p.nw == 4 ? 512 : 256;
  const int tiles = tiles_of(max_prefix);
  const int64_t base = static_cast<int64_t>(B) * Hkv * p.qgroups;
  // room for a long prefix among short ones
  int64_t n = (kSpare * p.want + base - 1) / base;
  const int most = tiles / kMinSplitTiles;
  if (n > most) n = most;
  const int least = (tiles + kMaxSplitTiles - 1) / kMaxSplitTiles;
  if (n < least) n = least;
  if (n < 1) n = 1;
  p.nsplit = static_cast<int>(n);
  if (p.nsplit > 1) p.ws_bytes = Layout(B, Hkv, p, D).bytes;
  return p;
}

__device__ __forceinline__ bool len_ok(const Args& a, int c) {
  return c >= 0 && c <= a.max_prefix &&
         static_cast<int64_t>(c) <= static_cast<int64_t>(a.max_pages) * kPage;
}

// Tiles of a split: such that the splits of all sequences come to `want`
// workgroups, within the limits and the launch's nsplit a sequence.  From the
// sequences' own lengths, so neither a max_prefix_len far above them nor
// uneven ones leave CUs idle.  Every lane takes part and gets it.
__device__ __forceinline__ int split_tiles(const Args& a) {
  if (a.nsplit == 1) return 1 << 30;
  int most = 0;
  int64_t total = 0;
  for (int i = lane_id(); i < a.B; i += kWave) {
    const int c = a.plen[i];
    const int t = len_ok(a, c) ? tiles_of(c) : 0;
    most = max(most, t);
    total += t;
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    most = max(most, __shfl_xor(most, off));
    total += __shfl_xor(static_cast<long long>(total), off);
  }
  const int64_t share =
      (total * a.Hkv * a.qgroups + a.want - 1) / a.want;
  const int64_t per = max(max(share, static_cast<int64_t>(kMinSplitTiles)),
                          static_cast<int64_t>((most + a.nsplit - 1) / a.nsplit));
  return static_cast<int>(min(per, static_cast<int64_t>(kMaxSplitTiles)));
}

// Splits in use by a prefix of c positions (one if it is empty).
__device__ __forceinline__ int splits_of(int c, int per) {
  return max(1, (tiles_of(c) + per - 1) / per);
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

// 16 bytes per lane from a raw buffer straight into LDS (lane l's at lds_addr +
// 16 l).  A vector memory instruction must not read a scalar register within
// five wait states of a vector instruction that wrote it (as readfirstlane
// does), nor M0 within one of its write; the compiler does not see the load
// in this text, so the states are part of it.
__device__ __forceinline__ void load_lds16(i32x4_t rsrc, int voff,
                                           uint32_t lds_addr) {
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen nt lds"
               :
               : "v"(voff), "s"(rsrc), "{m0}"(lds_addr));
}

// 2^(e - 127) of a scale's exponent (1 .. 254).
__device__ __forceinline__ float scale_of(int e) {
  return __uint_as_float(static_cast<uint32_t>(e) << 23);
}

// LDS of one workgroup: the ring (K and V^T of each step), the pages' ids and
// exponents.
//   K    [4 pages][16 rows][D]: 16-byte chunk c of row r of page g sits in
//        slot c ^ swz(r, g & 1), so that the 16 lanes of a read pass (rows 4a
//        .. 4a+7 of two pages) meet 64 different banks
//   V^T  [4 pages][D rows][16]
template <int D>
struct Lds {
  static constexpr int kPageBytes = kPage * D;
  static constexpr int kHalf = kStepPages * kPageBytes;   // K or V^T of a step
  static constexpr int kStep = 2 * kHalf;
  __device__ static __forceinline__ int swz(int r, int g) {
    return D == 128 ? ((r >> 1) & 3) | (g << 2) : ((r >> 2) & 1) | (g << 1);
  }
};

template <int D, int NW, int KW>
__global__ __launch_bounds__(NW * kWave)
__attribute__((amdgpu_waves_per_eu(2)))
void window_attn8_kernel(Args a) {
  using L = Lds<D>;
  constexpr int NJ = D / 32;          // 16-byte pieces of a key row per half
  constexpr int NK = D / 16;          // k-steps of the score MFMA
  constexpr int NM = D / 32;          // 32-row blocks of O^T
  constexpr int NQ = NW / KW;         // query blocks of a workgroup
  constexpr int NT = NW * kWave;
  constexpr bool kOwn = KW == NW;     // waves with keys (and a ring) of their own
  constexpr int kTile = L::kStep / 2;
  // loads of a wave per step, or per tile of its own
  constexpr int kLoads = kOwn ? kTile / 1024 : L::kStep / 1024 / NW;
  static_assert(L::kStep % (1024 * NW) == 0, "whole loads");
  static_assert(!kOwn || NW * 2 * kTile == kSlots * L::kStep, "the same LDS");
  __shared__ __attribute__((aligned(1024))) char ring[kSlots * L::kStep];
  __shared__ int32_t pg[kMaxSplitPages + kStepPages];
  __shared__ uint16_t ex[kMaxSplitPages + kStepPages];

  // the first splits of all sequences, then the second ones, ...: those that
  // are not in use come last
  int wg = blockIdx.x;
  const int qg = wg % a.qgroups;
  wg /= a.qgroups;
  const int kvh = __builtin_amdgcn_readfirstlane(wg % a.Hkv);
  wg /= a.Hkv;
  const int b = wg % a.B;
  const int split = wg / a.B;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = lane_id();
  const int col = lane & 31, hf = lane >> 5;
  const int kw = KW == 1 ? 0 : wave / NQ;
  const int rows = a.W * a.G;
  const int rb = (qg * NQ + wave % NQ) * 32;

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

  const int c = a.plen[b];
  const bool tells = threadIdx.x == 0 && split == 0 && qg == 0 && kvh == 0;
  if (!len_ok(a, c)) {
    if (tells && a.status) atomicOr(a.status + b, WEDLM_SEQ_BAD_LEN);
    if (tells && a.nsplit > 1) a.ws_n[b] = 0;
    return;
  }
  const int per = split_tiles(a);
  const int nsplit = splits_of(c, per);
  if (tells && a.nsplit > 1) a.ws_n[b] = nsplit;
  if (split >= nsplit) return;
  const int k0 = nsplit == 1 ? 0 : split * per * kTileKeys;
  const int k1 = split == nsplit - 1 ? c : k0 + per * kTileKeys;
  const bool last = split == nsplit - 1;
  const int pages = (k1 - k0 + kPage - 1) / kPage;
  const int steps = (pages + kStepPages - 1) / kStepPages;

  // ---- the split's pages; an id outside the cache becomes page 0 (in bounds)
  // and is told.  The last step is filled up with the last page.
  const int32_t* btb = a.bt + static_cast<int64_t>(b) * a.max_pages + k0 / kPage;
  for (int i = threadIdx.x; i < steps * kStepPages; i += NT) {
    int id = btb[min(i, pages - 1)];
    if (id < 0 || id >= a.num_pages) {
      if (a.status) atomicOr(a.status + b, WEDLM_SEQ_BAD_PAGE);
      id = 0;
    }
    pg[i] = id;
  }
  __syncthreads();
  // the queries have arrived by now: taken here, once, so that no later use
  // waits for loads that are under way then
#pragma unroll
  for (int kk = 0; kk < NK; ++kk) asm volatile("" : "+v"(qf[kk]));

  // ---- loads.  Kilobyte kb of a step is one of its K, then of its V^T; lane
  // l's 16 bytes land at byte 16 l of it, so K's swizzle is in the lane's
  // address.  A tile of a wave's own is laid out alike, with half the pages.
  constexpr int kPerPage = L::kPageBytes / 1024;          // kilobytes
  constexpr int kHalfKb = (kOwn ? kTile : L::kStep) / 2048;
  const uint32_t lds0 =
      static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void_t*)ring));
  // page of a step that kilobyte kb is of
  auto page_of = [](int kb) { return kb % kHalfKb / kPerPage; };
  auto load_kb = [&](int id, int kb, uint32_t dst) {
    const bool isv = kb >= kHalfKb;
    const int at = kb % kPerPage * 64 + lane;             // chunk of the page
    int off = at * 16;
    if (!isv) {
      const int row = at / (D / 16), s = at % (D / 16);
      off = row * D + ((s ^ L::swz(row, page_of(kb) & 1)) << 4);
    }
    const uint8_t* base = (isv ? a.v8 : a.k8) +
                          (static_cast<int64_t>(id) * a.Hkv + kvh) *
                              L::kPageBytes;
    load_lds16(buffer_rsrc(base, L::kPageBytes), off,
               __builtin_amdgcn_readfirstlane(dst + kb * 1024));
  };
  // the step of the split that is taken as the t-th one
  auto step_of = [&](int t) {
    return KW > 1 ? t : t == 0 ? steps - 1 : t - 1;
  };
  const int tiles = (pages + 1) / 2;
  // Loads of this wave's part of step t, or of its i-th own tile (indices past
  // the end load the last pages again: as many loads each time).  Their page
  // ids are read from LDS one call ahead.
  int ids[kLoads];
  auto read_ids = [&](int t) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      if constexpr (kOwn)
        ids[u] = pg[min(t * KW + kw, tiles - 1) * 2 + page_of(u)];
      else
        ids[u] = pg[step_of(min(t, steps - 1)) * kStepPages +
                    page_of(wave * kLoads + u)];
    }
  };
  auto load = [&](int t) {
    const uint32_t dst =
        lds0 + (kOwn ? (wave * 2 + (t & 1)) * kTile
                     : (t & (kSlots - 1)) * L::kStep);
    int now[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
      now[u] = __builtin_amdgcn_readfirstlane(ids[u]);
    read_ids(t + 1);
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
      load_kb(now[u], kOwn ? u : wave * kLoads + u, dst);
  };
  if (steps > 0) {
    read_ids(0);
#pragma unroll
    for (int t = 0; t < (kOwn ? 1 : kSlots - 1); ++t) load(t);
    // the exponents, under the first loads
    for (int i = threadIdx.x; i < steps * kStepPages; i += NT) {
      const int64_t at = static_cast<int64_t>(pg[i]) * a.Hkv + kvh;
      ex[i] = static_cast<uint16_t>(a.ke[at] | a.ve[at] << 8);
    }
  }

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
  // largest of a column's 32 scores
  auto col_max = [&](const floatx16_t& x) {
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, x[e]);
    float x0, x1;
    xor32_pair(mx, x0, x1);
    return fmaxf(x0, x1);
  };
  // weights 2^(x f - m2) in bf16 and l_run with their sum added
  auto weigh = [&](const floatx16_t& x, float f, bf16x8_t (&pf)[2]) {
    const float mc = m2 == kNegInf ? 0.f : m2;
    float p[16];
#pragma unroll
    for (int e = 0; e < 16; ++e)
      p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], f, -mc));
#pragma unroll
    for (int e = 0; e < 16; ++e) pf[e >> 3][e & 7] = static_cast<__bf16>(p[e]);
    float s[4];
#pragma unroll
    for (int g = 0; g < 4; ++g)
      s[g] = (p[4 * g] + p[4 * g + 1]) + (p[4 * g + 2] + p[4 * g + 3]);
    return l_run + ((s[0] + s[1]) + (s[2] + s[3]));
  };
  auto raise = [&](float mx) {
    if (ballot(mx > m2)) {
      const float m_new = fmaxf(m2, mx);
      rescale(m2 == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m2 - m_new));
      m2 = m_new;
    }
  };
  auto product = [&](const bf16x8_t (&vf)[2][NM], const bf16x8_t (&pf)[2]) {
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
      for (int m = 0; m < NM; ++m)
        o[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[h2][m], pf[h2], o[m],
                                                       0, 0, 0);
  };

  // ---- the window, with the last split (its tiles dealt to the key waves):
  // under the first loads
  if (last && rb < rows) {
    const int64_t wrow = static_cast<int64_t>(b) * a.W;
    for (int base = kw * kTileKeys; base < a.W; base += KW * kTileKeys) {
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
      const int at = base + 16 * hf;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = at + e <= qi ? s[e] : kNegInf;
      bf16x8_t vf[2][NM], pf[2];
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
      raise(col_max(s) * a.scale_log2);
      l_run = weigh(s, a.scale_log2, pf);
      product(vf, pf);
    }
  }

  // ---- the prefix
  // offsets in a tile: page (col >> 2) & 1 of its two, row key & 15
  const int kpg = (col >> 2) & 1, krow = key & 15;
  const int k_lane = kpg * L::kPageBytes + krow * D;
  const int k_swz = L::swz(krow, kpg);
  const int v_lane = hf * L::kPageBytes + col * kPage;
  auto read_k = [&](const char* kt, u32x4_t (&kr)[NJ]) {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      kr[j] = *reinterpret_cast<const u32x4_t*>(
          kt + k_lane + (((2 * j + hf) ^ k_swz) << 4));
  };
  auto read_v = [&](const char* vt, u32x4_t (&vr)[NM]) {
#pragma unroll
    for (int m = 0; m < NM; ++m)
      vr[m] = *reinterpret_cast<const u32x4_t*>(vt + v_lane + m * 32 * kPage);
  };
  auto scores = [&](const u32x4_t (&kr)[NJ]) {
    floatx16_t s = {};
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            widen(kr[j][2 * i], kr[j][2 * i + 1], 1.f), qf[2 * j + i], s, 0, 0,
            0);
    return s;
  };
  auto add_values = [&](const u32x4_t (&vr)[NM], float vs,
                        const bf16x8_t (&pf)[2]) {
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
      for (int m = 0; m < NM; ++m)
        o[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            widen(vr[m][2 * h2], vr[m][2 * h2 + 1], vs), pf[h2], o[m], 0, 0, 0);
  };
  // A whole tile whose K is in registers already (kr, exponents e), with the
  // next one's K read meanwhile.  One block of code, but for the rare raise:
  // under each score MFMA the conversions of the next one's keys and of an
  // eighth of the values.
  auto whole_tile = [&](const char* vt, u32x4_t (&kr)[NJ], int& e,
                        const char* next_kt, int next_n32) {
    u32x4_t vr[NM], kn[NJ];
    read_v(vt, vr);
    read_k(next_kt, kn);
    const int en = ex[next_n32 * 2 + hf];
    const float f = a.scale_log2 * scale_of(e & 0xff), vs = scale_of(e >> 8);
    const floatx16_t s = scores(kr);
    bf16x8_t vf[2][NM], pf[2];
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
      for (int m = 0; m < NM; ++m)
        vf[h2][m] = widen(vr[m][2 * h2], vr[m][2 * h2 + 1], vs);
    __builtin_amdgcn_sched_group_barrier(0x100, NM + NJ + 1, 0);  // LDS reads
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x002, 8, 0);          // VALU
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);          // MFMA
    }
    float sum = weigh(s, f, pf);
    if (ballot(!(sum <= kSumLimit))) {
      raise(col_max(s * f));
      sum = weigh(s, f, pf);
    }
    l_run = sum;
    product(vf, pf);
#pragma unroll
    for (int j = 0; j < NJ; ++j) kr[j] = kn[j];
    e = en;
  };
  // one tile: its K and V^T pages in LDS, its number in the split
  auto tile_of = [&](const char* kt, const char* vt, int n32) {
      const int base = k0 + n32 * kTileKeys;
      u32x4_t kr[NJ], vr[NM];
      read_k(kt, kr);
      read_v(vt, vr);
      const int e2 = ex[n32 * 2 + hf];
      float ks = scale_of(e2 & 0xff), vs = scale_of(e2 >> 8);
      floatx16_t s = scores(kr);
      bf16x8_t pf[2];
      if (k1 - base >= kTileKeys) {     // (base + kTileKeys may pass 2^31 - 1)
        const float f = a.scale_log2 * ks;
        if (ballot(m2 == kNegInf)) raise(col_max(s * f));
        float sum = weigh(s, f, pf);
        if (ballot(!(sum <= kSumLimit))) {
          raise(col_max(s * f));
          sum = weigh(s, f, pf);
        }
        l_run = sum;
      } else {
        // the prefix ends inside: keys of this lane's page that are in it.
        // Codes behind count as zero, and a page without any has any scale
        const int n = min(max(k1 - base - 16 * hf, 0), kPage);
        ks = n > 0 ? ks : 1.f;
        vs = n > 0 ? vs : 1.f;
        const float f = a.scale_log2 * ks;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = e < n ? s[e] * f : kNegInf;
        uint32_t mask[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int k = min(max(n - 4 * w, 0), 4);
          mask[w] = k == 4 ? ~0u : (1u << (8 * k)) - 1;
        }
#pragma unroll
        for (int m = 0; m < NM; ++m)
#pragma unroll
          for (int w = 0; w < 4; ++w) vr[m][w] &= mask[w];
        raise(col_max(s));
        l_run = weigh(s, 1.f, pf);
      }
      add_values(vr, vs, pf);
  };
  if constexpr (kOwn) {
    __syncthreads();      // the exponents are there
    for (int i = 0; i * KW + kw < tiles; ++i) {
      // every read of the other slot has returned; its next tile is loaded, and
      // the loads before that have arrived
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      load(i + 1);
      wait_vmcnt<kLoads>();
      asm volatile("" ::: "memory");
      const char* at = ring + (wave * 2 + (i & 1)) * kTile;
      tile_of(at, at + kTile / 2, i * KW + kw);
    }
  } else {
    // this wave's loads of step t (and the next, where K is read ahead) are
    // done, and with the barrier everyone's; nobody reads the slot of step
    // t - 1 any more
    auto begin = [&](int t) {
      wait_vmcnt<kLoads * (kSlots - (KW == 1 ? 3 : 2))>();
      __syncthreads();
      load(t + kSlots - 1);
      return ring + (t & (kSlots - 1)) * L::kStep;
    };
    auto by_tile = [&](const char* at, int n32) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        if (KW == 2 && g != kw) continue;
        if (n32 + g < tiles)
          tile_of(at + g * 2 * L::kPageBytes,
                  at + L::kHalf + g * 2 * L::kPageBytes, n32 + g);
      }
    };
    if constexpr (KW == 1) {
      // the last step first, tile by tile: it may end inside, and gives the
      // reference maxima; all others are whole
      if (steps > 0) by_tile(begin(0), 2 * (steps - 1));
      u32x4_t kr[NJ];
      int e = 0;
      if (steps > 1) {
        read_k(ring + L::kStep, kr);
        e = ex[hf];
      }
      for (int t = 1; t < steps; ++t) {
        const char* at = begin(t);
        const char* next = ring + ((t + 1) & (kSlots - 1)) * L::kStep;
        whole_tile(at + L::kHalf, kr, e, at + 2 * L::kPageBytes, 2 * t - 1);
        whole_tile(at + L::kHalf + 2 * L::kPageBytes, kr, e, next, 2 * t);
      }
    } else {
      for (int t = 0; t < steps; ++t) by_tile(begin(t), 2 * t);
    }
  }
  wait_vmcnt<0>();        // surplus loads have landed before LDS is used again

  // ---- the key waves' parts joined, in the first ones
  if constexpr (KW > 1) {
    constexpr int kPart = (NM * 16 + 2) * kWave;
    static_assert((KW - 1) * NQ * kPart * 4 <= kSlots * L::kStep, "parts in LDS");
    __syncthreads();
    float* part = reinterpret_cast<float*>(ring) + lane;
    if (kw > 0) {
      part += ((kw - 1) * NQ + wave % NQ) * kPart;
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) part[(m * 16 + e) * kWave] = o[m][e];
      part[NM * 16 * kWave] = m2;
      part[(NM * 16 + 1) * kWave] = l_run;
    }
    __syncthreads();
    if (kw > 0) return;
    part += wave % NQ * kPart;
#pragma unroll 1
    for (int w = 1; w < KW; ++w, part += NQ * kPart) {
      const float mo = part[NM * 16 * kWave];
      const float m_new = fmaxf(m2, mo);
      const float base = m_new == kNegInf ? 0.f : m_new;
      rescale(__builtin_amdgcn_exp2f(m2 - base));
      const float f = __builtin_amdgcn_exp2f(mo - base);
      l_run += f * part[(NM * 16 + 1) * kWave];
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[m][e] += f * part[(m * 16 + e) * kWave];
      m2 = m_new;
    }
  }

  float l0, l1;
  xor32_pair(l_run, l0, l1);
  const float l_tot = l0 + l1;
  if (!rvalid) return;
  const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
  const int64_t part =
      ((static_cast<int64_t>(b) * a.Hkv + kvh) * a.rows_pad + r) * a.nsplit +
      split;
  const int64_t orow = (static_cast<int64_t>(b) * a.W + qi) * a.Hq + qh;
  // (both branches store 4 consecutive d of an accumulator's quarter)
  if (nsplit == 1) {
    uint16_t* op = a.out + orow * D;
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
  } else {
    float* op = a.ws_o + part * D;
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const floatx4_t v = {o[m][4 * g], o[m][4 * g + 1], o[m][4 * g + 2],
                             o[m][4 * g + 3]};
        *reinterpret_cast<floatx4_t*>(op + m * 32 + g * 8 + hf * 4) = v;
      }
  }
  if (hf == 0) {
    if (nsplit > 1)
      a.ws_ml[part] = make_float2(m2, l_tot);
    else if (a.lse)
      a.lse[orow] = (m2 + __log2f(l_tot)) * kLn2;
  }
}

// Merge of the outputs of sequences with several splits: O = sum_s 2^(m_s - M)
// O_s / sum_s 2^(m_s - M) l_s, in fp32, the splits in order.  D/8 threads a
// row, 32 bytes of a split each.
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
  const int n = a.ws_n[b];
  if (n <= 1) return;                 // written already, or not at all
  const int64_t part = (bk * a.rows_pad + r) * a.nsplit;
  const float2* ml = a.ws_ml + part;
  const float* op = a.ws_o + part * D + d;
  // four splits' loads under way at a time
  constexpr int kAtOnce = 4;
  float M = kNegInf, L = 0.f, acc[8] = {};
  for (int s0 = 0; s0 < n; s0 += kAtOnce) {
    float2 x[kAtOnce];
    floatx4_t v[kAtOnce][2];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int s = min(s0 + i, n - 1);
      x[i] = ml[s];
      const floatx4_t* at =
          reinterpret_cast<const floatx4_t*>(op + static_cast<int64_t>(s) * D);
      v[i][0] = at[0];
      v[i][1] = at[1];
    }
    float top = M;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) top = fmaxf(top, x[i].x);
    const float base = top == kNegInf ? 0.f : top;
    const float old = __builtin_amdgcn_exp2f(M - base);
    L *= old;
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[k] *= old;
    M = top;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (s0 + i >= n) break;         // (a weight of 0 would not do: sums that
                                      // are infinite stay so)
      const float w = __builtin_amdgcn_exp2f(x[i].x - base);
      L += w * x[i].y;
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[k] += w * v[i][k / 4][k % 4];
    }
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

template <int D>
int launch(const Args& a, const Plan& p, int64_t grid, hipStream_t st) {
  const dim3 g(static_cast<unsigned>(grid)), n(p.nw * kWave);
  if (p.kw == 4)
    hipLaunchKernelGGL((window_attn8_kernel<D, 4, 4>), g, n, 0, st, a);
  else if (p.kw == 2)
    hipLaunchKernelGGL((window_attn8_kernel<D, 4, 2>), g, n, 0, st, a);
  else if (p.nw == 4)
    hipLaunchKernelGGL((window_attn8_kernel<D, 4, 1>), g, n, 0, st, a);
  else
    hipLaunchKernelGGL((window_attn8_kernel<D, 8, 1>), g, n, 0, st, a);
  WEDLM_LAUNCH_CHECK();
  return WEDLM_OK;
}

bool shape_ok(int B, int W, int Hq, int Hkv, int D, int max_prefix) {
  if (!(B >= 1 && W >= 1 && W <= WEDLM_MAX_WINDOW && Hkv >= 1 && Hq >= Hkv &&
        Hq % Hkv == 0 && (D == 64 || D == 128) && max_prefix >= 0))
    return false;
  // rows, padded to whole workgroups, and their workgroups fit 31 bits
  const int64_t rows = static_cast<int64_t>(W) * (Hq / Hkv) + 255;
  if (rows >= (1ll << 31) / Hkv || rows * Hkv >= (1ll << 31) / B) return false;
  // and so do the launch's threads 32
  const Plan p = make_plan(B, W, Hq, Hkv, D, max_prefix);
  return static_cast<int64_t>(p.nsplit) * B * Hkv * p.qgroups <
         (1ll << 32) / (p.nw * kWave);
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
  a.want = p.want;
  a.scale_log2 = softmax_scale * 1.4426950408889634f;
  if (p.nsplit > 1) {
    const Layout at(B, Hkv, p, D);
    char* base = static_cast<char*>(workspace);
    a.ws_o = reinterpret_cast<float*>(base);
    a.ws_ml = reinterpret_cast<float2*>(base + at.ml);
    a.ws_n = reinterpret_cast<int32_t*>(base + at.n);
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t grid = static_cast<int64_t>(p.nsplit) * B * Hkv * p.qgroups;
  const int e = D == 128 ? launch<128>(a, p, grid, st)
                         : launch<64>(a, p, grid, st);
  if (e != WEDLM_OK) return e;
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
