// Backward pass of the dual-stream training attention (Sec. 4.2): from the
// output's gradient to those of q, k and v, with the probabilities computed
// again from q, k and the forward's normaliser.
//
// For a row i and the keys j it sees (scale s, o and lse of the forward):
//   P_ij = exp(s q_i.k_j - lse_i)        dP_ij = do_i . v_j
//   D_i  = do_i . o_i                    dS_ij = P_ij (dP_ij - D_i)
//   dq_i = s sum_j dS_ij k_j             dk_j  = s sum_i dS_ij q_i
//                                        dv_j  = sum_i P_ij do_i
// where the sums over i run over the G = Hq/Hkv query heads of the kv head
// too.  Memory row p sees memory keys 0..p; prediction row p (block
// start f = p / block * block) sees memory keys 0..f-1 and prediction keys
// f..p.  In both directions the visible ones are an interval.
//
// Two kernels, each accumulating in registers what it owns, so that nothing
// is added atomically and the result does not depend on the run:
//   dq:    a wave owns 32 rows of one head and walks the keys.  It also
//          writes D_i and lse_i, laid out for the second kernel.
//   dk/dv: a wave owns 64 keys of one kv head and walks the rows of all its
//          heads.  (64, not 32: each operand read from LDS then feeds two
//          MFMAs; with 32 the LDS would be as busy as the MFMAs.)
// S and dP are formed in both: seven products instead of the five that a
// single pass needs, which would have to add dq (or dk and dv) in memory, once
// for every key tile, or write dS out, 4.3 GB for 4 x 4096 tokens.
// MFMA: v_mfma_f32_32x32x16_bf16.  The score tile has the streamed rows
// (keys in dq, query rows in dk/dv) as its M dimension and the owned ones as
// N, so a lane holds 16 scores of one owned row, eight at a time contiguous
// (row_of_m), which is the operand layout of the second product: P and dS
// go from accumulators to operands in registers.  The second product's other
// operand is read from the same LDS tile by columns (ds_read_b64_tr_b16).
//
// Roundings: P and dS to bf16 for the second products, as the forward rounds
// P; D from the forward's bf16 output, but exact where rows see few keys (see
// kExactRows); everything else, all sums among it, fp32.  Rounding dS adds as
// much as rounding the result does (0.17% of a gradient's norm): 0.23-0.24%
// together.  In wider operands the second products would run at a fraction of
// the rate.
//
// Bound by the MFMAs, and these by the card's power: 4 x 4096 tokens (32/8
// heads of 128) 3.30 to 3.45 ms from card to card, 797 to 834 TFLOP/s of the
// five products and 1.16 to 1.22 PFLOP/s of what runs, masked parts included;
// MFMAs on random values that do nothing else hold 1.30 PFLOP/s, a large
// library product 1.22.  Leaving out barriers, waits or exponentials does not
// change it.  Steps there (on one card): plain staging, with
// spills, 31.2 ms; tiles straight to LDS, accumulators held in AGPRs, 5.78;
// one MFMA a step with vector work under it 4.35; equal work per CU 3.62;
// prediction keys by single waves 3.41.  Heads of 64 are bound by the vector
// work of twice as many scores per product: 2.03 ms, of what runs dq at 0.99
// PFLOP/s, dk and dv at 0.87.  Shorter sequences are bound by latency: 1 x
// 2048 (16/8 heads) 160 us with other inputs from call to call, 155 with the
// same ones (as below), 1 x 256 (4/2 heads of 64) 27.9 us.
#include <algorithm>
#include <initializer_list>

#include "common.h"
#include "wedlm_train.h"

using namespace wedlm;

namespace {

constexpr int kRows = 32;             // streamed rows of an LDS tile
constexpr int kOwn = 64;              // keys that a wave owns
constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kKeysPerWg = kWaves * kOwn;
constexpr int kSlots = 6;             // dk, dv: ring of tile pairs
constexpr float kLog2e = 1.4426950408889634f;

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

struct BwdArgs {
  const uint16_t* q;      // [n_seq, 2L, Hq, D]
  const uint16_t* k;      // [n_seq, 2L, Hkv, D]
  const uint16_t* v;
  const uint16_t* out;    // [n_seq, 2L, Hq, D]
  const float* lse;       // [n_seq, 2L, Hq]
  const uint16_t* dout;
  uint16_t* dq;
  uint16_t* dk;
  uint16_t* dv;
  float* ld;              // [n_seq, Hq, 2, T, 2, 32]: -lse (log2 units), -D
  float* part;            // [2 W] pieces of cut tiles: see Piece
  int n_seq, L, block, Hq, Hkv, G, T;
  int4* cuts;             // [W + 1]: see Cut
  int W;                  // workgroups of dkv_kernel
  int group_cost;         // work of one (sequence, kv head) of it
  float scale, scale_log2;
};

// LDS tile of 32 rows of D bf16, as it is loaded: one 1 KB load instruction
// fills a group of 512 / D whole rows, groups are 16 bytes apart.  Chunk c (16
// bytes) of row i of its group sits in slot c ^ swz(i).  Rows read together
// (16 rows of one chunk; four rows of 64 bytes by columns) then hit different
// banks with D = 128 (counted: no conflict; with D = 64 conflicts take 40% of
// dq's LDS cycles and 22% of dk's and dv's), and the reads of a lane differ by
// constants but for the exclusive or with its row: few address registers.
template <int D>
struct RowTile {
  static constexpr int per_group = 512 / D;         // rows: 4 or 8
  static constexpr int groups = kRows / per_group;
  static constexpr int group_bytes = 1024 + 16;
  static constexpr int bytes = groups * group_bytes;
  static constexpr int chunks = D / 8;
  __device__ static __forceinline__ int swz(int i) {
    return D == 128 ? i << 2 : ((i & 2) << 1) | ((i & 4) >> 1);
  }
  __device__ static __forceinline__ int off(int r, int c) {
    const int i = r % per_group;
    return r / per_group * group_bytes + i * 2 * D + ((c ^ swz(i)) << 4);
  }
};

// Row of the streamed tile in MFMA row m: bits 2 and 3 swapped, so that
// output element e of a lane (hf = lane / 32) is row 16 (e / 8) + 8 hf + e % 8.
__device__ __forceinline__ int row_of_m(int m) {
  return (m & ~12) | ((m & 4) << 1) | ((m & 8) >> 1);
}

__device__ __forceinline__ bf16x8_t load8(const uint16_t* p) {
  return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u16x8_t*>(p));
}

// A lane's addresses into a tile.
template <int D>
struct Reader {
  using T = RowTile<D>;
  int row[4], col[4];
  __device__ __forceinline__ Reader() {
    const int l = lane_id(), i = l & 15, hf = l >> 5;
    // rows: lane's row, chunks 2 kk + hf; kk / 2 (D = 64: kk) meets the swizzle
#pragma unroll
    for (int x = 0; x < 4; ++x)
      row[x] = T::off(row_of_m(l & 31), (D == 128 ? 4 : 2) * x + hf);
    // columns: four rows on four lanes each, 16 columns per 16 lanes; the
    // block m of 32 columns (D = 64: and the half of eight rows) meets it
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int m = D == 128 ? x : x >> 1, j = D == 128 ? 0 : x & 1;
      col[x] = T::off(8 * hf + 4 * j + (i >> 2),
                      4 * m + 2 * ((l >> 4) & 1) + ((i & 3) >> 1)) +
               (i & 1) * 8;
    }
  }
  // lane's row, values 16 kk + 8 hf .. + 7
  __device__ __forceinline__ bf16x8_t rows(const char* tile, int kk) const {
    return load8(reinterpret_cast<const uint16_t*>(
        tile + (D == 128 ? row[kk >> 1] + (kk & 1) * 32 : row[kk])));
  }
  // lane's column 32 m + lane % 32, rows 16 h + 8 hf .. + 7
  __device__ __forceinline__ bf16x8_t cols(const char* tile, int h,
                                           int m) const {
    s16x4_t x[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
      x[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_s16x4_t*)(tile + h * (16 / T::per_group) * T::group_bytes +
                         (D == 128 ? col[m] + j * T::group_bytes
                                   : col[2 * m + j])));
    return __builtin_bit_cast(
        bf16x8_t, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// Loads of a pair of tiles (32 rows of two arrays of the same row stride)
// straight into LDS: of four waves two take the first array, two the second.
// kCount load instructions per wave; rows past the last one re-read it.
// kOneRow: one register for the rows of all u, whose sums are then made at
// every load.
template <int D, bool kOneRow>
struct PairLoader {
  using T = RowTile<D>;
  static constexpr int kCount = 2 * T::groups / kWaves;
  const uint16_t* src;
  int stride;                        // bytes
  int row, chunk;                    // lane's first row and its chunk, bytes
  uint32_t lds;                      // where the wave's share of a pair goes
  __device__ __forceinline__ PairLoader(const uint16_t* a, const uint16_t* b,
                                        int stride_elements, int wave,
                                        uint32_t lds0)
      : src(wave < kWaves / 2 ? a : b), stride(stride_elements * 2),
        lds(lds0 + wave * kCount * T::group_bytes) {
    const int i = lane_id() / T::chunks;
    row = (wave * kCount % T::groups * T::per_group + i) * stride;
    chunk = ((lane_id() % T::chunks) ^ T::swz(i)) * 16;
  }
  // instruction u: o elements from the arrays' starts to the tile's first row,
  // left rows from there to the last one; dst: bytes from lds0 to the pair
  __device__ __forceinline__ void load(int u, int64_t o, int left,
                                       uint32_t dst) const {
    int r = row;
    if (kOneRow) asm volatile("" : "+v"(r));
    load_to_lds16<false>(buffer_rsrc(src + o, 31 * stride + 2 * D),
                         min(r + u * T::per_group * stride,
                             min(left, kRows - 1) * stride) +
                             chunk,
                         lds + dst + u * T::group_bytes);
  }
};

// One dword per lane to LDS: lane l's at lds_addr + 4 l.
__device__ __forceinline__ void load_to_lds4(i32x4_t rsrc, int voff,
                                             uint32_t lds_addr) {
  asm volatile("buffer_load_dword %0, %1, 0 offen lds"
               :
               : "v"(voff), "s"(rsrc), "{m0}"(lds_addr));
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((lds_void_t*)p));
}

__device__ __forceinline__ floatx16_t mfma(bf16x8_t a, bf16x8_t b,
                                           floatx16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// acc += a b with the accumulator in the accumulation registers throughout:
// with the score tiles in plain registers neither file overflows (left to
// itself the compiler moves hundreds of accumulators per tile).  It does not
// know that this is an MFMA: operands that the VALU wrote go through
// settle() first, and drain() comes before anything else reads an
// accumulator.
__device__ __forceinline__ void mfma_acc(floatx16_t& acc, bf16x8_t a,
                                         bf16x8_t b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0"
               : "+a"(acc)
               : "v"(a), "v"(b));
}

// Two wait states between the VALU's writes of an operand and an MFMA's read;
// the operand is complete here.
__device__ __forceinline__ void settle(bf16x8_t& x) {
  asm volatile("s_nop 1" : "+v"(x));
}

// The value is computed here, not sunk past the next branch.
__device__ __forceinline__ void here(float& x) { asm volatile("" : "+v"(x)); }

// All waves are here.  Without the wait for this wave's own LDS reads that
// __syncthreads() has: those under way are of the next tile, which stays.
__device__ __forceinline__ void meet() {
  asm volatile("s_barrier" ::: "memory");
}

// x where bit e of see is set, -inf elsewhere.
__device__ __forceinline__ float seen(uint32_t see, int e, float x) {
  const uint32_t m = __builtin_amdgcn_sbfe(see, e, 1);       // 0 or ~0
  return __uint_as_float((__float_as_uint(x) & m) |
                         (__float_as_uint(kNegInf) & ~m));
}

// Bits e of the elements of a lane (tile rows 16 (e / 8) + 8 hf + e % 8) whose
// rows lie in from .. to-1, both relative to row 8 hf of the tile.
__device__ __forceinline__ uint32_t rows_between(int from, int to) {
  // rows 0 .. 7 and 16 .. 23 of 32 bits
  const uint32_t below_to = to <= 0 ? 0u : to >= 32 ? ~0u : (1u << to) - 1u;
  const uint32_t below_from =
      from <= 0 ? 0u : from >= 32 ? ~0u : (1u << from) - 1u;
  const uint32_t m = below_to & ~below_from;
  return (m & 0xffu) | (m >> 8 & 0xff00u);
}

// Lane index, computed where it stands (no register from outside the loop).
__device__ __forceinline__ int lane_here() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0"
               : "=v"(l));
  return l;
}

// Ends a step: what is written before it is issued before it.  The tiles are
// written as steps of one MFMA (32 cycles) and the vector work and LDS reads
// that run under it (measured, n fused multiply-adds beside an MFMA take
// 16 + 4 n cycles: four fit, or an exponential and two).
__device__ __forceinline__ void step() { __builtin_amdgcn_sched_barrier(0); }

// Sixteen columns 32 m + 16 j .. of the gradient of a lane's row, times scale,
// from elements 8 j .. 8 j + 7 of its accumulator: half-waves hold four of
// every eight columns each; after the exchange a lane has eight together.
__device__ __forceinline__ void store_row(uint16_t* row, int m, int j, int hf,
                                          const floatx16_t& acc, float scale) {
  bf16x8_t v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = static_cast<__bf16>(acc[8 * j + e] * scale);
  const u32x4_t x = __builtin_bit_cast(u32x4_t, v);
  u32x4_t y;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const auto z =
        __builtin_amdgcn_permlane32_swap(x[e], x[2 + e], false, false);
    y[e] = z[0];
    y[2 + e] = z[1];
  }
  *reinterpret_cast<u32x4_t*>(row + 32 * m + 16 * j + 8 * hf) = y;
}

// The accumulators of the last mfma_acc() are written (18 wait states).
template <int N>
__device__ __forceinline__ void drain(floatx16_t (&acc)[N]) {
  asm volatile("s_nop 15\n\ts_nop 3" : "+a"(acc[0]));
#pragma unroll
  for (int m = 1; m < N; ++m) asm volatile("" : "+a"(acc[m]));
}

// ---------------------------------------------------------------------------
// The work of dk and dv: key tiles of 256 keys, each with a walk of row tiles
// (its items).  The tiles of a (sequence, kv head) are listed in fours: memory
// tiles i and n-1-i, whose walks add up to the same for every i, and the
// prediction tiles i and n-1-i.  The list of all of them is cut into W
// stretches of equal work, one per workgroup (one per CU); a cut near a
// tile's end moves there, one inside a tile leaves two workgroups partial sums
// of it, which a last kernel adds up in order.
// ---------------------------------------------------------------------------
// Work in items of memory keys, from the clock at each part of 1 x 2048 tokens
// (16/8 heads of 128): an item 1.7 us, 2.1 where scores are masked (1 /
// kMaskMore more), a tile's start and end 5 + 4; prediction keys, each wave its
// own tiles, 2.7 an item (1 / kPredMore more), 6 + 5.  With 4 for every tile
// and equal items the slowest workgroup took 117 us where the mean was 87;
// without the masked items' share 160 us in all, 155 with it (2 x 2048 tokens,
// 32/8 heads, 516 and 500).
constexpr int kTileCost = 5, kPredTileCost = 7, kPredMore = 2;
constexpr int kMaskMore = 3;
constexpr int kSnap = 3;         // items: no cut nearer to a tile's end

// The key tile at position p of the list.
struct KeyTile {
  int stream, j0;
  int t_hi, t_mid;               // memory keys: both streams see them from row
                                 // tile t_mid on, memory rows alone before
  int items, fixed, cost;        // cost: of the tile and of its items
  int masked;                    // the last of them, in which some wave masks
};

__host__ __device__ inline int key_list(int L) {
  return ((L + kKeysPerWg - 1) / kKeysPerWg + 1) / 2 * 4;
}

__host__ __device__ inline KeyTile key_tile(int L, int block, int G, int p) {
  const int tiles = (L + kKeysPerWg - 1) / kKeysPerWg, T = (L + kRows - 1) / kRows;
  const int i = p >> 2, other = tiles - 1 - i;
  KeyTile x;
  x.stream = p >> 1 & 1;
  x.j0 = (p & 1 ? other : i) * kKeysPerWg;
  x.t_hi = T;
  x.t_mid = x.stream ? T : (x.j0 / block + 1) * block / kRows;
  if (x.t_mid > T) x.t_mid = T;
  // row tiles of a wave's 64 prediction keys: up to the end of the last one's
  // block
  const int own = kOwn % block == 0 ? kOwn / kRows
                                    : (kOwn - 1 + block + kRows - 1) / kRows;
  // the middle tile of an odd number is its own counterpart
  x.items = (p & 1) && other == i ? 0
            : x.stream            ? own * G
                       : ((T - x.t_mid) * 2 + (x.t_mid - x.j0 / kRows)) * G;
  // the row tiles of the keys' own positions end here
  const int diag = x.t_hi < (x.j0 + kKeysPerWg) / kRows
                       ? x.t_hi : (x.j0 + kKeysPerWg) / kRows;
  x.masked = x.stream ? 0
                      : ((x.t_mid < diag ? (diag - x.t_mid) * 2 : 0) +
                         (x.t_mid < diag ? x.t_mid : diag) - x.j0 / kRows) * G;
  x.fixed = x.stream ? kPredTileCost : kTileCost;
  x.cost = x.items == 0 ? 0
                        : x.fixed + (x.stream ? x.items + x.items / kPredMore
                                              : x.items + x.masked / kMaskMore);
  return x;
}

// Where stretch w begins: list position p of group g, after `item` items of
// its tile.
struct Cut {
  int g, p, item;
  __device__ __forceinline__ bool before(const Cut& c) const {
    return g != c.g ? g < c.g : p != c.p ? p < c.p : item < c.item;
  }
  // inside the same tile
  __device__ __forceinline__ bool shares(const Cut& c) const {
    return item > 0 && c.item > 0 && g == c.g && p == c.p;
  }
};

__device__ inline Cut cut_at(const BwdArgs& a, int w) {
  const int groups = a.n_seq * a.Hkv, list = key_list(a.L);
  if (w >= a.W) return {groups, 0, 0};
  const int64_t raw = static_cast<int64_t>(a.group_cost) * groups * w / a.W;
  int g = static_cast<int>(raw / a.group_cost);
  const int x = static_cast<int>(raw - static_cast<int64_t>(g) * a.group_cost);
  int base = 0, p = 0, off = 0;
  for (int p0 = 0; p0 < list; p0 += kWave) {
    const int lp = p0 + lane_id();
    int sum = lp < list ? key_tile(a.L, a.block, a.G, lp).cost : 0;
    const int c = sum;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int y = __shfl_up(sum, o);
      if (lane_id() >= o) sum += y;
    }
    const uint64_t past = ballot(base + sum > x);
    if (past) {
      const int l = __ffsll(static_cast<unsigned long long>(past)) - 1;
      off = x - base - __builtin_amdgcn_readlane(sum - c, l);
      p = p0 + l;
      break;
    }
    base += __builtin_amdgcn_readlane(sum, kWave - 1);
  }
  const KeyTile kt = key_tile(a.L, a.block, a.G, p);
  Cut r{g, p, off - kt.fixed};
  const int slow = r.item - (kt.items - kt.masked);
  if (kt.stream && r.item > 0)
    r.item -= r.item / (kPredMore + 1);
  else if (slow > 0)
    r.item -= slow / (kMaskMore + 1);
  if (r.item < kSnap) {
    r.item = 0;
  } else if (kt.items - r.item < kSnap) {
    r.item = 0;
    if (++r.p == list) {
      r.p = 0;
      ++r.g;
    }
  }
  return r;
}

// The cuts are found once, by dq_kernel's workgroups, the shortest walks first,
// at their ends, for the kernels after it.
__device__ inline void write_cuts(const BwdArgs& a) {
  for (int w = gridDim.x - 1 - blockIdx.x; w <= a.W; w += gridDim.x) {
    const Cut c = cut_at(a, w);
    if (lane_id() == 0) a.cuts[w] = make_int4(c.g, c.p, c.item, 0);
  }
}

__device__ __forceinline__ Cut read_cut(const BwdArgs& a, int w) {
  const int4 c = a.cuts[w];
  return {__builtin_amdgcn_readfirstlane(c.x),
          __builtin_amdgcn_readfirstlane(c.y),
          __builtin_amdgcn_readfirstlane(c.z)};
}

// dq: workgroup = four units (chunk of 32 positions, head) of one stream and
// kv head, one per wave; the longest first, of all sequences (sequence by
// sequence: 4 x 512 tokens 34.6 us against 30.8, 4 x 4096 the same, 2 x 1008
// with 28/4 heads 71 against 73).  Registers and a ring of four
// tiles let two workgroups share a CU (D = 64: three, 4 x 4096 tokens with 32/8
// heads 2.03 ms in all; with two, 2.07), so that the vector work
// of one runs under the products of the others.  With 64 rows a wave, half the
// LDS reads per product but one workgroup per CU: 4 x 4096 tokens (32/8 heads
// of 128) 1.53 ms against 1.47, 1 x 2048 (16/8) 92 us against 68.
constexpr int kDqSlots = 4;

// D from out carries out's rounding, which counts where rows see few keys:
// gradients of 16 to 64 tokens (N(0,1) inputs) were off by 1.5 to 1.8 times one
// rounding of the result.  With the exact D of the first 64 positions it is
// 1.38 to 1.48 at all lengths, of which 1.41 are dS's and the result's own.  The
// walks concerned are the shortest: 1 x 64 tokens (4/2 heads of 64) 27.6 us
// with it, 25.4 without; 1 x 256 28.6, 28.3; longer sequences the same.
constexpr int kExactRows = 64;

template <int D>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(1, D == 64 ? 3 : 2)))
void dq_kernel(BwdArgs a) {
  constexpr int NK = D / 16, NM = D / 32;
  using T = RowTile<D>;
  constexpr int kPair = 2 * T::bytes;
  constexpr int kLoads = PairLoader<D, false>::kCount;
  __shared__ __attribute__((aligned(1024))) char smem[kDqSlots * kPair];
  const int groups = (a.T * a.G + kWaves - 1) / kWaves;
  int wg = blockIdx.x;
  const int kvh = wg % a.Hkv;
  wg /= a.Hkv;
  const int stream = wg & 1;
  wg >>= 1;
  const int grp = groups - 1 - wg / a.n_seq;
  const int sq = wg % a.n_seq;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = lane_id(), col = lane & 31, hf = lane >> 5;
  const int last_unit = a.T * a.G - 1;
  // (past the last unit: it again, its results dropped)
  const int unit = min(grp * kWaves + wave, last_unit);
  const bool live = grp * kWaves + wave <= last_unit;
  const int p0 = unit / a.G * kRows;
  const int head = kvh * a.G + unit % a.G;
  const int64_t row0 = (static_cast<int64_t>(sq) * 2 + stream) * a.L;

  // tiles: memory keys from 0, then for prediction rows their own blocks'
  const int first = grp * kWaves / a.G * kRows;
  const int end = min(a.L, (min(grp * kWaves + kWaves - 1, last_unit) / a.G +
                            1) * kRows);
  const int n_mem =
      ((stream ? (end - 1) / a.block * a.block : end) + kRows - 1) / kRows;
  const int own0 = first / a.block * a.block / kRows;
  const int n = n_mem + (stream ? (end + kRows - 1) / kRows - own0 : 0);
  // memory keys that all of the wave's rows see
  const int full = stream ? p0 / a.block * a.block : p0 + 1;
  const int64_t kv0 = (static_cast<int64_t>(sq) * 2 * a.L * a.Hkv + kvh) * D;
  const PairLoader<D, false> loader(a.k + kv0, a.v + kv0, a.Hkv * D, wave,
                             lds_address(smem));
  // the tile that is loaded next, and its first key's row
  int ahead = 0, ahead_p = n_mem == 0 ? a.L + own0 * kRows : 0;
  auto fetch = [&](int u, int slot) {
    loader.load(u, static_cast<int64_t>(ahead_p) * (a.Hkv * D),
                a.L - 1 - (ahead >= n_mem ? ahead_p - a.L : ahead_p),
                slot * kPair);
  };
  // past the end: the last tile again, into a slot that nobody reads
  auto advance = [&]() {
    ahead = min(ahead + 1, n - 1);
    ahead_p = ahead >= n_mem ? a.L + (own0 + ahead - n_mem) * kRows
                             : ahead * kRows;
  };
  auto prime = [&]() {
#pragma unroll
    for (int i = 0; i < kDqSlots - 1; ++i) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) fetch(u, i);
      advance();
    }
  };
  prime();

  // the lane's row: q, dout, lse and D; it sees memory keys below lo
  // (prediction) or hi (memory), and the own stream's lo .. hi-1
  bf16x8_t qf[NK], dof[NK];
  const int p = p0 + col, pc = min(p, a.L - 1);
  const int lo = stream ? pc / a.block * a.block : 0, hi = pc + 1;
  const int64_t o = ((row0 + pc) * a.Hq + head) * D;
  float delta = 0.f;
#pragma unroll
  for (int kk = 0; kk < NK; ++kk) {
    const int at = kk * 16 + hf * 8;
    qf[kk] = load8(a.q + o + at);
    dof[kk] = load8(a.dout + o + at);
    const bf16x8_t of = load8(a.out + o + at);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      delta += static_cast<float>(dof[kk][e]) * static_cast<float>(of[e]);
  }
  delta += __shfl_xor(delta, 32);
  const float lse2 = a.lse[(row0 + pc) * a.Hq + head] * kLog2e;
  const Reader<D> rd;
  // keys of tile i that the lane's row sees
  auto hide = [=](int i, floatx16_t& x) {
    const bool own = i >= n_mem;
    const int k0 = (own ? own0 + i - n_mem : i) * kRows + 8 * (lane_here() >> 5);
    const uint32_t see =
        rows_between((own ? lo : 0) - k0, (own || !stream ? hi : lo) - k0);
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = seen(see, e, x[e]);
  };
  // rows that see few keys: D from the probabilities, in a walk of its own
  if (first < kExactRows) {
    delta = 0.f;
    for (int i = 0; i < n; ++i) {
      // tile i has landed; everybody is done with the slot of tile i - 1
      wait_vmcnt<0>();
      __syncthreads();
      if (i + kDqSlots - 1 < n) {
#pragma unroll
        for (int u = 0; u < kLoads; ++u) fetch(u, (i + kDqSlots - 1) % kDqSlots);
        advance();
      }
      const char* kt = smem + i % kDqSlots * kPair;
      floatx16_t s{}, dp{};
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) {
        s = mfma(rd.rows(kt, kk), qf[kk], s);
        dp = mfma(rd.rows(kt + T::bytes, kk), dof[kk], dp);
      }
      hide(i, s);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        delta += dp[e] * __builtin_amdgcn_exp2f(
                             __builtin_fmaf(s[e], a.scale_log2, -lse2));
    }
    delta += __shfl_xor(delta, 32);
    // (tiles that all fit are still where prime() put them)
    if (n >= kDqSlots) {
      __syncthreads();
      ahead = 0;
      ahead_p = n_mem == 0 ? a.L + own0 * kRows : 0;
      prime();
    }
  }
  if (live && hf == 0) {
    float* ld = a.ld + ((((static_cast<int64_t>(sq) * a.Hq + head) * 2 + stream) *
                         a.T + p / kRows) * 2) * kRows + col;
    ld[0] = p < a.L ? -lse2 : 0.f;
    ld[kRows] = p < a.L ? -delta : 0.f;
  }
  floatx16_t acc[NM];
#pragma unroll
  for (int m = 0; m < NM; ++m) acc[m] = floatx16_t{};

  // take delivery of the rows: no wait for them in the loop
#pragma unroll
  for (int kk = 0; kk < NK; ++kk)
    asm volatile("" : "+v"(qf[kk]), "+v"(dof[kk]));
  wait_vmcnt<(kDqSlots - 2) * kLoads>();
  __syncthreads();
  constexpr int kE = 16 / NK;              // elements per step
  bf16x8_t f[NK];          // the operands from LDS, read a phase ahead
#pragma unroll
  for (int kk = 0; kk < NK; ++kk) f[kk] = rd.rows(smem, kk);
  int slot = 0, next_slot = 1, load_slot = kDqSlots - 1;
  int i = 0;               // (n > 0: a loop that runs at least once)
  do {
    // this wave's loads of tile i + 1, then everybody's; the barrier also
    // frees the slot of tile i - 1
    wait_vmcnt<(kDqSlots - 3) * kLoads>();
    meet();
    const char* kt = smem + slot * kPair;
    const char* vt = kt + T::bytes;
    // A tile that this wave's rows do not see is computed all the same, P = 0:
    // the waves are in step, and a branch around the accumulators costs copies
    floatx16_t s, dp;
    float w[16];
    bf16x8_t ds[2];
    // Three phases of NK = 2 NM MFMAs: S, dP, dq
    step();
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      s = mfma(f[kk], qf[kk], kk ? s : floatx16_t{});
      f[kk] = rd.rows(vt, kk);
      if (kk >= 1 && kk <= kLoads) fetch(kk - 1, load_slot);
      step();
    }
    if (i >= n_mem || (i + 1) * kRows > full) hide(i, s);
    step();
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      dp = mfma(f[kk], dof[kk], kk ? dp : floatx16_t{});
      f[kk] = rd.cols(kt, kk / NM, kk % NM);
#pragma unroll
      for (int e = kk * kE; e < kk * kE + kE; ++e) {
        w[e] = __builtin_amdgcn_exp2f(
            __builtin_fmaf(s[e], a.scale_log2, -lse2));
        here(w[e]);
      }
      step();
    }
#pragma unroll
    for (int e = 0; e < 16; ++e)
      ds[e >> 3][e & 7] = static_cast<__bf16>(w[e] * (dp[e] - delta));
    const char* nt = smem + next_slot * kPair;
#pragma unroll
    for (int x = 0; x < NK; ++x) {
      if (x % NM == 0) settle(ds[x / NM]);
      mfma_acc(acc[x % NM], f[x], ds[x / NM]);
      f[x] = rd.rows(nt, x);
      step();
    }
    advance();
    load_slot = slot;
    slot = next_slot;
    next_slot = next_slot == kDqSlots - 1 ? 0 : next_slot + 1;
  } while (++i < n);
  wait_vmcnt<0>();      // surplus loads land before the LDS is given up
  drain(acc);
  if (wave == 0) write_cuts(a);
  if (!live || p >= a.L) return;
  uint16_t* dst = a.dq + o;
#pragma unroll
  for (int m = 0; m < NM; ++m)
#pragma unroll
    for (int j = 0; j < 2; ++j) store_row(dst, m, j, hf, acc[m], a.scale);
}

// Partial sums of one tile, float4 by float4 as the waves' lanes hold them (a
// lane's keys are rows of memory apart, its own order is whole lines):
// [wave][dk, dv][b][m][g][lane], dk without the scale.
template <int D>
struct Piece {
  static constexpr int per_wave = 2 * kOwn * D / 4;
  static constexpr int n = kWaves * per_wave;
  __device__ static __forceinline__ int64_t at(int piece, int wave) {
    return static_cast<int64_t>(piece) * n + wave * per_wave;
  }
};

// dk and dv: workgroup w walks stretch w; workgroups of one XCD take
// neighbouring stretches, of kv heads whose rows then stay in its L2.
template <int D>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(1)))
void dkv_kernel(BwdArgs a) {
  constexpr int NK = D / 16, NM = D / 32;
  using T = RowTile<D>;
  constexpr int kPair = 2 * T::bytes;
  constexpr int kSlot = kPair + 2 * kRows * 4;     // rows' -lse, -D behind
  // the ring, or two slots for each wave and one that nobody reads
  constexpr int kAll = 2 * kWaves + 1;
  static_assert(kAll >= kSlots, "the ring");
  __shared__ __attribute__((aligned(1024))) char smem[kAll * kSlot];
  // the first row of the block after a lane's key's (divisions, and no register
  // is left for their results in the loop)
  __shared__ int s_next[2][kThreads];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int W = a.W, list = key_list(a.L);
  const int w = W % 8 == 0 ? blockIdx.x % 8 * (W / 8) + blockIdx.x / 8
                           : static_cast<int>(blockIdx.x);
  const Cut end = read_cut(a, w + 1);
  Cut at = read_cut(a, w);
  const Reader<D> rd;
  for (; at.before(end); at.item = 0, at.p = at.p + 1 == list ? 0 : at.p + 1,
                         at.g += at.p == 0) {
  const KeyTile kt = key_tile(a.L, a.block, a.G, at.p);
  const int it0 = at.item;
  const int it1 = at.g == end.g && at.p == end.p ? end.item : kt.items;
  if (it0 >= it1) continue;
  const int stream = kt.stream, j0 = kt.j0;
  const int kvh = at.g / a.n_seq, sq = at.g - kvh * a.n_seq;
  const int kw0 = j0 + wave * kOwn;
  // the last tile's reads of the ring are done
  __syncthreads();
  const int lane = lane_here(), col = lane & 31, hf = lane >> 5;

  bf16x8_t kf[2][NK], vf[2][NK];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int jc = min(kw0 + 32 * b + col, a.L - 1);
    const int64_t o =
        (((static_cast<int64_t>(sq) * 2 + stream) * a.L + jc) * a.Hkv + kvh) * D;
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      kf[b][kk] = load8(a.k + o + kk * 16 + hf * 8);
      vf[b][kk] = load8(a.v + o + kk * 16 + hf * 8);
    }
  }
  floatx16_t dk[2][NM], dv[2][NM];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int m = 0; m < NM; ++m) dk[b][m] = dv[b][m] = floatx16_t{};

  // Items of memory keys: row tiles t from the last down, in each the streams
  // that see the keys (memory, prediction) and their heads; the waves share
  // the tiles.  Every workgroup of a kv head starts at the same rows, which
  // they then find in the L2.  Items of prediction keys: each wave's own few
  // row tiles from its first key on, in each the heads; every wave loads for
  // itself, a tile ahead, into two slots of its own.
  // Steps are branches, so that everything stays in scalar registers
  const int t_hi = kt.t_hi, t_mid = kt.t_mid;
  const int n1 = (t_hi - t_mid) * 2 * a.G;
  struct Item {
    int t, rs, g;             // row tile, its rows' stream, head of the group
  };
  auto item_at = [&](int it) {
    Item x;
    if (stream) {
      x.t = kw0 / kRows + it / a.G;
      x.g = it;
      x.rs = 1;
    } else if (it < n1) {
      x.t = t_hi - 1 - it / (2 * a.G);
      x.g = it % (2 * a.G);
      x.rs = x.g / a.G;
    } else {
      x.t = t_mid - 1 - (it - n1) / a.G;
      x.g = it - n1;
      x.rs = 0;
    }
    x.g %= a.G;
    return x;
  };
  auto next_item = [&](Item& x) {
    if (++x.g < a.G) return;
    x.g = 0;
    if (stream) {
      ++x.t;
    } else if (x.rs == 0 && x.t >= t_mid) {
      x.rs = 1;
    } else {
      x.rs = 0;
      --x.t;
    }
  };
  const uint32_t lds0 = lds_address(smem);
  const int64_t q0 = (static_cast<int64_t>(sq) * 2 * a.L * a.Hq + kvh * a.G) * D;
  const PairLoader<D, true> loader(a.q + q0, a.dout + q0, a.Hq * D, wave,
                                   lds0);
  constexpr int kLoads = PairLoader<D, true>::kCount + 1;
  const float* ld0 = a.ld + (static_cast<int64_t>(sq) * a.Hq + kvh * a.G) * 2 *
                                a.T * 2 * kRows;
  // the item that is loaded next
  Item ahead = item_at(it0);
  int n_ahead = it0;
  auto row_values_at = [&]() {
    return ld0 + static_cast<int64_t>((ahead.g * 2 + ahead.rs) * a.T +
                                      min(ahead.t, a.T - 1)) * (2 * kRows);
  };
  auto rows_at = [&]() {       // elements from q0 (row tiles past the last: it)
    return static_cast<int64_t>(ahead.rs * a.L + min(ahead.t, a.T - 1) * kRows) *
               (a.Hq * D) + ahead.g * D;
  };
  auto fetch = [&](int u, int slot) {
    const int left = a.L - 1 - min(ahead.t, a.T - 1) * kRows;
    if (u < PairLoader<D, true>::kCount)
      loader.load(u, rows_at(), left, slot * kSlot);
    else
      // every wave the same 256 bytes, so that all wait for as many loads
      load_to_lds4(buffer_rsrc(row_values_at(), 2 * kRows * 4), lane_here() * 4,
                   lds0 + slot * kSlot + kPair);
  };
  // the whole of a tile by this wave
  auto fetch_own = [&](int slot) {
    const int left = a.L - 1 - min(ahead.t, a.T - 1) * kRows;
    const int64_t o = rows_at();
    const int l = lane_here(), i = l / T::chunks;
    const int chunk = ((l % T::chunks) ^ T::swz(i)) * 16, stride = a.Hq * D * 2;
#pragma unroll
    for (int g = 0; g < 2 * T::groups; ++g)
      load_to_lds16<false>(
          buffer_rsrc((g < T::groups ? a.q : a.dout) + q0 + o,
                      31 * stride + 2 * D),
          min(g % T::groups * T::per_group + i, left) * stride + chunk,
          lds0 + slot * kSlot + g * T::group_bytes);
    load_to_lds4(buffer_rsrc(row_values_at(), 2 * kRows * 4), l * 4,
                 lds0 + slot * kSlot + kPair);
  };
  // past the end: the last item again, into a slot that nobody reads
  auto advance = [&]() {
    if (++n_ahead < it1) next_item(ahead);
  };
  constexpr int kE = 16 / NK;              // elements per step
  bf16x8_t f[NK];          // the operands from LDS, read a phase ahead
  const int kwl = min(kw0 + kOwn, a.L) - 1;         // the wave's last key
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int k0 = min(kw0 + 32 * b + (lane_here() & 31), a.L - 1);
    s_next[b][threadIdx.x] = min(a.L, (k0 / a.block + 1) * a.block);
  }
  const int next_hi = (kwl / a.block + 1) * a.block;
  Item cur = item_at(it0);
  int slot, next_slot, load_slot;
  if (stream) {
    slot = 2 * wave;
    next_slot = slot + 1;
    load_slot = 2 * kWaves;        // the shared loads go where nobody reads
    fetch_own(slot);
    advance();
  } else {
    slot = 0;
    next_slot = 1;
    load_slot = kSlots - 1;
#pragma unroll
    for (int i = 0; i < kSlots - 1; ++i) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) fetch(u, i);
      advance();
    }
  }
  // take delivery of the keys: no wait for them in the loop
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int kk = 0; kk < NK; ++kk)
      asm volatile("" : "+v"(kf[b][kk]), "+v"(vf[b][kk]));
  if (!stream) {
    wait_vmcnt<(kSlots - 2) * kLoads>();
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) f[kk] = rd.rows(smem, kk);
  }
  int it = it0;            // (it0 < it1)
  do {
    if (stream) {
      // this wave's tile; the other slot is free
      wait_vmcnt<0>();
      asm volatile("" ::: "memory");
      fetch_own(next_slot);
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) f[kk] = rd.rows(smem + slot * kSlot, kk);
    } else {
      // this wave's loads of the next item, then everybody's; the barrier also
      // frees the slot of the previous one
      wait_vmcnt<(kSlots - 3) * kLoads>();
      meet();
    }
    const char* qt = smem + slot * kSlot;
    const char* ot = qt + T::bytes;
    const floatx4_t* ldt =
        reinterpret_cast<const floatx4_t*>(qt + kPair) + 2 * hf;
    const int p0 = cur.t * kRows;
    // a mask unless every row sees all keys of the wave.  (A tile of which it
    // sees none is computed all the same, P = 0, as in dq_kernel)
    const bool pred = cur.rs > stream;      // prediction rows, memory keys
    const bool mask = stream || p0 < (pred ? next_hi : kwl) ||
                      p0 + kRows > a.L || kw0 + kOwn > a.L;
    floatx16_t s[2], dp[2];
    floatx4_t nl[4];
    float p[2][16];
    bf16x8_t pb[2][2], ds[2][2];
    auto hide = [&](int b) {
      // a lane's key k0 of the memory is seen by memory rows k0 .. L-1 and
      // prediction rows next .. L-1 (next: the block after the key's), one of
      // the prediction by prediction rows k0 .. next-1
      const int l = lane_here();
      const int k0 = kw0 + 32 * b + (l & 31), i0 = p0 + 8 * (l >> 5);
      const int next = s_next[b][threadIdx.x];
      const int from = pred ? next : k0;
      const int to = k0 < a.L ? stream ? next : a.L : 0;
      const uint32_t see = rows_between(from - i0, to - i0);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[b][e] = seen(see, e, s[b][e]);
    };
    // -lse (x < 4) and -D (x >= 4) of rows 16 (x / 2 % 2) + 8 hf + 4 (x % 2) ..
    auto row_values = [&](int x) {
      return ldt[8 * (x >> 2) + 4 * (x >> 1 & 1) + (x & 1)];
    };
    auto weigh = [&](int b, int kk) {       // P
#pragma unroll
      for (int e = kk * kE; e < kk * kE + kE; ++e) {
        p[b][e] = __builtin_amdgcn_exp2f(
            __builtin_fmaf(s[b][e], a.scale_log2, nl[e >> 2][e & 3]));
        here(p[b][e]);
        pb[b][e >> 3][e & 7] = static_cast<__bf16>(p[b][e]);
      }
    };
    // dP starts from -D, read straight into its accumulator
    auto minus_d = [&](int b, int x) {
      const floatx4_t v = row_values(4 + x);
#pragma unroll
      for (int e = 0; e < 4; ++e) dp[b][4 * x + e] = v[e];
    };
    auto grad = [&](int b, int kk) {        // dS
#pragma unroll
      for (int e = kk * kE; e < kk * kE + kE; ++e)
        ds[b][e >> 3][e & 7] = static_cast<__bf16>(p[b][e] * dp[b][e]);
    };
    // Eight phases of NK = 2 NM MFMAs: S, dV, dP, dK for either group of keys
    // (dV before dP, so that P's operands are gone when dP needs registers).
    // The vector work on a product starts a step after its last MFMA
    step();
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      s[0] = mfma(f[kk], kf[0][kk], kk ? s[0] : floatx16_t{});
      if (kk < 4) nl[kk] = row_values(kk);
      if (kk >= 1 && kk <= kLoads) fetch(kk - 1, load_slot);
      step();
    }
    if (mask) hide(0);
    step();
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      s[1] = mfma(f[kk], kf[1][kk], kk ? s[1] : floatx16_t{});
      f[kk] = rd.cols(ot, kk / NM, kk % NM);
      if (kk) weigh(0, kk - 1);
      step();
    }
    if (mask) hide(1);
    step();
#pragma unroll
    for (int x = 0; x < NK; ++x) {
      if (x % NM == 0) settle(pb[0][x / NM]);
      mfma_acc(dv[0][x % NM], f[x], pb[0][x / NM]);
      weigh(x ? 1 : 0, x ? x - 1 : NK - 1);
      step();
    }
#pragma unroll
    for (int x = 0; x < NK; ++x) {
      if (x % NM == 0) settle(pb[1][x / NM]);
      mfma_acc(dv[1][x % NM], f[x], pb[1][x / NM]);
      f[x] = rd.rows(ot, x);
      if (x == 0) weigh(1, NK - 1);
      if (x < 4) minus_d(0, x);
      step();
    }
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      dp[0] = mfma(f[kk], vf[0][kk], dp[0]);
      if (kk < 4) minus_d(1, kk);
      step();
    }
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      dp[1] = mfma(f[kk], vf[1][kk], dp[1]);
      f[kk] = rd.cols(qt, kk / NM, kk % NM);
      if (kk) grad(0, kk - 1);
      step();
    }
#pragma unroll
    for (int x = 0; x < NK; ++x) {
      if (x % NM == 0) settle(ds[0][x / NM]);
      mfma_acc(dk[0][x % NM], f[x], ds[0][x / NM]);
      grad(x ? 1 : 0, x ? x - 1 : NK - 1);
      step();
    }
    const char* nt = smem + next_slot * kSlot;
#pragma unroll
    for (int x = 0; x < NK; ++x) {
      if (x % NM == 0) settle(ds[1][x / NM]);
      mfma_acc(dk[1][x % NM], f[x], ds[1][x / NM]);
      f[x] = rd.rows(nt, x);
      if (x == 0) grad(1, NK - 1);
      step();
    }
    next_item(cur);
    advance();
    if (stream) {
      slot = next_slot;
      next_slot ^= 1;
    } else {
      load_slot = slot;
      slot = next_slot;
      next_slot = next_slot == kSlots - 1 ? 0 : next_slot + 1;
    }
  } while (++it < it1);
  wait_vmcnt<0>();      // surplus loads land before the LDS is given up
  drain(dv[0]);
  drain(dv[1]);
  drain(dk[0]);
  drain(dk[1]);
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int l = lane_here(), hf = l >> 5;
    const int key = kw0 + 32 * b + (l & 31);
    if (key >= a.L) continue;
    if (it0 == 0 && it1 == kt.items) {
      const int64_t o =
          (((static_cast<int64_t>(sq) * 2 + stream) * a.L + key) * a.Hkv + kvh) *
          D;
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          store_row(a.dk + o, m, j, hf, dk[b][m], a.scale);
          store_row(a.dv + o, m, j, hf, dv[b][m], 1.f);
        }
    } else {
      floatx4_t* o = reinterpret_cast<floatx4_t*>(a.part) +
                     Piece<D>::at(2 * w + (it0 == 0), (kw0 - j0) / kOwn) + l;
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          floatx4_t x, y;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[e] = dk[b][m][4 * g + e];
            y[e] = dv[b][m][4 * g + e];
          }
          o[((b * NM + m) * 4 + g) * kWave] = x;
          o[(((2 + b) * NM + m) * 4 + g) * kWave] = y;
        }
    }
  }
  }
}

// dk and dv of the cut tiles: workgroup row w adds up the partial sums of the
// tile whose first cut is w (the piece before it is stretch w-1's last, the
// others are their stretches' first).
template <int D>
__global__ __launch_bounds__(kThreads) void join_kernel(BwdArgs a) {
  const int w = blockIdx.x + 1;
  const Cut c = read_cut(a, w);
  if (c.item == 0 || read_cut(a, w - 1).shares(c)) return;
  int n = 1;
  while (w + n < a.W && read_cut(a, w + n).shares(c)) ++n;
  const KeyTile kt = key_tile(a.L, a.block, a.G, c.p);
  const int kvh = c.g / a.n_seq, sq = c.g - kvh * a.n_seq;
  const floatx4_t* part = reinterpret_cast<const floatx4_t*>(a.part);
  const floatx4_t* first = part + Piece<D>::at(2 * w - 1, 0);
  const floatx4_t* others = part + Piece<D>::at(2 * w, 0);
  for (int i = blockIdx.y * kThreads + threadIdx.x; i < Piece<D>::n;
       i += gridDim.y * kThreads) {
    const int lane = i % kWave, g = i / kWave % 4;
    const int m = i / (4 * kWave) % (D / 32), x2 = i / (2 * kWave * D / 16);
    const int key = kt.j0 + x2 / 4 * kOwn + x2 % 2 * 32 + lane % 32;
    if (key >= a.L) continue;
    floatx4_t s = first[i];
    // in order, four loads under way
    for (int k0 = 0; k0 < n; k0 += 4) {
      floatx4_t x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        x[k] = others[Piece<D>::at(2 * min(k0 + k, n - 1), 0) + i];
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += k0 + k < n ? x[k][e] : 0.f;
    }
    const float scale = x2 & 2 ? 1.f : a.scale;
    u16x4_t o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = to_bf16(s[e] * scale);
    *reinterpret_cast<u16x4_t*>(
        (x2 & 2 ? a.dv : a.dk) +
        (((static_cast<int64_t>(sq) * 2 + kt.stream) * a.L + key) * a.Hkv +
         kvh) * D + 32 * m + 8 * g + lane / 32 * 4) = o;
  }
}

struct BwdPlan {
  int T, W, group_cost;
  size_t cuts, part, total;
  unsigned dq_grid;
};

size_t up256(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }

bool bwd_plan(int n_seq, int L, int block, int Hq, int Hkv, int D,
              BwdPlan* p) {
  // the forward's limits
  if (wedlm_dual_stream_attn_workspace_size(n_seq, L, block, Hq, Hkv, D) == 0)
    return false;
  const int G = Hq / Hkv;
  p->T = (L + kRows - 1) / kRows;
  // offsets within a tile of rows, and a tile's items, are 32-bit numbers
  if (static_cast<int64_t>(Hq) * D * 2 * kRows > 0x7fffffffll ||
      2ll * p->T * G > 0x3fffffffll)
    return false;
  const int64_t dq = 2ll * n_seq * Hkv *
                     ((static_cast<int64_t>(p->T) * G + kWaves - 1) / kWaves);
  int64_t cost = 0;
  for (int i = 0; i < key_list(L); ++i) {
    cost += key_tile(L, block, G, i).cost;
  }
  // cut_at() counts a (sequence, kv head)'s work in 32 bits; beyond them a call
  // would take the card more than ten seconds
  if (dq > 0x7fffffffll || cost > 0x7fffffffll) return false;
  // One workgroup per CU, but none with less than six items' work.  (At least
  // 16 items, longer walks but fewer partial sums: 1 x 256 tokens, 4/2 heads of
  // 64, dk and dv 28 us against 15; 1 x 1024, 8/2 heads of 128, 42 against 28
  // with a join of 8 against 16; eight items tie)
  const int64_t all = cost * n_seq * Hkv;
  p->W = static_cast<int>(std::min<int64_t>(256, std::max<int64_t>(1, all / 6)));
  p->group_cost = static_cast<int>(cost);
  p->dq_grid = static_cast<unsigned>(dq);
  p->cuts = up256(static_cast<size_t>(n_seq) * Hq * 2 * p->T * 2 * kRows * 4);
  p->part = p->cuts + up256((p->W + 1) * sizeof(int4));
  p->total = p->part;
  if (p->W > 1)
    p->total += static_cast<size_t>(p->W) * 2 * 2 * kKeysPerWg * D * 4;
  return true;
}

}  // namespace

extern "C" size_t wedlm_dual_stream_attn_backward_workspace_size(
    int32_t n_seq, int32_t L, int32_t block, int32_t Hq, int32_t Hkv,
    int32_t D) {
  BwdPlan p;
  return bwd_plan(n_seq, L, block, Hq, Hkv, D, &p) ? p.total : 0;
}

extern "C" int wedlm_dual_stream_attn_backward(
    const uint16_t* q, const uint16_t* k, const uint16_t* v,
    const uint16_t* out, const float* lse, const uint16_t* dout, int32_t n_seq,
    int32_t L, int32_t block, int32_t Hq, int32_t Hkv, int32_t D,
    float softmax_scale, uint16_t* dq, uint16_t* dk, uint16_t* dv,
    void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !k || !v || !out || !lse || !dout || !dq || !dk || !dv)
    return WEDLM_E_ARG;
  if (!(softmax_scale > 0.f) || !(softmax_scale < 1e30f)) return WEDLM_E_ARG;
  // rows are loaded in 16-byte pieces
  for (const void* x : std::initializer_list<const void*>{
           q, k, v, out, dout, dq, dk, dv, workspace})
    if (reinterpret_cast<uintptr_t>(x) % 16 != 0) return WEDLM_E_ARG;
  BwdPlan p;
  if (!bwd_plan(n_seq, L, block, Hq, Hkv, D, &p)) return WEDLM_E_SHAPE;
  if (!workspace || workspace_bytes < p.total) return WEDLM_E_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  BwdArgs a{};
  a.q = q;
  a.k = k;
  a.v = v;
  a.out = out;
  a.lse = lse;
  a.dout = dout;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.ld = reinterpret_cast<float*>(ws);
  a.cuts = reinterpret_cast<int4*>(ws + p.cuts);
  a.part = reinterpret_cast<float*>(ws + p.part);
  a.n_seq = n_seq;
  a.L = L;
  a.block = block;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  a.T = p.T;
  a.W = p.W;
  a.group_cost = p.group_cost;
  a.scale = softmax_scale;
  a.scale_log2 = softmax_scale * kLog2e;
  hipLaunchKernelGGL(D == 128 ? dq_kernel<128> : dq_kernel<64>,
                     dim3(p.dq_grid), dim3(kThreads), 0, st, a);
  WEDLM_LAUNCH_CHECK();
  hipLaunchKernelGGL(D == 128 ? dkv_kernel<128> : dkv_kernel<64>,
                     dim3(p.W), dim3(kThreads), 0, st, a);
  WEDLM_LAUNCH_CHECK();
  if (p.W > 1) {
    hipLaunchKernelGGL(D == 128 ? join_kernel<128> : join_kernel<64>,
                       dim3(p.W - 1, 2 * kKeysPerWg * (D / 4) / kThreads),
                       dim3(kThreads), 0, st, a);
    WEDLM_LAUNCH_CHECK();
  }
  return WEDLM_OK;
}
