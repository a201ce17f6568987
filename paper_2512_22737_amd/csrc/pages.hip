// Pages of a pool shared between the rows of a block table: free, fork,
// compact (wedlm_cache_free, _fork, _compact).
//
// The bookkeeping is integer work on the table and the pages' counts, done by
// one workgroup per call where an order has to be kept (free pages are given
// lowest first, requests in order): its scan of the counts reads 16 or 32 KB a
// step; a fork's ends when enough free pages are found.  The tables and the
// copies of all arrays and layers follow in one launch, copies as wide as the
// pages are aligned.  No result depends on an order of atomics: they only add
// integers.
// Bound by latency where little is copied (8 samples of one prompt, 36 layers:
// free 2.3, plan 6.8, tables and copies 5.4 us); by HBM where much is
// (compaction of 8192 pages, 1.03 GB read and written: 211 us, 4.9 TB/s, and
// 16 us of plan).
#include "common.h"
#include "wedlm_serve.h"

using namespace wedlm;

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;

// ---------------------------------------------------------------------------
// sums over a workgroup
// ---------------------------------------------------------------------------

template <typename T>
__device__ __forceinline__ T wave_scan(T v) {          // inclusive
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const T u = __shfl_up(v, off);
    if (lane_id() >= off) v += u;
  }
  return v;
}

// Exclusive sums over the workgroup's threads; `total` to all of them.
template <typename T>
__device__ __forceinline__ T group_scan(T v, T* lds, T& total) {
  const int wave = threadIdx.x / kWave;
  const T s = wave_scan(v);
  __syncthreads();                      // lds is free again
  if (lane_id() == kWave - 1) lds[wave] = s;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const T t = lds[w];
    before += w < wave ? t : 0;
    all += t;
  }
  total = all;
  return before + s - v;
}

// ---------------------------------------------------------------------------
// free
// ---------------------------------------------------------------------------

struct FreeArgs {
  const int32_t* rows;
  int32_t* bt;
  int32_t* ref;
  int32_t* plen;
  int num_pages, B, max_pages;
};

__global__ __launch_bounds__(256) void cache_free_kernel(FreeArgs a) {
  const int row = a.rows[blockIdx.x];
  if (row < 0 || row >= a.B) return;
  if (a.plen && blockIdx.y == 0 && threadIdx.x == 0) a.plen[row] = 0;
  int32_t* bt = a.bt + static_cast<int64_t>(row) * a.max_pages;
  for (int64_t j = static_cast<int64_t>(blockIdx.y) * 256 + threadIdx.x;
       j < a.max_pages; j += static_cast<int64_t>(gridDim.y) * 256) {
    // the exchange gives an entry to one of the workgroups that have this row
    const int id = atomicExch(bt + j, -1);
    if (id < 0 || id >= a.num_pages) continue;
    // (a count that was 0 already is put back)
    if (atomicSub(a.ref + id, 1) <= 0) atomicAdd(a.ref + id, 1);
  }
}

// ---------------------------------------------------------------------------
// fork
// ---------------------------------------------------------------------------

struct ForkArgs {
  const int32_t* parent;
  const int32_t* child;
  const int32_t* reserve;
  int32_t* plen;
  int32_t* bt;
  int32_t* ref;
  int32_t* status;
  int32_t* first;         // n: its first page among the free ones
  int32_t* free_ids;      // the free pages that are given
  int n, B, max_pages, num_pages;
};

// One request's shape: entries [0, full) are the parent's, [full, upto) need
// pages (of an extended row: those that have none).
struct Request {
  int why, p, c, row, full, upto, need;
  bool extend;
};

__device__ Request read_request(const ForkArgs& a, int i) {
  Request q;
  q.p = a.parent[i];
  q.row = a.child[i];
  q.why = 0;
  q.c = q.full = q.upto = q.need = 0;
  q.extend = q.p == q.row;
  if (q.row < 0 || q.row >= a.B || q.p < -1 || q.p >= a.B) {
    q.why = WEDLM_SEQ_BAD_ROW;
    return q;
  }
  q.c = q.p < 0 ? 0 : a.plen[q.p];
  const int want = max(q.c, a.reserve[i]);
  // whole pages without overflow near 2^31
  const int64_t upto = (static_cast<int64_t>(max(want, 0)) + kPage - 1) / kPage;
  if (q.c < 0 || upto > a.max_pages) {
    q.why = WEDLM_SEQ_BAD_LEN;
    return q;
  }
  q.full = q.extend ? 0 : q.c / kPage;
  q.upto = static_cast<int>(upto);
  return q;
}

// Checks request i, one wave (every lane gets the same answer), and counts
// the pages it needs.
__device__ Request check_request(const ForkArgs& a, int i) {
  Request q = read_request(a, i);
  if (q.why) return q;
  const int lane = lane_id();
  // another request's child or parent
  bool clash = false;
  for (int k = lane; k < a.n; k += kWave)
    if (k != i && (a.child[k] == q.row || a.parent[k] == q.row)) clash = true;
  const int32_t* own = a.bt + static_cast<int64_t>(q.row) * a.max_pages;
  int need = q.upto - q.full;
  if (q.extend) {
    int have = 0;
    for (int j = lane; j < q.upto; j += kWave) have += own[j] >= 0 ? 1 : 0;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) have += __shfl_xor(have, off);
    need = q.upto - have;
  } else {
    // (unsigned: the step behind the last of 2^31 - 1 entries counts on)
#pragma unroll 8
    for (uint32_t j = lane; j < static_cast<uint32_t>(a.max_pages); j += kWave)
      if (own[j] >= 0) clash = true;
  }
  if (ballot(clash)) {
    q.why = WEDLM_SEQ_BAD_ROW;
    return q;
  }
  if (!q.extend && q.p >= 0) {
    const int32_t* from = a.bt + static_cast<int64_t>(q.p) * a.max_pages;
    bool bad = false;
    const int pages = q.c / kPage + (q.c % kPage != 0 ? 1 : 0);
#pragma unroll 8
    for (int j = lane; j < pages; j += kWave) {
      const int id = from[j];
      if (id < 0 || id >= a.num_pages) bad = true;
    }
    if (ballot(bad)) {
      q.why = WEDLM_SEQ_BAD_PAGE;
      return q;
    }
  }
  q.need = need;
  return q;
}

// The checks, a wave per request: status, and the need in first[].
__global__ __launch_bounds__(256) void fork_check_kernel(ForkArgs a) {
  const int i = blockIdx.x * (256 / kWave) + threadIdx.x / kWave;
  if (i >= a.n) return;
  const Request q = check_request(a, i);
  if (lane_id() == 0) {
    a.status[i] = q.why;
    a.first[i] = q.why ? 0 : q.need;
  }
}

// First pages of the requests (in order, as far as the free pages reach) and
// the list of the lowest free pages, one workgroup.  Up to as many requests as
// it has waves are checked here too, which saves a launch (8 requests: 6.8 us
// for both; the check alone takes 4.2 and a gap before the next kernel).
__global__ __launch_bounds__(kThreads) void fork_plan_kernel(ForkArgs a) {
  __shared__ int lds[kWaves];
  __shared__ long long sums[kWaves];
  int total;
  long long wanted;       // a few requests can ask for 2^31 pages together
  if (a.n <= kWaves) {
    const int i = threadIdx.x / kWave;
    if (i < a.n) {
      const Request q = check_request(a, i);
      if (lane_id() == 0) {
        a.status[i] = q.why;
        a.first[i] = q.why ? 0 : q.need;
      }
    }
    __syncthreads();
  }
  // pages wanted in all
  int64_t want = 0;
  for (int base = 0; base < a.n; base += kThreads) {
    const int i = base + threadIdx.x;
    group_scan<long long>(i < a.n ? a.first[i] : 0, sums, wanted);
    want += wanted;
  }
  // the lowest free pages, until there are enough
  int found = 0;
  for (int64_t base = 0; base < a.num_pages && found < want;
       base += 4 * kThreads) {
    int f[4], here = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t id = base + 4 * static_cast<int64_t>(threadIdx.x) + k;
      f[k] = id < a.num_pages && a.ref[id] <= 0 ? 1 : 0;
      here += f[k];
    }
    int at = found + group_scan(here, lds, total);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (f[k]) {
        if (at < want)
          a.free_ids[at] =
              static_cast<int>(base + 4 * static_cast<int64_t>(threadIdx.x) + k);
        ++at;
      }
    found += total;
  }
  // the first request that does not fit gets none, nor does any later one that
  // needs some (the sums only grow)
  int64_t given = 0;
  for (int base = 0; base < a.n; base += kThreads) {
    const int i = base + threadIdx.x;
    const int need = i < a.n ? a.first[i] : 0;
    const int64_t at = given + group_scan<long long>(need, sums, wanted);
    if (i < a.n) {
      if (need > 0 && at + need > found) a.status[i] = WEDLM_SEQ_CAPACITY;
      a.first[i] = static_cast<int>(min(at, static_cast<int64_t>(found)));
    }
    given += wanted;
  }
}

// ---------------------------------------------------------------------------
// copies
// ---------------------------------------------------------------------------

struct CopyArgs {
  struct {
    char* base;
    int64_t bytes;        // of a page
    int shift;            // log2 of the words that a page is copied in
  } array[WEDLM_MAX_ARRAYS];
  int n_arrays;
  int64_t num_pages;
};

// One page of `words` words: `lanes` threads, this one the `at`-th.
template <typename T>
__device__ __forceinline__ void copy_words(const char* from, char* to,
                                           int64_t words, int at, int lanes) {
  const T* s = reinterpret_cast<const T*>(from);
  T* d = reinterpret_cast<T*>(to);
  int64_t i = at;
  // four loads under way before the first store
  for (; i + 3 * lanes < words; i += 4 * lanes) {
    const T w0 = s[i], w1 = s[i + lanes], w2 = s[i + 2 * lanes],
            w3 = s[i + 3 * lanes];
    d[i] = w0;
    d[i + lanes] = w1;
    d[i + 2 * lanes] = w2;
    d[i + 3 * lanes] = w3;
  }
  for (; i < words; i += lanes) d[i] = s[i];
}

// Page copies m = first, first + step, ... < n of one array and layer, by a
// workgroup of 256; pair(m, from, to) is false for none.  Pages of few words
// (exponents) are taken several at a time.
template <typename F>
__device__ __forceinline__ void copy_pages(const CopyArgs& a, int which,
                                           int64_t layer, int n, int first,
                                           int step, F pair) {
  const int64_t bytes = a.array[which].bytes;
  char* base = a.array[which].base + layer * a.num_pages * bytes;
  const int shift = a.array[which].shift;
  const int64_t words = bytes >> shift;
  const int lanes = words <= 4 ? 4 : words <= 32 ? 32 : 256;
  const int at = threadIdx.x % lanes, many = 256 / lanes;
  const int64_t by = static_cast<int64_t>(step) * many;
  int64_t m = static_cast<int64_t>(first) * many + threadIdx.x / lanes;
  int64_t from = 0, to = 0;
  bool have = m < n && pair(static_cast<int>(m), from, to);
  while (m < n) {
    // the next pair is read under this copy
    const int64_t s_at = from * bytes, d_at = to * bytes;
    const bool now = have;
    m += by;
    have = m < n && pair(static_cast<int>(m), from, to);
    if (!now) continue;
    const char* s = base + s_at;
    char* d = base + d_at;
    if (shift == 4) copy_words<u32x4_t>(s, d, words, at, lanes);
    else if (shift == 2) copy_words<uint32_t>(s, d, words, at, lanes);
    else copy_words<uint8_t>(s, d, words, at, lanes);
  }
}

// Tables and counts of request i, a workgroup.
__device__ void assign(const ForkArgs& a, int i) {
  if (a.status[i]) return;
  const Request q = read_request(a, i);
  const int first = a.first[i];
  int32_t* own = a.bt + static_cast<int64_t>(q.row) * a.max_pages;
  if (q.extend) {
    // entries without a page, in order: one wave
    if (threadIdx.x >= kWave) return;
    int at = first;
    for (int base = 0; base < q.upto; base += kWave) {
      const int j = base + lane_id();
      const bool miss = j < q.upto && own[j] < 0;
      const uint64_t m = ballot(miss);
      if (miss) {
        const int id = a.free_ids[at + __popcll(m & ((1ull << lane_id()) - 1))];
        own[j] = id;
        a.ref[id] = 1;
      }
      at += __popcll(m);
    }
    return;
  }
  const int32_t* from =
      a.bt + static_cast<int64_t>(max(q.p, 0)) * a.max_pages;
  for (int j = threadIdx.x; j < q.upto; j += 256) {
    if (j < q.full) {
      const int id = from[j];
      own[j] = id;
      atomicAdd(a.ref + id, 1);
    } else {
      const int id = a.free_ids[first + j - q.full];
      own[j] = id;
      a.ref[id] = 1;
    }
  }
  if (threadIdx.x == 0) a.plen[q.row] = q.c;
}

// y = 0: the requests' tables and counts, a workgroup each.  y > 0: their
// partly filled pages, one array and layer.  Neither needs what the other
// writes: a copy reads the parent's row and length, which no request changes,
// and the plan.
__global__ __launch_bounds__(256) void fork_assign_kernel(ForkArgs a,
                                                          CopyArgs c) {
  if (blockIdx.y > 0) {
    copy_pages(c, (blockIdx.y - 1) % c.n_arrays, (blockIdx.y - 1) / c.n_arrays,
               a.n, blockIdx.x, gridDim.x,
               [&](int m, int64_t& from, int64_t& to) {
                 if (a.status[m]) return false;
                 const Request q = read_request(a, m);
                 if (q.extend || q.p < 0 || q.c % kPage == 0) return false;
                 from = a.bt[static_cast<int64_t>(q.p) * a.max_pages + q.full];
                 to = a.free_ids[a.first[m]];
                 return true;
               });
    return;
  }
  for (int i = blockIdx.x; i < a.n; i += gridDim.x) assign(a, i);
}

// ---------------------------------------------------------------------------
// compact
// ---------------------------------------------------------------------------

struct CompactArgs {
  const int32_t* bt;
  const int32_t* ref;
  int32_t* new_bt;
  int32_t* new_ref;
  int32_t* n_used;
  int32_t* moves;         // (from, to) pairs
  int32_t* count;         // how many
  int32_t* name;          // [num_pages] a page's new number
  int64_t entries;
  int num_pages;
};

// The pages in use, the moves and the new numbers and counts, one workgroup;
// eight consecutive pages a thread and step (8192 pages: one step a pass).
__global__ __launch_bounds__(kThreads) void compact_plan_kernel(CompactArgs a) {
  __shared__ int lds[kWaves];
  constexpr int N = 8, kStep = N * kThreads;
  const int64_t P = a.num_pages, t0 = N * static_cast<int64_t>(threadIdx.x);
  int total;
  int used = 0;
  for (int64_t base = t0; base < P; base += kStep)
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int64_t id = base + k;
      used += id < P && a.ref[id] > 0 ? 1 : 0;
    }
  group_scan(used, lds, total);
  const int n = total;
  // free pages below n, pages in use from n on: as many of each.  A page's
  // own number meanwhile.
  int frees = 0, far = 0;
  for (int64_t step = 0; step < P; step += kStep) {
    int f = 0, g = 0;
    uint32_t is = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int64_t id = step + t0 + k;
      if (id >= P) continue;
      const bool in_use = a.ref[id] > 0;
      a.name[id] = static_cast<int>(id);
      if (in_use == (id >= n)) {
        is |= 1u << k;
        if (id < n) ++f;
        else ++g;
      }
    }
    int at_f = frees + group_scan(f, lds, total);
    frees += total;
    int at_g = far + group_scan(g, lds, total);
    far += total;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int64_t id = step + t0 + k;
      if (!(is >> k & 1)) continue;
      if (id < n) a.moves[2 * at_f++ + 1] = static_cast<int>(id);
      else a.moves[2 * at_g++] = static_cast<int>(id);
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    *a.count = far;
    *a.n_used = n;
  }
  for (int m = threadIdx.x; m < far; m += kThreads) {
    const int from = a.moves[2 * m], to = a.moves[2 * m + 1];
    a.name[from] = to;
    // (to is free and below n, from at or above it: no other thread reads or
    // writes their counts)
    a.new_ref[to] = a.ref[from];
  }
  __syncthreads();
  for (int64_t id = threadIdx.x; id < P; id += kThreads) {
    if (id >= n) a.new_ref[id] = 0;
    else if (a.new_ref != a.ref && a.ref[id] > 0) a.new_ref[id] = a.ref[id];
  }
}

// y = 0: the table's new numbers.  y > 0: the moves, shared by the workgroups
// of one array and layer.
__global__ __launch_bounds__(256) void compact_apply_kernel(CompactArgs a,
                                                            CopyArgs c) {
  if (blockIdx.y > 0) {
    copy_pages(c, (blockIdx.y - 1) % c.n_arrays, (blockIdx.y - 1) / c.n_arrays,
               *a.count, blockIdx.x, gridDim.x,
               [&](int m, int64_t& from, int64_t& to) {
                 from = a.moves[2 * m];
                 to = a.moves[2 * m + 1];
                 return true;
               });
    return;
  }
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
       i < a.entries; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int id = a.bt[i];
    a.new_bt[i] = id >= 0 && id < a.num_pages ? a.name[id] : -1;
  }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

bool aligned(const void* p, size_t n) {
  return reinterpret_cast<uintptr_t>(p) % n == 0;
}

int check_arrays(const wedlm_page_array* arrays, int32_t n_arrays,
                 int32_t n_layers, CopyArgs* c) {
  if (n_arrays < 0 || n_arrays > WEDLM_MAX_ARRAYS || n_layers < 1 ||
      n_layers > 8191)
    return WEDLM_E_SHAPE;
  if (n_arrays > 0 && !arrays) return WEDLM_E_ARG;
  c->n_arrays = n_arrays;
  for (int i = 0; i < n_arrays; ++i) {
    if (!arrays[i].base || arrays[i].page_bytes < 1) return WEDLM_E_ARG;
    c->array[i].base = static_cast<char*>(arrays[i].base);
    c->array[i].bytes = arrays[i].page_bytes;
    const uintptr_t low = reinterpret_cast<uintptr_t>(arrays[i].base) |
                          static_cast<uintptr_t>(arrays[i].page_bytes);
    c->array[i].shift = low % 16 == 0 ? 4 : low % 4 == 0 ? 2 : 0;
  }
  return WEDLM_OK;
}

// Workgroups that share `most` copies of one array and layer: about eight a CU
// on the pages of more than a few words, 16 KB under way in each.  (Counted over
// all arrays, exponents too, half as many were left for the wide ones: 232 us
// in place of 211 for the compaction of 8192 pages.)
unsigned sharers(int64_t most, const CopyArgs& c, int n_layers) {
  int64_t wide = 0;
  for (int i = 0; i < c.n_arrays; ++i)
    wide += (c.array[i].bytes >> c.array[i].shift) > 32 ? n_layers : 0;
  const int64_t x = wide > 0 ? (2048 + wide - 1) / wide : 256;
  return static_cast<unsigned>(x < most ? x : most);
}

}  // namespace

extern "C" int wedlm_cache_free(const int32_t* rows, int32_t n,
                                int32_t* block_table, int32_t B,
                                int32_t max_pages, int32_t* ref,
                                int64_t num_pages, int32_t* prefix_len,
                                void* stream) {
  if (!rows || !block_table || !ref) return WEDLM_E_ARG;
  if (n < 1 || n > 65535 || B < 1 || max_pages < 1 || num_pages < 1 ||
      num_pages >= (1ll << 31))
    return WEDLM_E_SHAPE;
  FreeArgs a{rows, block_table, ref, prefix_len, static_cast<int>(num_pages),
             B, max_pages};
  const unsigned y = static_cast<unsigned>((max_pages + 255ll) / 256);
  hipLaunchKernelGGL(cache_free_kernel, dim3(n, y < 64 ? y : 64), dim3(256), 0,
                     static_cast<hipStream_t>(stream), a);
  WEDLM_LAUNCH_CHECK();
  return WEDLM_OK;
}

static size_t fork_bytes(int64_t n, int64_t max_pages, int64_t num_pages) {
  // first n, and the free pages: at most all, at most n rows' worth
  const int64_t ids = num_pages / max_pages < n ? num_pages : n * max_pages;
  return static_cast<size_t>(n + ids) * sizeof(int32_t);
}

extern "C" size_t wedlm_cache_fork_workspace_size(int32_t n, int32_t max_pages,
                                                  int64_t num_pages) {
  if (n < 1 || n > 65535 || max_pages < 1 || num_pages < 1 ||
      num_pages >= (1ll << 31))
    return 0;
  return fork_bytes(n, max_pages, num_pages);
}

extern "C" int wedlm_cache_fork(
    const int32_t* parent, const int32_t* child, const int32_t* reserve,
    int32_t n, int32_t* prefix_len, int32_t* block_table, int32_t B,
    int32_t max_pages, int32_t* ref, int64_t num_pages,
    const wedlm_page_array* arrays, int32_t n_arrays, int32_t n_layers,
    int32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
  if (!parent || !child || !reserve || !prefix_len || !block_table || !ref ||
      !status)
    return WEDLM_E_ARG;
  if (n < 1 || n > 65535 || B < 1 || max_pages < 1 || num_pages < 1 ||
      num_pages >= (1ll << 31))
    return WEDLM_E_SHAPE;
  CopyArgs c{};
  int e = check_arrays(arrays, n_arrays, n_layers, &c);
  if (e != WEDLM_OK) return e;
  const size_t need = fork_bytes(n, max_pages, num_pages);
  if (!workspace || workspace_bytes < need) return WEDLM_E_WORKSPACE;
  if (!aligned(workspace, 8)) return WEDLM_E_ARG;
  ForkArgs a{};
  a.parent = parent; a.child = child; a.reserve = reserve;
  a.plen = prefix_len; a.bt = block_table; a.ref = ref; a.status = status;
  a.first = static_cast<int32_t*>(workspace);
  a.free_ids = a.first + n;
  a.n = n; a.B = B; a.max_pages = max_pages;
  a.num_pages = static_cast<int>(num_pages);
  hipStream_t st = static_cast<hipStream_t>(stream);
  c.num_pages = num_pages;
  if (n > kWaves) {
    hipLaunchKernelGGL(fork_check_kernel, dim3((n + 3) / 4), dim3(256), 0, st,
                       a);
    WEDLM_LAUNCH_CHECK();
  }
  hipLaunchKernelGGL(fork_plan_kernel, dim3(1), dim3(kThreads), 0, st, a);
  WEDLM_LAUNCH_CHECK();
  const int64_t copies = static_cast<int64_t>(n_arrays) * n_layers;
  hipLaunchKernelGGL(fork_assign_kernel,
                     dim3(sharers(n, c, n_layers),
                          static_cast<unsigned>(copies + 1)),
                     dim3(256), 0, st, a, c);
  WEDLM_LAUNCH_CHECK();
  return WEDLM_OK;
}

extern "C" size_t wedlm_cache_compact_workspace_size(int64_t num_pages) {
  if (num_pages < 1 || num_pages >= (1ll << 31)) return 0;
  // moves: at most half the pages; the count; the pages' new numbers
  return static_cast<size_t>(num_pages / 2 * 2 + 2 + num_pages) *
         sizeof(int32_t);
}

extern "C" int wedlm_cache_compact(
    const int32_t* block_table, int32_t B, int32_t max_pages,
    const int32_t* ref, int64_t num_pages, const wedlm_page_array* arrays,
    int32_t n_arrays, int32_t n_layers, int32_t* new_table, int32_t* new_ref,
    int32_t* n_used, void* workspace, size_t workspace_bytes, void* stream) {
  if (!block_table || !ref || !new_table || !new_ref || !n_used)
    return WEDLM_E_ARG;
  if (B < 1 || max_pages < 1 || num_pages < 1 || num_pages >= (1ll << 31))
    return WEDLM_E_SHAPE;
  const int64_t entries = static_cast<int64_t>(B) * max_pages;
  if (entries >= (1ll << 31)) return WEDLM_E_SHAPE;   // one launch
  CopyArgs c{};
  const int e = check_arrays(arrays, n_arrays, n_layers, &c);
  if (e != WEDLM_OK) return e;
  if (!workspace ||
      workspace_bytes < wedlm_cache_compact_workspace_size(num_pages))
    return WEDLM_E_WORKSPACE;
  if (!aligned(workspace, 8)) return WEDLM_E_ARG;
  CompactArgs a{};
  a.bt = block_table; a.ref = ref; a.new_bt = new_table; a.new_ref = new_ref;
  a.n_used = n_used; a.entries = entries;
  a.num_pages = static_cast<int>(num_pages);
  a.moves = static_cast<int32_t*>(workspace);
  a.count = a.moves + num_pages / 2 * 2;
  a.name = a.count + 2;
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(kThreads), 0, st, a);
  WEDLM_LAUNCH_CHECK();
  c.num_pages = num_pages;
  // (the copies of one page need none, but the table does)
  const int64_t copies =
      num_pages > 1 ? static_cast<int64_t>(n_arrays) * n_layers : 0;
  hipLaunchKernelGGL(compact_apply_kernel,
                     dim3(sharers(1 << 20, c, n_layers),
                          static_cast<unsigned>(copies + 1)),
                     dim3(256), 0, st, a, c);
  WEDLM_LAUNCH_CHECK();
  return WEDLM_OK;
}
