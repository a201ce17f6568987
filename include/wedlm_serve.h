/*
 * wedlm_serve.h -- C ABI of the serving operators around the WeDLM decode
 * step (arXiv 2512.22737) on MI355X (gfx950): a paged cache in 8 bits with
 * the window attention over it and the commit that writes it, the pages'
 * sharing between sequences, and sampling in place of the greedy token.
 *
 * Conventions of wedlm.h hold (device pointers owned by the caller, bf16 as
 * uint16_t bits, nothing allocated or synchronised, enqueued on `stream`,
 * WEDLM_E_* codes returned before anything is enqueued).
 *
 * 8-bit cache
 * -----------
 *    k8    [num_pages, Hkv, 16, D]   e4m3 codes (OCP: no infinities, 0x7f and
 *    v8    [num_pages, Hkv, D, 16]   0xff are NaN), laid out like the bf16
 *                                    caches of wedlm.h
 *    k_exp, v_exp [num_pages, Hkv]   uint8, one scale per page and kv head:
 *                                    2^(exp - 127), 1 <= exp <= 254
 * A code stands for its e4m3 value times its page's scale.  Power-of-two
 * scales keep the codes' relative precision whatever a page's range, and a
 * page whose scale has to grow loses nothing but what falls below the
 * smallest normal code.
 */
#ifndef WEDLM_SERVE_H
#define WEDLM_SERVE_H

#include "wedlm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* further status bit (see wedlm.h) */
#define WEDLM_SEQ_BAD_ROW 8 /* a row of the block table that cannot be taken */

/*
 * wedlm_cache8_append -- write rows of keys and values into 8-bit caches.
 *
 * Row j (0 <= j < count[b]) of sequence b takes position start[b] + j of every
 * layer's cache.  For each page and kv head that gets rows, with `need` the
 * smallest exponent >= 1 whose 448 * 2^(need - 127) holds the largest finite
 * magnitude of the new rows (1 if they are all zero):
 *   exp'  = need, if the page's row 0 is among the new rows, else
 *           max(exp, need): the rows before the first new one stay
 *   new rows become e4m3(x * 2^(127 - exp')), rounded to nearest even;
 *   infinities and NaN become NaN
 *   where exp' > exp, the rows before the first new one are rounded again, to
 *   the new scale
 * Rows of a page behind the last new one keep their bytes.
 * In:
 *   k, v   [n_layers, B, T, Hkv, D] bf16
 *   start, count [B] int32; 0 <= count[b] <= T
 *   block_table [B, max_pages]; pages that get rows must belong to one
 *          sequence alone
 * In/out: k8, v8, k_exp, v_exp [n_layers, num_pages, ...].
 * Out: status [B] or NULL: WEDLM_SEQ_* bits are OR-ed in.  A negative start
 *   or a count outside 0 .. T (WEDLM_SEQ_BAD_LEN) writes nothing; rows whose
 *   position has no page (WEDLM_SEQ_CAPACITY) or a page outside the cache
 *   (WEDLM_SEQ_BAD_PAGE) are left out.
 * n_layers, B, T, Hkv >= 1, D 64 or 128, 1 <= num_pages < 2^31,
 * max_pages >= 1, and n_layers * B * Hkv * (ceil(T / 16) + 1) < 2^26
 * (WEDLM_E_SHAPE); k, v, k8 and v8 on 16-byte boundaries (WEDLM_E_ARG).
 */
int wedlm_cache8_append(const uint16_t* k, const uint16_t* v,
                        const int32_t* start, const int32_t* count,
                        int32_t n_layers, int32_t B, int32_t T, int32_t Hkv,
                        int32_t D, uint8_t* k8, uint8_t* v8, uint8_t* k_exp,
                        uint8_t* v_exp, int64_t num_pages,
                        const int32_t* block_table, int32_t max_pages,
                        int32_t* status, void* stream);

/* Bytes of workspace wedlm_window_attn_cache8 needs (0: none, or an
 * unsupported shape). */
size_t wedlm_window_attn_cache8_workspace_size(int32_t B, int32_t W,
                                               int32_t Hq, int32_t Hkv,
                                               int32_t D,
                                               int32_t max_prefix_len);

/*
 * wedlm_window_attn_cache8 -- wedlm_window_attn over an 8-bit cache.  The
 * window's own keys and values stay bf16.  Arguments, outputs, limits and
 * errors are those of wedlm_window_attn with k8, v8, k_exp, v_exp in the
 * place of k_cache, v_cache; D = 64 or 128, W = 1 (single tokens) to 64.
 * Codes behind a sequence's prefix are not used, whatever they hold.  Weights
 * enter their product with the values in bf16 (as over bf16 pages; half a step
 * of 2^-8, as much as the result's own rounding), sums are fp32, also where
 * splits are merged; their number goes by the batch's own prefix lengths, and
 * nothing depends on the run.  bf16 arrays, k8 and v8 on 16-byte
 * boundaries, the workspace on a 256-byte one (WEDLM_E_ARG); a max_prefix_len
 * whose splits pass one launch is refused (WEDLM_E_SHAPE).
 * What is not finite: a NaN code in a key of the prefix makes the outputs and
 * lse of its kv head's rows NaN, one in a value its element of their outputs; in
 * the window a query its own row, a key the rows that see it, a value its
 * element of all the window's rows (NaN, or infinite).  Weights are summed
 * before their maximum is known: with values of 2^44 and more a sum can become
 * infinite where the result is not.
 */
int wedlm_window_attn_cache8(
    const uint16_t* q_phys, const uint16_t* k_phys, const uint16_t* v_phys,
    const uint8_t* k8, const uint8_t* v8, const uint8_t* k_exp,
    const uint8_t* v_exp, int64_t num_pages, const int32_t* block_table,
    int32_t max_pages, const int32_t* prefix_len, int32_t B, int32_t W,
    int32_t Hq, int32_t Hkv, int32_t D, int32_t max_prefix_len,
    float softmax_scale, uint16_t* out, float* lse, int32_t* status,
    void* workspace, size_t workspace_bytes, void* stream);

/*
 * wedlm_commit_cache8 -- wedlm_commit_layers for 8-bit caches: the same
 * commit, selection and refill under `rule`, with the committed rows of every
 * layer appended as by wedlm_cache8_append.  k_win, v_win [n_layers, B, W,
 * Hkv, D]; k8, v8, k_exp, v_exp [n_layers, num_pages, ...]; other arguments,
 * outputs and errors as in wedlm_commit_layers, limits and alignment also as
 * in wedlm_cache8_append with T = W.
 */
int wedlm_commit_cache8(int32_t* win_tok, int32_t* win_start,
                        const int32_t* argmax, const float* entropy,
                        double tau, double lambda, const uint16_t* k_win,
                        const uint16_t* v_win, uint8_t* k8, uint8_t* v8,
                        uint8_t* k_exp, uint8_t* v_exp, int64_t num_pages,
                        const int32_t* block_table, int32_t max_pages,
                        int32_t B, int32_t W, int32_t Hkv, int32_t D,
                        int32_t n_layers, int32_t* n_commit,
                        int32_t* committed_tok, int32_t* committed_slot,
                        uint8_t* selected, int32_t* status, int32_t rule,
                        void* stream);

/*
 * Pages shared between sequences
 * ------------------------------
 * A pool of num_pages pages serves the rows of a block table.  ref
 * [num_pages] int32 counts the table's entries that hold each page: 0 = free.
 * Entries without a page are negative.  A pool's arrays are those that are
 * indexed by page: the bf16 caches of wedlm.h, or the four arrays of an 8-bit
 * cache.
 */
#define WEDLM_MAX_ARRAYS 8

/* One array of a pool: n_layers times num_pages pages of page_bytes bytes,
 * contiguous. */
typedef struct {
  void* base;
  int64_t page_bytes;
} wedlm_page_array;

/*
 * wedlm_cache_free -- sequences end: for each row rows[i] of the block table,
 * every entry that holds a page gives it back (ref - 1) and becomes -1, and
 * prefix_len of the row becomes 0.  Row numbers outside the table are passed
 * over; a row that is listed twice is freed once.  Entries outside the pool
 * become -1 and count for nothing; a count that is 0 already stays.
 *   rows [n] int32; block_table [B, max_pages], ref [num_pages],
 *   prefix_len [B] (or NULL): in/out
 * 1 <= n <= 65535; B, max_pages >= 1, 1 <= num_pages < 2^31 (WEDLM_E_SHAPE).
 */
int wedlm_cache_free(const int32_t* rows, int32_t n, int32_t* block_table,
                     int32_t B, int32_t max_pages, int32_t* ref,
                     int64_t num_pages, int32_t* prefix_len, void* stream);

/* Bytes of workspace wedlm_cache_fork needs (0: an unsupported shape). */
size_t wedlm_cache_fork_workspace_size(int32_t n, int32_t max_pages,
                                       int64_t num_pages);

/*
 * wedlm_cache_fork -- sequences start: request i gives the empty row child[i]
 * of the block table the prefix of row parent[i].  With c the parent's prefix
 * length and f = c / 16:
 *   entries 0 .. f-1 share the parent's pages (ref + 1);
 *   entries f .. ceil(max(c, reserve[i]) / 16) - 1 are free pages, ref = 1,
 *     the lowest first, the requests in order;
 *   if c is not a multiple of 16, page f of the parent is copied into the
 *     child's, in every array and layer;
 *   prefix_len of the child becomes c.
 * parent[i] = -1 starts an empty sequence (c = 0), parent[i] = child[i]
 * extends one: its entries below ceil(max(c, reserve[i]) / 16) that hold no
 * page get one.
 * status[i] is set to 0 or to why request i changed nothing:
 *   WEDLM_SEQ_BAD_ROW  a row outside the table; a child whose row holds
 *     pages, that another request has for its child, or that another request
 *     has for its parent
 *   WEDLM_SEQ_BAD_LEN  the parent's prefix_len is negative, or it or
 *     reserve[i] needs more than max_pages entries
 *   WEDLM_SEQ_BAD_PAGE a page of the parent's prefix is outside the pool
 *   WEDLM_SEQ_CAPACITY too few free pages are left for it; the requests after
 *     it that need free pages get this too
 * In:  parent, child, reserve [n]; arrays [n_arrays] (a host array, at most
 *   WEDLM_MAX_ARRAYS, read before the call returns)
 * In/out: block_table [B, max_pages], ref [num_pages], prefix_len [B], the
 *   arrays.   Out: status [n].
 * 1 <= n <= 65535; B, max_pages >= 1, 1 <= num_pages < 2^31, 1 <= n_layers <=
 * 8191, n_arrays >= 0 (WEDLM_E_SHAPE), page_bytes >= 1 (WEDLM_E_ARG).
 * workspace: wedlm_cache_fork_workspace_size() bytes on an 8-byte boundary
 * (WEDLM_E_ARG); its contents on entry do not matter.  Two calls that overlap
 * in time must not share a workspace or a pool.
 */
int wedlm_cache_fork(const int32_t* parent, const int32_t* child,
                     const int32_t* reserve, int32_t n, int32_t* prefix_len,
                     int32_t* block_table, int32_t B, int32_t max_pages,
                     int32_t* ref, int64_t num_pages,
                     const wedlm_page_array* arrays, int32_t n_arrays,
                     int32_t n_layers, int32_t* status, void* workspace,
                     size_t workspace_bytes, void* stream);

/* Bytes of workspace wedlm_cache_compact needs (0: an unsupported shape). */
size_t wedlm_cache_compact_workspace_size(int64_t num_pages);

/*
 * wedlm_cache_compact -- the pages in use move to the pool's lowest numbers:
 * with n_used of them, the i-th page in use (in rising order) with a number
 * >= n_used moves into the i-th free page below n_used, in every array and
 * layer; the others stay where they are.  The least number of pages moves,
 * none into a page that is in use.
 * In:  block_table [B, max_pages], ref [num_pages]
 * In/out: the arrays (as in wedlm_cache_fork).  Pages >= n_used keep their
 *   bytes.
 * Out: new_table [B, max_pages] with the pages' new numbers (entries outside
 *   the pool become -1) and new_ref [num_pages], either of which may be its
 *   input itself; n_used [1] int32.  They must not overlap anything else.
 * Limits as in wedlm_cache_fork, B * max_pages < 2^31.
 * workspace: wedlm_cache_compact_workspace_size() bytes on an 8-byte boundary
 * (WEDLM_E_ARG); its contents on entry do not matter.  Two calls that overlap
 * in time must not share a workspace or a pool.
 */
int wedlm_cache_compact(const int32_t* block_table, int32_t B,
                        int32_t max_pages, const int32_t* ref,
                        int64_t num_pages, const wedlm_page_array* arrays,
                        int32_t n_arrays, int32_t n_layers, int32_t* new_table,
                        int32_t* new_ref, int32_t* n_used, void* workspace,
                        size_t workspace_bytes, void* stream);

/* types of wedlm_sample's logits */
#define WEDLM_SAMPLE_F32 0
#define WEDLM_SAMPLE_BF16 1

/*
 * wedlm_sample -- one token per masked row from given random numbers, in the
 * place of wedlm_score's greedy token (a decoder without windows calls it
 * with W = 1).  For row i >= n_obs[b] of sequence b, with x its logits and
 * the sequence's settings:
 *   1. the tokens in falling order of x, equal ones by rising id;
 *   2. the first top_k of them;
 *   3. weights w = exp((x - max x) / temperature);
 *   4. of those, the shortest leading run whose weights sum up to at least
 *      top_p times the sum of all that step 2 left (one token at least);
 *   5. of those, the tokens with w >= min_p;
 *   token = the lowest id t for which the weights of the remaining ids <= t
 *           sum up to more than u times their total
 *   logp  = ln(w_t / total)
 * Weights are fixed-point numbers with f = min(46, 62 - ceil(log2 V)) bits
 * after the point, from fp64; their sums are exact, so the result does not
 * depend on an order of summation.  The total is at least 1 and each weight is
 * off by at most half a unit, logp therefore by at most V 2^-(f+1) beside its
 * rounding to fp32: one that is nearer to 0 is not resolved.  A weight below
 * 2^-(f+1) is 0, and its token is not drawn.
 * In:
 *   logits [B, W, row_stride] of logits_type (WEDLM_SAMPLE_*), row_stride >=
 *     V; NaN counts as -inf (a token that is ruled out), +inf as the largest
 *     fp32.  Of a row of nothing but -inf token 0 is taken, with logp 0.
 *   u [B, W] fp32 in [0, 1) (others are taken as the nearest that is)
 *   n_obs [B] int32, or NULL (all rows)
 *   temperature [B] fp32, or NULL (1): 0, negative or NaN: greedy, the first
 *     of the largest logits, logp = 0
 *   top_k [B] int32, or NULL: <= 0 or >= V: no limit
 *   top_p [B] fp32, or NULL: >= 1 or NaN: no limit
 *   min_p [B] fp32, or NULL: <= 0 or NaN: no limit; above 1 as 1
 * Out: token [B, W] int32, logp [B, W] fp32 or NULL; entries of observed rows
 *   are left untouched.
 * B, W >= 1, B * W < 2^22, 1 <= V <= 2^22 (WEDLM_E_SHAPE).  Rows may start
 * anywhere (row_stride of any size); no workspace is needed.
 */
int wedlm_sample(const void* logits, int32_t logits_type, int64_t row_stride,
                 const float* u, const int32_t* n_obs,
                 const float* temperature, const int32_t* top_k,
                 const float* top_p, const float* min_p, int32_t B, int32_t W,
                 int32_t V, int32_t* token, float* logp, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* WEDLM_SERVE_H */
