/*
 * wedlm_train.h -- C ABI of the training-time operators of WeDLM (arXiv
 * 2512.22737, Sec. 4.2 "Dual-Stream Masking") on MI355X (gfx950): attention
 * over a clean memory stream and a block-wise reordered prediction stream,
 * forward and backward, the backward passes of the decoder's norms
 * (wedlm_model.h), and the loss of the masked tokens with the gradient of its
 * logits (Eq. 7, Eq. 10).
 *
 * Conventions of wedlm.h hold (device pointers owned by the caller, bf16 as
 * uint16_t bits, nothing allocated or synchronised, enqueued on `stream`,
 * WEDLM_E_* codes returned before anything is enqueued).
 */
#ifndef WEDLM_TRAIN_H
#define WEDLM_TRAIN_H

#include "wedlm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of workspace wedlm_dual_stream_attn needs (0: unsupported shape). */
size_t wedlm_dual_stream_attn_workspace_size(int32_t n_seq, int32_t L,
                                             int32_t block, int32_t Hq,
                                             int32_t Hkv, int32_t D);

/*
 * wedlm_dual_stream_attn -- attention of Eq. (7)'s input under the block
 * attention pattern of Sec. 4.2, for n_seq sequences of L tokens.
 *
 * Physical rows of one sequence (2L): the memory stream, logical positions
 * 0..L-1 in order; then the prediction stream in L/block blocks of `block`
 * rows, each reordered as in Sec. 4.1 (the block's observed positions
 * first, then its masked ones, each group ascending).  Both streams carry
 * the logical positions 0..L-1 (Eq. 8), so q and k come rotated at the
 * logical position of their row.
 *   memory row at position p      attends to memory rows 0..p;
 *   prediction row of block k     attends to memory positions < k*block and
 *                                 to the rows of its own block up to itself.
 * In:
 *   q [n_seq, 2L, Hq, D], k, v [n_seq, 2L, Hkv, D] bf16 (rows as above),
 *   softmax_scale (usually 1/sqrt(D)); query head h reads kv head
 *   h / (Hq/Hkv).
 * Out:
 *   out [n_seq, 2L, Hq, D] bf16; lse [n_seq, 2L, Hq] fp32 (natural log of
 *   each row's softmax normaliser), or NULL.
 * Limits: block <= 64, L a multiple of block and of 16, D 64 or 128,
 * 2 * n_seq * L / block <= 65535.
 * workspace: wedlm_dual_stream_attn_workspace_size() bytes (the memory
 * stream's keys and values laid out as pages, the block tables, the
 * attention's split partials); its contents on entry do not matter.
 */
int wedlm_dual_stream_attn(const uint16_t* q, const uint16_t* k,
                           const uint16_t* v, int32_t n_seq, int32_t L,
                           int32_t block, int32_t Hq, int32_t Hkv, int32_t D,
                           float softmax_scale, uint16_t* out, float* lse,
                           void* workspace, size_t workspace_bytes,
                           void* stream);

/* Bytes of workspace wedlm_dual_stream_attn_backward needs (0: unsupported
 * shape). */
size_t wedlm_dual_stream_attn_backward_workspace_size(int32_t n_seq, int32_t L,
                                                      int32_t block,
                                                      int32_t Hq, int32_t Hkv,
                                                      int32_t D);

/*
 * wedlm_dual_stream_attn_backward -- gradients of wedlm_dual_stream_attn:
 * from dout, the gradient of its out, those of q, k and v.  The
 * probabilities are computed again from q, k and lse.
 * In:
 *   q, k, v, softmax_scale and the sizes as in the forward call; out and lse
 *   as it wrote them; dout [n_seq, 2L, Hq, D] bf16.  Values must be finite.
 * Out:
 *   dq [n_seq, 2L, Hq, D], dk, dv [n_seq, 2L, Hkv, D] bf16 (overwritten; the
 *   gradients of a kv head are summed over its query heads).  They must not
 *   overlap the inputs or each other.
 * Products take bf16 operands (the probabilities and the scores' gradients
 * are rounded to it) with fp32 sums, in an order that the sizes fix: the
 * result does not depend on the run.
 * Limits: those of the forward, Hq * D < 2^25 and
 * ceil(L / 256) * (ceil(L / 32) + 24) * Hq/Hkv < 2^31.  The last is the work
 * of one kv head; somewhat beyond it shapes are refused (workspace size 0,
 * WEDLM_E_SHAPE).  bf16 arrays and the workspace on 16-byte boundaries
 * (WEDLM_E_ARG).
 * workspace: wedlm_dual_stream_attn_backward_workspace_size() bytes (each
 * row's normaliser and sum of P dP; fp32 sums of keys whose work is split over
 * workgroups); its contents on entry do not matter.  Two calls that overlap in
 * time must not share a workspace.
 */
int wedlm_dual_stream_attn_backward(
    const uint16_t* q, const uint16_t* k, const uint16_t* v,
    const uint16_t* out, const float* lse, const uint16_t* dout, int32_t n_seq,
    int32_t L, int32_t block, int32_t Hq, int32_t Hkv, int32_t D,
    float softmax_scale, uint16_t* dq, uint16_t* dk, uint16_t* dv,
    void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of workspace wedlm_rmsnorm_backward needs for dgain (0: unsupported
 * shape). */
size_t wedlm_rmsnorm_backward_workspace_size(int32_t M, int32_t Hd);

/*
 * wedlm_rmsnorm_backward -- gradients of wedlm_rmsnorm: from dy, the gradient
 * of its y, those of x and of the gain.  With r = 1 / sqrt(mean(x^2) + eps)
 * and u = dy gain:
 *   dx = dres + r (u - x r mean(u x r)),  dgain = sum over rows of dy x r
 * in fp32.
 * In:
 *   x [M, Hd] fp32, gain [Hd] bf16, eps as in the forward call; dy [M, Hd]
 *   bf16; dres [M, Hd] fp32 or NULL (none): the residual stream's gradient
 *   past the norm.
 * Out:
 *   dx [M, Hd] fp32 (may be dres itself: the gradient is then added in
 *   place), dgain [Hd] fp32 or NULL (a frozen gain); both overwritten.
 *   Otherwise they must not overlap the inputs or each other.
 * M >= 1, Hd a multiple of 4 up to 2^20; x, dres, dx and the workspace on
 * 16-byte boundaries, gain and dy on 8-byte ones (WEDLM_E_ARG).
 * workspace: wedlm_rmsnorm_backward_workspace_size() bytes (partial sums of
 * dgain; none needed without it); its contents on entry do not matter.  The
 * sums' order is fixed by the sizes.  Two calls that overlap in time must not
 * share a workspace.
 */
int wedlm_rmsnorm_backward(const float* x, const uint16_t* gain,
                           const uint16_t* dy, const float* dres, int32_t M,
                           int32_t Hd, float eps, float* dx, float* dgain,
                           void* workspace, size_t workspace_bytes,
                           void* stream);

/* Bytes of workspace wedlm_qk_norm_rope_backward needs for the gains'
 * gradients (0: unsupported shape). */
size_t wedlm_qk_norm_rope_backward_workspace_size(int32_t M, int32_t Hq,
                                                  int32_t Hkv, int32_t D);

/*
 * wedlm_qk_norm_rope_backward -- gradients of wedlm_qk_norm_rope: those of
 * its q|k|v rows and gains from dq, dk and dv, the gradients of its outputs.
 * Each head's gradient is rotated back (angles in fp64, their cosines and
 * sines in fp32), then taken through the head's RMSNorm in fp32; dv is
 * copied.
 * In:
 *   qkv [M, (Hq + 2 Hkv) D], q_gain, k_gain [D], pos_ids [M], rope_theta and
 *   eps as in the forward call; dq [M, Hq, D], dk, dv [M, Hkv, D] bf16.
 * Out:
 *   dqkv [M, (Hq + 2 Hkv) D] bf16; dq_gain, dk_gain [D] fp32, each NULL if
 *   not wanted; all overwritten, no overlap with the inputs or each other.
 * M, Hq, Hkv >= 1, D 64 or 128; bf16 arrays on 16-byte boundaries
 * (WEDLM_E_ARG).
 * workspace: wedlm_qk_norm_rope_backward_workspace_size() bytes on a 4-byte
 * boundary (WEDLM_E_ARG; partial sums of the gains' gradients, none needed
 * without them); its contents on entry do not matter.  The sums' order is
 * fixed by the sizes.  Two calls that overlap in time must not share a
 * workspace.
 */
int wedlm_qk_norm_rope_backward(
    const uint16_t* qkv, const uint16_t* q_gain, const uint16_t* k_gain,
    const int32_t* pos_ids, const uint16_t* dq, const uint16_t* dk,
    const uint16_t* dv, int32_t M, int32_t Hq, int32_t Hkv, int32_t D,
    double rope_theta, float eps, uint16_t* dqkv, float* dq_gain,
    float* dk_gain, void* workspace, size_t workspace_bytes, void* stream);

/* types of wedlm_token_loss's logits */
#define WEDLM_LOGITS_F32 0
#define WEDLM_LOGITS_BF16 1

/* Bytes of workspace wedlm_token_loss needs (0: none, or an invalid shape). */
size_t wedlm_token_loss_workspace_size(int32_t R, int32_t V);

/*
 * wedlm_token_loss -- the negative log-likelihood of the masked tokens and
 * its gradient, row by row (Eq. 7; Eq. 10's 1/gamma_k of a row's block, and
 * whatever the mean divides by, come as the row's weight):
 *   loss[r]       = -weight[r] ln p[target[r]],  p = softmax(logits[r])
 *   dlogits[r][v] = weight[r] (p[v] - [v = target[r]])
 * A row whose target is outside 0 .. V-1 (a position without loss) or whose
 * weight is 0 has loss 0 and gradient 0, and its logits are not used.
 * In (R, V >= 1):
 *   logits [R, row_stride] of logits_type (WEDLM_LOGITS_*), row_stride >= V;
 *   values finite or -inf (a token that is ruled out: p = 0).  A row of
 *   nothing but -inf has loss weight * inf and gradient 0.
 *   target [R] int32; weight [R] fp32, finite, or NULL (all 1).
 * Out:
 *   loss [R] fp32; dlogits [R, row_stride] of logits_type, or NULL (the loss
 *   alone).  dlogits may be logits itself (in place); otherwise the arrays
 *   must not overlap.  Columns V .. row_stride-1 are left as they are.
 * Maxima, sums and the loss are fp32; the gradient is rounded once.  The
 * sums' order is fixed by the sizes and the arrays' alignment.  Rows on
 * 16-byte boundaries (logits and dlogits) are read and written faster.
 * workspace: wedlm_token_loss_workspace_size() bytes on an 8-byte boundary
 * (WEDLM_E_ARG; NULL when that is 0); its contents on entry do not matter.  Two
 * calls that overlap in time must not share a workspace.
 */
int wedlm_token_loss(const void* logits, int32_t logits_type,
                     int64_t row_stride, const int32_t* target,
                     const float* weight, int32_t R, int32_t V, float* loss,
                     void* dlogits, void* workspace, size_t workspace_bytes,
                     void* stream);

#ifdef __cplusplus
}
#endif

#endif /* WEDLM_TRAIN_H */
