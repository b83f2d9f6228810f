/*
 * fp8train, operators on tokens and rows -- the two ends of a language model
 * and its joints: token embeddings with their gradient, the norm of a residual
 * sum with its gradient, and the log probabilities of given tokens with theirs.
 * Same library, formats (FP8 = 1-5-2 codes in uint8_t, FP16 = 1-6-9 codes in
 * uint16_t), status codes and conventions as fp8train.h and fp8train_lm.h: all
 * pointers are device pointers owned by the caller, the library never
 * allocates or synchronizes, work is enqueued on `stream`, arguments are
 * validated before anything is enqueued, sizes and strides count elements,
 * matrices are row-major with a row stride _ld and may start at any address of
 * their elements.
 *
 * Results are functions of the arguments alone on a given device (no atomics
 * whose order could change them); a workspace, where it is optional, chooses
 * the order of sums.  Nothing in a workspace is kept from one call for the
 * next; calls that may overlap need workspaces of their own.  Sums and
 * statistics are FP32 or better; every result is rounded once, from FP32, to
 * its storage format: Q below (FP8: nearest even, saturating at 57344; FP16:
 * nearest even; F32: as is).
 */
#ifndef FP8TRAIN_TOKENS_H
#define FP8TRAIN_TOKENS_H

#include "fp8train_lm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest vocabulary of embed_bwd, token_logprobs and token_logprobs_bwd. */
#define FP8T_MAX_VOCAB (1 << 24)
/* Widest row of rms_norm_fwd and rms_norm_bwd. */
#define FP8T_MAX_NORM_W (1 << 20)
/* Most alternatives token_logprobs gives. */
#define FP8T_MAX_TOP 128

/*
 * embed_fwd -- rows of a table by tokens:
 *   y[t, :] = Q(RN32(value(table[tokens[t], :]) * scale))
 * A token outside [0, V) (padding) has a row of +0.
 * tokens: T int64; table: V x W in table_format; y: T x W in y_format; both
 * formats F32, FP16 or FP8.  y must not overlap the table.
 * Errors: FP8T_EINVAL (negative size, T, V or W above 2^31 - 4097, unknown
 * format, a stride below W, NULL pointer for non-empty data); FP8T_EHIP.
 */
int embed_fwd(const int64_t* tokens, int64_t T, const void* table, int table_format,
              int64_t table_ld, int64_t V, int64_t W, float scale, void* y, int y_format,
              int64_t y_ld, hipStream_t stream);

/*
 * embed_bwd -- the table's gradient from the error e of y:
 *   g[v, :] = Q(RN32(scale * sum of value(e[t, :]) over t with tokens[t] = v))
 * for every v in [0, V): a row that no token names is +0.  Errors of tokens
 * outside [0, V) are not read.  The tokens are sorted on the device, and a
 * row's sum is taken in the order of t, in pieces that the sorted order alone
 * decides, in doubles.
 * e: T x W in e_format; g: V x W in g_format; both F32, FP16 or FP8; g must not
 * overlap e.
 * workspace: at least embed_bwd_workspace_size bytes, 16-byte aligned.
 * Errors: FP8T_EINVAL (negative size, T or W above 2^31 - 4097, V above
 * FP8T_MAX_VOCAB, unknown format, a stride below W, NULL pointer for
 * non-empty data, a workspace that is not 16-byte aligned); FP8T_EWORKSPACE
 * (workspace_bytes below the query); FP8T_EHIP.
 */
int embed_bwd(const int64_t* tokens, int64_t T, const void* e, int e_format, int64_t e_ld,
              int64_t V, int64_t W, float scale, void* g, int g_format, int64_t g_ld,
              void* workspace, size_t workspace_bytes, hipStream_t stream);

/* embed_bwd_workspace_size -- bytes of workspace embed_bwd needs (0 for
 * invalid or empty sizes). */
size_t embed_bwd_workspace_size(int64_t T, int64_t V, int64_t W);

/*
 * rms_norm_fwd -- a residual sum and its root-mean-square norm.  For row t:
 *   x'   = value(x[t, :]), or RN32(value(x[t, :]) / x_row_scale[t])
 *   u    = value(Q(RN32(x' + value(r[t, :])))), Q to s_format, written to h
 *   rstd = RN32(1 / sqrt(mean(u^2) + eps)), formed in doubles
 *   n    = RN32(RN32(u rstd) value(w))            (w NULL: 1)
 *   y    = Q(RN32(n * c))
 * With neither r nor h, u = x' (not rounded); with h alone, u = value(Q(x')).
 * The norm is of the sum as it is stored, which is what rms_norm_bwd reads.
 * c = y_scale; with y_row_scale the row's own scale: c = RN32(y_scale / max |n|),
 * at most 2^126 (1 where that maximum is 0, infinite or NaN), written to
 * y_row_scale[t], so that the row's largest result is y_scale.  A product with
 * y in place of n c, given to the next norm as x with that y_row_scale as its
 * x_row_scale, is divided by it again.
 * Inf and NaN follow IEEE arithmetic within their row (a row with an Inf has
 * rstd 0) and leave the other rows alone.
 *
 * x: T x W in x_format (F32 or FP16); r, h: T x W in s_format (F32 or FP16); w:
 * W contiguous in w_format (F32 or FP16); y: T x W in y_format (F32, FP16 or
 * FP8); x_row_scale, y_row_scale, rstd: T floats.  r, w, x_row_scale and the
 * results h, y, y_row_scale, rstd are optional (NULL), one of h, y and rstd is
 * not.  h may be r or x itself (same format and stride); other results must
 * not overlap an operand.
 * Errors: FP8T_EINVAL (negative size, T above 2^31 - 4097, W above
 * FP8T_MAX_NORM_W, unknown format, a stride below W, eps not from 2^-100 to
 * 2^100, NULL pointer for non-empty data, no result, y_row_scale without y or
 * with a y_scale that is not positive and finite); FP8T_EHIP.
 */
int rms_norm_fwd(const void* x, int x_format, int64_t x_ld, const float* x_row_scale,
                 const void* r, int64_t r_ld, const void* w, int w_format, int64_t T, int64_t W,
                 float eps, void* h, int s_format, int64_t h_ld, void* y, int y_format,
                 int64_t y_ld, float y_scale, float* y_row_scale, float* rstd,
                 hipStream_t stream);

/*
 * rms_norm_bwd -- gradients of rms_norm_fwd.  With h the sum that was normed
 * (x where there was none) and its rstd, dy the error of n, dr the error that
 * reaches h past the norm (NULL: 0), m = mean over the row of value(h) rstd
 * value(w) value(dy):
 *   d  = value(dr) + rstd (value(w) value(dy) - value(h) rstd m)
 *   dx = Q(d) in d_format,  dx8 = Q(RN32(d * dx8_scale)) in FP8
 *   dw = Q(sum over t of value(dy) value(h) rstd) in dw_format
 * The products are FP32, m's sum and dw's are doubles (parts of dw's, the rows
 * of a workgroup, are stored as floats).  d is the error of x' and of r alike.
 * The scales of y are constants: dy is the error of n c times c.
 * h: h_format F32 or FP16; w: F32, FP16 or NULL; rstd: T floats; dy: F32, FP16
 * or FP8; dr, dx: d_format F32 or FP16, dx may be dr itself (same stride); dw:
 * W contiguous, F32 or FP16 (all +0 with T = 0).  dx, dx8 and dw are optional
 * (NULL), one is not; but for dx in dr's place they must not overlap an operand.
 * workspace: with dw at least rms_norm_bwd_workspace_size bytes, 16-byte
 * aligned (partial sums of dw); without dw none is used.
 * Errors: FP8T_EINVAL (as rms_norm_fwd, and for a workspace that is not 16-byte
 * aligned); FP8T_EWORKSPACE (dw with workspace_bytes below the query);
 * FP8T_EHIP.
 */
int rms_norm_bwd(const void* h, int h_format, int64_t h_ld, const void* w, int w_format,
                 const float* rstd, const void* dy, int dy_format, int64_t dy_ld, const void* dr,
                 int64_t dr_ld, int64_t T, int64_t W, void* dx, int d_format, int64_t dx_ld,
                 uint8_t* dx8, int64_t dx8_ld, float dx8_scale, void* dw, int dw_format,
                 void* workspace, size_t workspace_bytes, hipStream_t stream);

/* rms_norm_bwd_workspace_size -- bytes of workspace rms_norm_bwd needs for dw
 * on the current device (0 for invalid or empty sizes). */
size_t rms_norm_bwd_workspace_size(int64_t T, int64_t W);

/*
 * token_logprobs -- log probabilities of given tokens under softmax(z / tau),
 * the distribution's entropy and its likeliest tokens.  For row n with logits
 * z = value(z[n, .]), M = max z, d = (z - M) / tau, S = sum exp(d):
 *   logp[n, i]  = d[idx[n, i]] - ln S        (idx outside [0, V): +0)
 *   entropy[n]  = ln S - (sum d exp(d)) / S  (terms with exp(d) = 0 add 0)
 *   stats[n, 0] = M,  stats[n, 1] = ln S
 *   top_idx[n, j], top_logp[n, j]: the j-th largest logit's token and log
 *     probability, among equal logits the lowest token first (-0 equals +0, NaN
 *     is above +Inf); past the vocabulary's end -1 and -Inf.
 * Powers are taken of a logit's distance from the row's largest; below 2^-126
 * they are 0.  A row whose largest logit is +Inf or -Inf (every token masked),
 * or that holds a NaN, has NaN log probabilities, entropy and ln S, and M is
 * +Inf, -Inf or NaN; masked tokens (-Inf) of other rows have a log probability
 * of -Inf.
 * The top entries are what distill_loss takes of a teacher (top_idx as idx,
 * top_logp as t), the statistics what token_logprobs_bwd takes.
 *
 * z: N x V in z_format (F32 or FP16), V >= 1; idx: N x m contiguous int64; logp
 * N x m, entropy N, stats N x 2, top_idx (int64) and top_logp N x k, contiguous
 * floats but for top_idx.  Each result is optional (NULL), not all of them;
 * m = 0 with logp NULL; k from 0 to FP8T_MAX_TOP.
 * workspace: token_logprobs_workspace_size bytes for the fastest plan, or none
 * (workspace_bytes == 0, then a plan that needs none); it holds the partial
 * results of parts of rows that several workgroups share.
 * Errors: FP8T_EINVAL (negative size, N above 2^31 - 4097, V above
 * FP8T_MAX_VOCAB, V = 0 with N > 0, m > 4096, k > FP8T_MAX_TOP, tau not from
 * 2^-30 to 2^30, unknown format, a stride below V, NULL pointer for non-empty
 * data, no result, NULL workspace with workspace_bytes > 0, or one that is not
 * 16-byte aligned where it is used); FP8T_EWORKSPACE (0 < workspace_bytes < the query); FP8T_EHIP.
 */
int token_logprobs(const void* z, int z_format, int64_t z_ld, const int64_t* idx, int64_t m,
                   int64_t N, int64_t V, float tau, float* logp, float* entropy, float* stats,
                   int64_t k, int64_t* top_idx, float* top_logp, void* workspace,
                   size_t workspace_bytes, hipStream_t stream);

/* token_logprobs_workspace_size -- bytes of workspace token_logprobs' fastest
 * plan needs on the current device (0 if none, or for invalid sizes). */
size_t token_logprobs_workspace_size(int64_t N, int64_t V, int64_t k);

/*
 * token_logprobs_bwd -- the logits' gradient from those of logp and entropy.
 * With token_logprobs' stats, l = (z - M) / tau - ln S, p = exp(l), D the sum
 * of d_logp[n, i] over the used idx:
 *   g[n, v] = Q(grad_scale / tau (sum of d_logp[n, i] with idx[n, i] = v
 *               - p[v] (D + d_entropy[n] (l[v] + entropy[n]))))
 * (terms with p = 0 are 0).  Entries with idx outside [0, V) are unused, their
 * d_logp is not looked at; an entry that occurs twice counts twice.  A row whose
 * d_logp (of used entries) and d_entropy are all 0 has g +0, whatever z holds.
 * d_logp: N x m contiguous floats (NULL: all 0); d_entropy: N floats (NULL: all
 * 0) with entropy: N floats (NULL is fine without d_entropy); one of d_logp and
 * d_entropy is not NULL.  g: N x V in g_format (F32, FP16 or FP8), may be z
 * itself (same format and stride), otherwise they must not overlap.
 * Errors: FP8T_EINVAL (as token_logprobs; stats or g NULL, neither gradient,
 * d_entropy without entropy); FP8T_EHIP.
 */
int token_logprobs_bwd(const void* z, int z_format, int64_t z_ld, const int64_t* idx, int64_t m,
                       const float* stats, const float* entropy, const float* d_logp,
                       const float* d_entropy, int64_t N, int64_t V, float tau, float grad_scale,
                       void* g, int g_format, int64_t g_ld, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif
