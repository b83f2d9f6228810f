/*
 * fp8train, language-model operators -- what a transformer trained with the
 * GEMMs of fp8train.h needs between them: rotary positions, attention over
 * packed sequences (forward and backward) and a distillation loss with its
 * gradient.  Same library, formats (FP8 = 1-5-2 codes in uint8_t, FP16 =
 * 1-6-9 codes in uint16_t), status codes and conventions as fp8train.h: all
 * pointers are device pointers owned by the caller, the library never
 * allocates or synchronizes, work is enqueued on `stream`, arguments are
 * validated before anything is enqueued, sizes and strides count elements.
 *
 * Results are functions of the arguments alone on a given device (no atomics
 * whose order could change them); attention's size hints and workspace choose
 * the order of its sums, so a call with others may differ in the last bits.
 * Sums, softmax statistics and log-sum-exps are FP32; every result is rounded
 * once, from FP32, to its storage format.
 */
#ifndef FP8TRAIN_LM_H
#define FP8TRAIN_LM_H

#include "fp8train.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Storage formats (the first two are fp8_quantize's source formats). */
enum {
    FP8T_FMT_F32 = 0,
    FP8T_FMT_FP16 = 1,    /* 1-6-9 codes                                     */
    FP8T_FMT_FP8 = 2,     /* 1-5-2 codes                                     */
    FP8T_FMT_HALF = 3     /* IEEE binary16 (fp16_dequantize's results only)  */
};

/* Largest head dimension of the attention calls. */
#define FP8T_ATTN_MAX_D 128

/*
 * fp16_dequantize -- values of FP16 codes for programs outside the library:
 *   dst[i] = value(src[i]) * scale
 * (one IEEE single-precision product; 1 / loss scale removes a loss scale).
 * dst_format FP8T_FMT_F32: float, with scale 1 exact; FP8T_FMT_HALF: IEEE
 * binary16, the float rounded to nearest even (with scale 1 exact for
 * magnitudes from 2^-14 to 65472; larger ones become Inf).  n contiguous
 * elements; n == 0 is a no-op.
 * Errors: FP8T_EINVAL (n < 0, NULL pointer with n > 0, another dst_format);
 * FP8T_EHIP.
 */
int fp16_dequantize(const uint16_t* src, float scale, void* dst, int dst_format, int64_t n,
                    hipStream_t stream);

/*
 * rotary_embed -- rotary positions: pairs of a head's first R entries turned
 * by an angle that grows with the token's position.
 *
 * For token t, head h, pair j in [0, R/2), with x = value(x[t, h, .]),
 * a = positions[t] * freqs[j] (radians), c = mscale cos a, s = mscale sin a
 * (inverse: s = -mscale sin a):
 *   interleaved = 0: (i0, i1) = (j, j + R/2);  1: (i0, i1) = (2 j, 2 j + 1)
 *   r[i0] = x[i0] c - x[i1] s      r[i1] = x[i1] c + x[i0] s
 * and r[i] = x[i] for i in [R, D); y = Q(RN32(r * scale)) in y_format
 * (FP8: nearest even, saturating; FP16: nearest even; F32: as is).
 *
 * inverse = 1 is the gradient: with y = rotary_embed(x) and an error e of y,
 * the error of x is rotary_embed(e) with inverse = 1 and the same mscale.
 * The angle is reduced exactly enough that positions of any size keep float
 * accuracy (frequencies up to 2^16).  freqs: R/2 doubles on the device; scaling for long
 * contexts is in the table (and mscale).  positions: T int64, any sign.
 *
 * x: T x H x D in x_format with strides x_ts (tokens) and x_hs (heads), the D
 * entries contiguous; y likewise.  y may be x itself (same format and
 * strides), otherwise they must not overlap.  R even, 0 <= R <= D.
 * Errors: FP8T_EINVAL (negative size, R odd or > D, D > 65536, unknown format or flag,
 * negative input stride, an output stride that makes rows overlap, NULL
 * pointer for non-empty data); FP8T_EHIP.
 */
int rotary_embed(const void* x, int x_format, int64_t x_ts, int64_t x_hs, const int64_t* positions,
                 const double* freqs, int64_t T, int64_t H, int64_t D, int64_t R, int interleaved,
                 int inverse, float mscale, float scale, void* y, int y_format, int64_t y_ts,
                 int64_t y_hs, hipStream_t stream);

/*
 * attn_fwd_fp8 -- attention over packed sequences with FP8 operands.
 *
 * S sequences lie one after the other: queries of sequence s are tokens
 * cu_q[s] .. cu_q[s+1]-1 of q (nq of them), its keys and values tokens
 * cu_k[s] .. cu_k[s+1]-1 of k and v (nk).  Query head h reads key/value head
 * h / (Hq / Hkv).  With a query's row q, keys K_j and values V_j of its
 * sequence and head, over the keys it sees (causal = 0: all; causal = 1:
 * query i sees key j iff j <= i + nk - nq, the last query sees all keys):
 *   s_j = sm_scale <q, K_j>,  p_j = exp(s_j) / sum exp(s),  o = sum p_j V_j,
 *   lse = log(sum exp(s))
 * A row that sees no key has o = +0 and lse = -Inf.  Keys that a row does not
 * see do not enter it, whatever they hold (NaN and Inf included); an infinite
 * value that it sees enters as that infinity, however small its p is.
 * <q, K_j> and sums are FP32 of exact products; p_j enters the second
 * product as IEEE half relative to the row's running maximum.
 *
 * Outputs, each optional (NULL) but not all: o: FP16 codes (needed by the
 * backward pass); o8: FP8 codes of o * o8_scale (the next GEMM's operand);
 * lse: Hq x Tq floats (lse[h * Tq + t]; needed by the backward pass).
 * q, o, o8: Tq x Hq x D; k, v: Tk x Hkv x D, each with a token stride _ts and
 * a head stride _hs, the D entries contiguous (slices of one projection's
 * result are fine).  16-byte aligned pointers and strides with D a multiple
 * of 16 load 16 bytes at a time; other operands are read byte by byte.
 * cu_q, cu_k: S + 1 int64 each, non-decreasing from 0 to Tq / Tk (values
 * outside are clamped there; tokens of no sequence are not written).
 * max_q, max_k: the longest nq and nk, which choose the plan (a wrong value
 * costs speed only).  sm_scale > 0 and finite.
 * workspace: attn_fwd_fp8_workspace_size bytes for the fastest plan, or none
 * (workspace_bytes == 0, then a plan that needs none); it holds keys and
 * values laid out for the matrix cores, an order of the tiles and the partial
 * results of key ranges that several workgroups share.  Nothing in it is kept
 * from one call for the next.
 * Errors: FP8T_EINVAL (negative size, D not 1 .. FP8T_ATTN_MAX_D, Hq not a
 * multiple of Hkv, Hq above 65535, S, Tk or Tq Hq / Hkv above 2^31 - 4097, more
 * than 2^24 - 1 tiles of rows or keys (S Hkv and one for every 32 or more rows
 * or 64 or more keys of a head), a
 * flag not 0/1, sm_scale not positive and finite, negative input stride, an
 * output stride that makes rows overlap, NULL pointer for non-empty data, no output, NULL
 * workspace with workspace_bytes > 0, or one that is not 16-byte aligned where
 * it is used); FP8T_EWORKSPACE (0 < workspace_bytes < the query); FP8T_EHIP.
 */
int attn_fwd_fp8(const uint8_t* q, int64_t q_ts, int64_t q_hs, const uint8_t* k, int64_t k_ts,
                 int64_t k_hs, const uint8_t* v, int64_t v_ts, int64_t v_hs, const int64_t* cu_q,
                 const int64_t* cu_k, int64_t S, int64_t Tq, int64_t Tk, int64_t max_q,
                 int64_t max_k, int64_t Hq, int64_t Hkv, int64_t D, int causal, float sm_scale,
                 uint16_t* o, int64_t o_ts, int64_t o_hs, uint8_t* o8, int64_t o8_ts, int64_t o8_hs,
                 float o8_scale, float* lse, void* workspace, size_t workspace_bytes,
                 hipStream_t stream);

/*
 * attn_fwd_fp8_workspace_size -- bytes of workspace attn_fwd_fp8's fastest
 * plan needs on the current device (0 if none, or for invalid sizes).
 */
size_t attn_fwd_fp8_workspace_size(int64_t S, int64_t Tq, int64_t Tk, int64_t max_q, int64_t max_k,
                                   int64_t Hq, int64_t Hkv, int64_t D, int causal);

/*
 * attn_bwd_fp8 -- gradients of attn_fwd_fp8.  With e = value(d_o[t, h, .])
 * the error of o (FP8 codes, loss-scaled), p_j recomputed from lse,
 * delta = <e, o>:
 *   dV_j = sum p_j e          dS_j = p_j (<e, V_j> - delta) sm_scale
 *   dq   = sum_j dS_j K_j     dK_j = sum dS_j q
 * the sums of dK_j and dV_j over the queries that see key j, in every query
 * head that shares its key head.  dq, dk, dv: codes of grad_format
 * (FP8T_FMT_FP16 or FP8T_FMT_FP8) of the FP32 sums times grad_scale, strides
 * as q, k, v's.  Rows that see no key have dq = +0; keys that no query sees
 * have dK = dV = +0.
 * o (FP16 codes) and lse are attn_fwd_fp8's results for the same arguments.
 * p_j carries lse's rounding: it is off by up to 2^-22 max |s| of itself, so
 * gradients want scores below some 2^15 (attn_fwd_fp8 takes any).
 * The two products with p_j and dS_j use them as IEEE half: p_j times 2^15 (dV
 * loses up to 2^-40 of each error e), dS_j times a power of two that the row
 * (for dq) or the key (for dK) finds for itself, whatever other rows, keys and
 * sequences hold.
 * workspace: at least attn_bwd_fp8_workspace_size bytes, 16-byte aligned (it
 * holds delta, queries, errors, keys and values laid out for the
 * matrix cores, an order of the tiles and partial results of dk and dv).
 * Every other convention is attn_fwd_fp8's.
 * Errors: as attn_fwd_fp8, FP8T_EINVAL for another grad_format or a workspace
 * that is not 16-byte aligned, and FP8T_EWORKSPACE for workspace_bytes below
 * the query (0 included, where the query is not 0).
 */
int attn_bwd_fp8(const uint8_t* q, int64_t q_ts, int64_t q_hs, const uint8_t* k, int64_t k_ts,
                 int64_t k_hs, const uint8_t* v, int64_t v_ts, int64_t v_hs, const int64_t* cu_q,
                 const int64_t* cu_k, int64_t S, int64_t Tq, int64_t Tk, int64_t max_q,
                 int64_t max_k, int64_t Hq, int64_t Hkv, int64_t D, int causal, float sm_scale,
                 const uint16_t* o, int64_t o_ts, int64_t o_hs, const uint8_t* d_o, int64_t do_ts,
                 int64_t do_hs, const float* lse, void* dq, int64_t dq_ts, int64_t dq_hs, void* dk,
                 int64_t dk_ts, int64_t dk_hs, void* dv, int64_t dv_ts, int64_t dv_hs,
                 int grad_format, float grad_scale, void* workspace, size_t workspace_bytes,
                 hipStream_t stream);

/* attn_bwd_fp8_workspace_size -- bytes of workspace attn_bwd_fp8 needs (0 for
 * invalid or empty sizes). */
size_t attn_bwd_fp8_workspace_size(int64_t S, int64_t Tq, int64_t Tk, int64_t max_q, int64_t max_k,
                                   int64_t Hq, int64_t Hkv, int64_t D, int causal);

/*
 * distill_loss -- Kullback-Leibler distillation from a teacher's top logits,
 * loss and gradient in one pass over the student's logits.
 *
 * For row n with logits z = value(z[n, .]) (V of them) and the teacher's k
 * entries (idx[n, i], t[n, i]); an entry with idx outside [0, V) is unused:
 *   p = softmax(z / tau),  q = softmax over the used entries of t / tau
 *   loss[n] = w[n] tau^2 sum_i q_i (log q_i - log p[idx_i])
 *   g[n, v] = w[n] tau grad_scale (p[v] - sum of q_i with idx_i = v)
 * g is the gradient of the loss for z, times grad_scale (a loss scale), in
 * g_format (FP16 or FP8 codes rounded to nearest even as the quantizers do,
 * or floats).  w: per-row weights (1 / rows of a batch mean; 0 for padding),
 * NULL for 1.  A row with w = 0, without a used entry, or with no used
 * teacher logit above -Inf has loss +0 and g +0, whatever z holds.  An
 * entry that occurs twice counts twice.  Terms with q_i = 0 add 0.  Powers are
 * taken of a logit's distance from the row's largest; below 2^-126 they are 0.
 *
 * z: N x V in z_format (F32 or FP16), row stride z_ld >= V; idx (int64) and
 * t (t_format F32 or FP16): N x k contiguous, 0 <= k <= 4096; w, loss: N
 * floats; g: N x V, g_ld >= V.  loss or g may be NULL, not both.  g may be z
 * itself (same format and stride); otherwise they must not overlap.
 * Errors: FP8T_EINVAL (negative size, N above 2^31 - 4097 or V above 2^31 - 16385, k > 4096, tau
 * not from 2^-30 to 2^30, unknown format, a stride too small, NULL pointer
 * for non-empty data, no output); FP8T_EHIP.
 */
int distill_loss(const void* z, int z_format, int64_t z_ld, const int64_t* idx, const void* t,
                 int t_format, int64_t k, const float* w, int64_t N, int64_t V, float tau,
                 float grad_scale, float* loss, void* g, int g_format, int64_t g_ld,
                 hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif
