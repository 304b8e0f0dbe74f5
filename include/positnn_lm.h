/* positnn_lm.h - C ABI of the operators that a language model needs around the products of positnn.h:
 * the RMS norm with the residual's addition, attention with a sliding window and sinks, and the log
 * probabilities of given tokens; each forward and backward.
 *
 * The conventions of positnn.h hold: device pointers owned by the caller, calls asynchronous on `stream`, no
 * device memory allocated, freed or kept, a pnn_status from every function, nothing launched where the
 * arguments are refused, zero-sized problems PNN_OK with nothing touched.  That is a problem without rows, columns or
 * vocabulary, without sequences, heads or elements of a head, and attention without queries (backward: without
 * queries and keys): sums over nothing (dw of no rows, a row's statistics where it has no columns) are the caller's to fill in.  In addition:
 *  - An element format is a posit of at most 16 bits, PNN_BF16 or PNN_F32 (PNN_EUNSUPPORTED for posit<32,2> and
 *    PNN_F64, PNN_EINVAL for an unknown code).  Posit tensors hold patterns.  NaR reads as NaN, and a NaN or an
 *    infinity that is stored in a posit format becomes NaR; a nonzero finite value never becomes zero in one.
 *  - These operators have no quire: values are computed in binary32 (posits of at most 16 bits and products of two
 *    of them with 8 significant bits are exact there), sums and softmax statistics are kept in binary32, and each
 *    output is rounded once, to its format.  Results do not depend on other work on the device: no sum is taken in
 *    an order that varies from call to call.
 *  - Sizes: fewer than 2^31 rows and columns, a vocabulary below 2^31; in attention B < 16384, HQ < 65536, D <= 128, LQ * HQ / HKV and LK at
 *    most 2^31 - 128, and no more rows and keys than the workgroups of a launch (else PNN_EUNSUPPORTED).  Squares and exponents have binary32's range: a row whose
 *    sum of squares passes it has rstd 0, a logit whose product with the inverse temperature does counts as infinite.
 *  - ld* are row pitches in elements, at least the row's length (else PNN_EINVAL).  Any alignment that the element
 *    type has is accepted.  A workspace is 16-byte aligned (else PNN_EINVAL) and at least as large as the matching
 *    query says (else PNN_EWORKSPACE); its contents on entry do not matter and are not preserved.
 */
#ifndef POSITNN_LM_H
#define POSITNN_LM_H

#include "positnn.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { PNN_BF16 = 102 }; /* bfloat16: an element format of the entry points of this header only */

/* ---- RMS norm with the residual's addition ----
 * For each row of `cols` elements:
 *   h = round_fres(x + res)  (sum in binary32; res NULL: h = x, and res_out is not written)
 *   rstd = 1 / sqrt(mean(h^2) + eps),  t_j = h_j * w_j
 *   scale NULL:  y_j = round_fy(t_j * rstd)
 *   else:        y_j = round_fy(t_j * 2^(2-e)) and scale = rstd * 2^(e-2), where 2^e <= max |t_j| < 2^(e+1) (e = 2 for
 *                a row of zeros): the row's largest magnitude lies in [4, 8), where a posit keeps most of its bits for
 *                the rest of the row, and row = scale * patterns' values.  A row with a NaN or an infinity is NaR
 *                throughout and its scale NaN.
 * x (fx), res and res_out (fres), y (fy) are rows x cols with pitches; w (fw) has cols elements; scale and rstd (each may
 * be NULL) are one binary32 per row.  res_out is required where res is given and may be res itself. */
int posit_rmsnorm_fwd(void* stream, int fx, int fres, int fw, int fy, int64_t rows, int64_t cols,
                      const void* x, int64_t ldx, const void* res, int64_t ldr, const void* w, float eps,
                      void* res_out, int64_t ldo, void* y, int64_t ldy, float* scale, float* rstd);

/* Gradient of  y = h * w * rstd  (the unscaled output) for dy (fd):
 *   g = dy * w,  dx = round_fdx( rstd * g - rstd^3 * mean(g * h) * h + dres ),  dw = round_fdw( sum over rows of dy * h * rstd )
 * h (fh) is res_out of the forward call (x where it had no residual), rstd what it returned.  dres (fdres, may be NULL)
 * is the gradient that reaches h past the norm; dx is that of both x and res.  dw may be NULL. */
int posit_rmsnorm_bwd(void* stream, int fd, int fh, int fw, int fdres, int fdx, int fdw, int64_t rows, int64_t cols,
                      const void* dy, int64_t lddy, const void* h, int64_t ldh, const void* w, const float* rstd,
                      const void* dres, int64_t lddr, void* dx, int64_t lddx, void* dw, void* workspace, size_t workspace_bytes);
size_t posit_rmsnorm_bwd_workspace(int64_t rows, int64_t cols);

/* y[r][j] = round_fout(scale[r] * x[r][j]): what a row's scale still owes after a product of patterns, or the values that
 * scaled rows stand for. */
int posit_scale_rows(void* stream, int fin, int fout, int64_t rows, int64_t cols, const void* x, int64_t ldx,
                     const float* scale, void* y, int64_t ldy);

/* ---- attention with a sliding window and sinks ----
 * Batch b, query i (0 <= i < LQ), head h; key and value heads are shared by HQ / HKV query heads each.  A sequence holds
 * n = lens[b] keys (lens NULL: LK; values outside 0 .. LK are taken as the nearest of them), and its queries are the last
 * LQ positions: p = n - LQ + i.  Query i sees key j where  0 <= j <= p  and  (window == 0 or j > p - window or j < sinks).
 *   s_j = scale * sum_d q[b,i,h,d] * k[b,j,h',d]   o[b,i,h,:] = sum_j softmax(s)_j * v[b,j,h',:]   lse[b,h,i] = log sum_j exp(s_j)
 * A query that sees nothing (p < 0) has o = 0 and lse = -inf.  Only what a query sees can make its output NaN.
 * Formats: q in fq, k and v in fkv, one of those that bfloat16 holds exactly: posit<8,0>, (8,1), (8,2), (10,1), (10,2),
 * (12,2) and PNN_BF16 (else PNN_EUNSUPPORTED); o in any element format.  Products of q and k are exact; the
 * probabilities go into the second product rounded to 16 bits, or to 8 where o and o_copy are PNN_BF16, which keeps no more.
 * Strides are in elements; the elements of a head are contiguous.  Output layouts: o dense [b][i][h][d]. */
typedef struct {
    int64_t B, HQ, HKV, LQ, LK, D;   /* D <= 128, HQ a multiple of HKV */
    int64_t window, sinks;           /* both >= 0; window 0 = none */
    float scale;
    int64_t qb, ql, qh;              /* strides of q (and, backward, of d_o): batch, position, head */
    int64_t kb, kl, kh;              /* of k */
    int64_t vb, vl, vh;              /* of v */
} pnn_attention_desc;

/* o_copy (fcopy, may be NULL) receives the same output rounded to fcopy: what posit_attention_bwd reads beside the
 * narrow o that the next product reads.  lse may be NULL. */
int posit_attention_fwd(void* stream, int fq, int fkv, int fout, const pnn_attention_desc* desc, const void* q, const void* k,
                        const void* v, const int32_t* lens, void* o, float* lse, int fcopy, void* o_copy,
                        void* workspace, size_t workspace_bytes);

/* Gradients for d_o (fd, one of the formats of q; strides of q):  P = exp(s - lse),  dV = P^T dO,  dS = P * (dO V^T - rowsum(dO * o)),
 * dQ = scale * dS K,  dK = scale * dS^T Q;  dK and dV are summed over the query heads that share them.  o (fo, dense) and lse
 * are outputs of the forward call; D = rowsum(dO * o) is as exact as fo, so where fout of that call is narrow pass its o_copy.  dq is dense like o, dk and
 * dv dense [b][j][h'][d], all in fout; keys that nothing sees get zeros.  P and dS go into the products behind them rounded to 16 bits, or to 8 where fout is
 * PNN_BF16, which keeps no more: PNN_F32 gradients are the more exact ones. */
int posit_attention_bwd(void* stream, int fd, int fq, int fkv, int fo, int fout, const pnn_attention_desc* desc, const void* d_o,
                        const void* q, const void* k, const void* v, const int32_t* lens, const void* o, const float* lse,
                        void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes);

/* which: 0 = forward, 1 = backward.  Depends on which, fkv and the sizes in desc only. */
size_t posit_attention_workspace(int which, int fkv, const pnn_attention_desc* desc);

/* ---- log probabilities of given tokens ----
 * For each row of `vocab` logits z (fz), with z' = inv_temperature * z (> 0, finite):
 *   lse = log sum exp z',  logprob = z'[target] - lse,  entropy = lse - sum_j p_j z'_j  with  p = exp(z' - lse)
 *   top alternatives: the `top` (<= 64) largest logits, ties to the lowest index, with their log probabilities
 * Logits of -inf have probability zero and are never listed; places that are left hold index -1 and -inf.  A negative target
 * means none: logprob 0 and no gradient through it; one >= vocab gives NaN.  A row with a NaN or +inf is NaN throughout
 * (indices -1); a row of -inf alone has lse -inf, logprob -inf, entropy 0.  targets (int32), logprob, lse and entropy are one
 * value per row (targets and logprob may both be NULL); top_logprob and top_index are [rows][top]. */
int posit_token_logprob_fwd(void* stream, int fz, int64_t rows, int64_t vocab, const void* logits, int64_t ldz, const int32_t* targets,
                            float inv_temperature, int top, float* logprob, float* lse, float* entropy, float* top_logprob,
                            int32_t* top_index, void* workspace, size_t workspace_bytes);
size_t posit_token_logprob_workspace(int fz, int64_t rows, int64_t vocab, int top);

/* dlogits[r][j] = round_fg( inv_temperature * ( g_logprob[r] * ([j == target] - p_j) - g_entropy[r] * p_j * (log p_j + entropy[r]) ) )
 * from lse and entropy of the forward call.  g_logprob (with targets) and g_entropy may each be NULL.  A probability of zero has no gradient. */
int posit_token_logprob_bwd(void* stream, int fz, int fg, int64_t rows, int64_t vocab, const void* logits, int64_t ldz, const int32_t* targets,
                            float inv_temperature, const float* lse, const float* entropy, const float* g_logprob, const float* g_entropy,
                            void* dlogits, int64_t ldg);

#ifdef __cplusplus
}
#endif
#endif /* POSITNN_LM_H */
