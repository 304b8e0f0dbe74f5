/* positnn_generate.h - C ABI of the operators with which a language model generates text, beside those of positnn_lm.h: norms of queries
 * and keys with the rotation by their positions (forward and backward), a cache of keys and values in pages with the attention that
 * reads it, and the draw of the next token from given random numbers.
 *
 * The conventions of positnn.h and positnn_lm.h hold: device pointers owned by the caller, calls asynchronous on `stream`, no device memory
 * allocated, freed or kept, a pnn_status from every function, nothing launched where the arguments are refused, zero-sized problems PNN_OK with
 * nothing touched; element formats are posits of at most 16 bits, PNN_BF16 and PNN_F32; each output is rounded once; sums, norms and softmax
 * statistics have 32 bits or more; results do not depend on other work on the device.  Strides are in elements, not negative, and the elements of a head are
 * contiguous.  Any alignment that the element type has is accepted; a cache's tensors and a workspace are 16-byte aligned (else PNN_EINVAL).
 */
#ifndef POSITNN_GENERATE_H
#define POSITNN_GENERATE_H

#include "positnn_lm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A cache's format of 4 bits: binary floats with the magnitudes 0 1/2 1 3/2 2 3 4 6, sign in bit 3, in blocks of 32 elements of a head (the last one shorter
 * where D is no multiple of 32), each with a byte b that stands for 2^(b-127), or for NaN throughout where it is 255.  A block's power is the
 * smallest that leaves its largest magnitude at 7 or below, so that nothing is off by more than half a step of its own binade; elements are
 * rounded to nearest, ties to even, and to 6 above it.  Powers from 2^-124 to 2^125 are written (of others, what is read is binary32's value, infinite from 2^128 on).  A block with a NaN or an infinity becomes NaN.
 * Unlike posits these round to zero what is below a quarter of the power. */
enum { PNN_F4 = 103 };

/* ---- norms of queries and keys, with the rotation by positions ----
 * For each row of T, head h of q (HQ heads, weight wq) and of k (HKV heads, weight wk), each of D elements x:
 *   rstd = 1 / sqrt(mean(x^2) + eps),  t_j = x_j * w_j * rstd      (wq and wk NULL: t = x, no norm)
 *   of the first R elements, pair i (0 <= i < R / 2) is (a, b) = (i, i + R / 2), or (2i, 2i + 1) with `neighbours`; with angle = pos[row] * inv_freq[i] in 64 bits
 *   y_a = t_a cos - t_b sin,  y_b = t_b cos + t_a sin              (pos NULL: y = t); the elements from R on stay
 * q, k in fx; weights in fw; outputs in fy, dense [T][HQ][D] and [T][HKV][D]; rstd (may be NULL) one binary32 per row and head, [T][HQ + HKV], queries
 * first.  inv_freq is R / 2 values of binary64, pos T of int32 (of either sign).
 * D even and at most 256, T below 2^31, HQ + HKV below 65536, strides below 2^32 (else PNN_EUNSUPPORTED); R even and at most D (else PNN_EINVAL). */
typedef struct {
    int64_t T, HQ, HKV, D, R;
    int64_t ql, qh, kl, kh;      /* strides of q and k: row, head */
    int64_t gql, gqh, gkl, gkh;  /* backward: of the outputs' gradients */
    int32_t neighbours;
    float eps;
} pnn_heads_desc;

int posit_qk_norm_rope_fwd(void* stream, int fx, int fw, int fy, const pnn_heads_desc* desc, const void* q, const void* k, const void* wq, const void* wk,
                           const int32_t* pos, const double* inv_freq, void* yq, void* yk, float* rstd);

/* Gradients for dyq and dyk (fd): with g the gradient rotated back (by -angle) and xhat = x * rstd
 *   dx = round_fdx( rstd * (g * w - xhat * mean(g * w * xhat)) ),  dw = round_fdw( sum over rows and heads of g * xhat )
 * (without norm dx = g).  rstd is that of the forward call (NULL without norm).  dq and dk are dense; dwq and dwk may be NULL, and are zeros where queries or keys alone have no
 * heads. */
int posit_qk_norm_rope_bwd(void* stream, int fd, int fx, int fw, int fdx, int fdw, const pnn_heads_desc* desc, const void* dyq, const void* dyk, const void* q,
                           const void* k, const void* wq, const void* wk, const float* rstd, const int32_t* pos, const double* inv_freq, void* dq, void* dk, void* dwq,
                           void* dwk, void* workspace, size_t workspace_bytes);
size_t posit_qk_norm_rope_bwd_workspace(const pnn_heads_desc* desc);

/* ---- a cache of keys and values in pages ----
 * Two tensors of `pages` pages, each [pages][HKV][a page's elements], `page` tokens to a page (a power of two from 16 to 4096), in fcache: an 8-bit posit,
 * PNN_BF16 or PNN_F4.  A page of one head holds keys as [token][D] and values as [token / 4][D / 8][token % 4][8] (four tokens' eight elements
 * side by side, as attention takes them).  PNN_F4: that is the order of half bytes, low one first; behind the page * D / 2 bytes lie the blocks' powers, of
 * keys [token][block], of values [token / 4][block][token % 4], page * ceil(D / 32) bytes.  D is a multiple of 8, at most 128.
 * Token j of sequence b lies in page table[b * pitch + j / page] (int32), at j % page.  Entries that no token of a sequence needs are not read.  Where an entry that is
 * needed is no page's number (below 0 or from `pages` on), nothing is written there and what is read there is NaN.
 * New tokens of B sequences are packed rows: those of sequence b are starts[b] .. starts[b+1]-1 (B + 1 values of int32, ascending; NULL: row b is sequence b's only one,
 * T = B), the last ones of its lens[b] tokens (int32, the new ones included): row t is token lens[b] - (starts[b+1] - t).  Rows of no sequence are left as they were. */
typedef struct {
    int64_t T, B, HQ, HKV, D, R;
    int64_t page, pages, columns, pitch;  /* columns: page numbers that a sequence's row of the table holds */
    int64_t ql, qh, kl, kh, vl, vh;       /* strides: row, head */
    int64_t window, sinks, most, longest; /* attention, read */
    float scale, eps;
    int32_t neighbours;
} pnn_paged_desc;

/* q, k and v (fx; strides) of the new tokens: q and k normalised (wq, wk in fw, both or none) and rotated (inv_freq, NULL for none) as above, by a token's place in its sequence; q
 * to yq (fq, dense [T][HQ][D]; q NULL: left out), k and v (as it is) into the pages.  What goes into the pages, and yq where fq is a posit, is computed in 64 bits and so the nearest to
 * the formulas' values; yq in PNN_BF16 and PNN_F32 in 32, as by posit_qk_norm_rope_fwd.  Strides below 2^32 (else PNN_EUNSUPPORTED).
 * A token without a place (before 0, beyond `columns` pages, in a page that is none) is left out of the cache; its query is written all the same.
 * The places of one call's tokens are the caller's to keep apart: of two sequences that share a page both may not write to the same place. */
int posit_cache_append(void* stream, int fx, int fw, int fq, int fcache, const pnn_paged_desc* desc, const void* q, const void* k, const void* v, const void* wq, const void* wk,
                       const double* inv_freq, const int32_t* starts, const int32_t* lens, const int32_t* table, void* k_pages, void* v_pages, void* yq);

/* The cache's values as dense rows k, v [B][longest][HKV][D] in fout: what posit_attention_fwd takes for a prompt on a filled cache.  Zeros behind a
 * sequence's end; NaN for tokens that lens counts beyond `columns` pages. */
int posit_cache_read(void* stream, int fcache, int fout, const pnn_paged_desc* desc, const int32_t* lens, const int32_t* table, const void* k_pages, const void* v_pages, void* k, void* v);

/* Attention of the packed rows q (fq, a format that bfloat16 holds exactly; strides ql, qh) over the pages, as posit_attention_fwd: row t of sequence b, at position
 * p = lens[b] - (starts[b+1] - t), sees token j where 0 <= j <= p and (window == 0 or j > p - window or j < sinks); the scores' factor is `scale`.
 * o (fout) dense [T][HQ][D], lse (may be NULL) [T][HQ]; a row that sees nothing has o = 0 and lse = -inf, one that sees a token in a page that is none NaN.
 * `longest` bounds lens and `most` the new tokens of a sequence: a length beyond `longest` (or beyond `columns` pages) is taken as that, and of more rows than `most` the first `most`
 * are written.  For few rows: most * HQ / HKV at most 1024 (else PNN_EUNSUPPORTED; a prompt's rows go through posit_cache_read and posit_attention_fwd). */
int posit_attention_paged(void* stream, int fq, int fcache, int fout, const pnn_paged_desc* desc, const void* q, const int32_t* starts, const int32_t* lens, const int32_t* table,
                          const void* k_pages, const void* v_pages, void* o, float* lse, void* workspace, size_t workspace_bytes);
size_t posit_attention_paged_workspace(const pnn_paged_desc* desc);

/* ---- the draw of the next token ----
 * For each row of `vocab` logits z (fz), in the order of falling logits, equal ones by rising index, and with w_j = exp((z_j - max z) / temperature):
 *   the first top_k stay (0 and below: all that are above -inf); of these the first whose weights before them sum to less than top_p of the sum (1 and above, and NaN: all;
 *   0 and below: the first one); of these the ones of w_j >= min_p (NaN: all; above 1 as 1)
 *   token: the first one whose weights up to it, itself included, sum to more than u times the sum of those that stay
 *   logprob: log of its share in that sum;  kept: how many stay
 * temperature, top_k (int32), top_p, min_p are one value per row, each may be NULL (1, 0, 1, 0).  A temperature of 0 takes the first token; one below 0 or NaN gives token -1 and
 * logprob NaN.  u is one binary32 per row; below 0 and NaN count as 0, what is not below 1 as the largest number below it.  Weights are rounded to multiples of 2^-s, s =
 * min(51, 62 - ceil(log2(vocab))), and their sums are exact; a min_p below 2^(-s-2) counts as 0.
 * A row with a NaN or +inf gives token -1, logprob NaN, kept 0; one of -inf alone -1, -inf and 0.  token (int32), logprob and kept (int32; each but token may be NULL) are one
 * value per row.  vocab and rows below 2^31 (else PNN_EUNSUPPORTED). */
int posit_sample(void* stream, int fz, int64_t rows, int64_t vocab, const void* logits, int64_t ldz, const float* u, const float* temperature, const int32_t* top_k,
                 const float* top_p, const float* min_p, int32_t* token, float* logprob, int32_t* kept, void* workspace, size_t workspace_bytes);
size_t posit_sample_workspace(int fz, int64_t rows, int64_t vocab);

#ifdef __cplusplus
}
#endif
#endif /* POSITNN_GENERATE_H */
