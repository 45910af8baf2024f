/*
 * libmoe -- rows and weights held in 8 bits, and the operators of a served block on them: the norm that
 * writes such rows, a linear map with bias, activation and residual, the gated experts' products, and the
 * dispatch of such rows.
 *
 * A row v of K values is held as
 *   most  = max |v|            scale = most / 127 (fp32)
 *   code  = round(127 v / most), ties to even, int8 of -127 .. 127; 0 where most is 0
 * and stands for code * scale.  A row with an infinity or NaN is held as codes 0 and scale NaN: it has no
 * finite product, the others are untouched.
 *
 *   rows      q int8 [R, K], scale fp32 [R]
 *   weights   q int8 [E, N, K], scale fp32 [E, N]: a row per output column, held as any other row is
 *
 * Products are of whole numbers with 32-bit sums, which are exact, so that every kernel, tile and split gives the same
 * sums; a sum becomes (float)sum * scale of the row * scale of the column in fp32.  Codes of -128 are taken as they are.
 * Nothing is packed beforehand: the kernels read these as they are.
 *
 * Conventions as in moe.h: device pointers, 16-byte aligned, enqueue only, caller-owned buffers and
 * workspaces, status codes, moe_last_error.
 */
#ifndef MOE_Q8_H
#define MOE_Q8_H

#include "moe.h"
#include "moe_norm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types below: 0 fp32, 1 bf16, 2 fp16 (as in moe_norm_shape). */

/* x [R, K] of `type` to codes and scales; K a multiple of 16, 16 .. 65536.  The codes are the rounded quotients
 * themselves, not those of an approximation.  For weights: R = E N. */
moe_status moe_q8_rows(int64_t R, int32_t K, int32_t type, const void *x, void *q, float *scale, void *stream);

/* The values that codes stand for: the fp32 products code * scale, of which 16-bit types are rounded from (so twice in all: where the first
 * rounding meets a border of two values, one of 2^14 in fp16, the one that is farther by 2^-24 may be taken); K as above. */
moe_status moe_q8_values(int64_t R, int32_t K, int32_t type, const void *q, const float *scale, void *x, void *stream);

/* moe_norm_before and moe_norm_after (moe_norm.h) with next also, or (next NULL) only, in 8 bits: q [T, d], scale [T], of
 * norm_next's fp32 value, which is not rounded in between.  d a multiple of 16.  The backward calls of moe_norm.h take the
 * same buffers: gradients pass the rounding as if it were not there. */
moe_status moe_norm_before_q8(const moe_norm_shape *n, const void *x, const float *w_next, const float *b_next, void *next,
                              void *q, float *scale, void *stream);
moe_status moe_norm_after_q8(const moe_norm_shape *n, const void *x, const void *z, const float *w, const float *b,
                             const float *gate, void *r, const float *w_next, const float *b_next, void *next, void *q,
                             float *scale, void *stream);

/* R rows in all, of E experts (1..64) with matrices [N, K]; K a multiple of 16, 16 .. 65536. */
typedef struct {
    int32_t R;
    int32_t E;
    int32_t N;
    int32_t K;
    int32_t act;         /* moe_act, of any kind */
    int32_t res;         /* type of r */
    int32_t y;           /* type of y */
} moe_q8_shape;

/* y [R, N] = act(x W^T + bias) + r, in fp32 and rounded once to y's type.  act(v) is off by some roundings of fp32: silu and the tanh form
 * by (8 + 3 |e|) 2^-24 of its size, 2^e their exponential (from 2^126 on the value is 0); the erf form by (14 + 1.5 v^2) 2^-24 under an fp32 y,
 * under a 16-bit y by 2^-17.8 for |v| up to 2, 2^-13.5 down to v = -8, and 1e-16 below; relu and identity by nothing.
 *   x, x_scale         the rows; expert e owns rows [offsets[e], offsets[e+1])
 *   w, w_scale         the experts' matrices
 *   bias               fp32 [E, N] or NULL
 *   r                  [R, N] or NULL; it may be y where their types are the same
 * N below 2^21.  The same bits whichever kernel a shape's size chooses.  Rows of y at or beyond offsets[E] are left as they are. */
moe_status moe_q8_linear(const moe_q8_shape *s, const void *x, const float *x_scale, const int32_t *offsets, const void *w,
                         const float *w_scale, const float *bias, const void *r, void *y, void *stream);

/* Which kernel moe_q8_linear launches for the shape, and moe_gated_ffn_q8 for its product `which` (0: first projections; 1: second), written
 * to name (host, len bytes, always terminated) as "<kernel> <tile rows>x<tile columns>", with " split" behind it where a block shares out
 * a tile's depth, " deep" where five stages of loads are on their way, " once" where the weights go past the caches and " tail" for the form of a
 * kernel of tiles that takes depths of no whole stages of 128, and, of those without " deep", of fewer than four; so that a measurement or a
 * test can say which kernel it ran.  MOE_EINVAL for a null name, len == 0 or another which; else as the call that launches it. */
moe_status moe_q8_linear_kernel(const moe_q8_shape *s, char *name, size_t len);
moe_status moe_gated_q8_kernel(const moe_shape *s, int32_t which, char *name, size_t len);

/* moe_dispatch of rows in 8 bits: x [T, d_model] with x_scale [T] to xe [moe_max_rows, d_model] with xe_scale
 * [moe_max_rows].  xe and xe_scale may both be NULL: only counts, offsets, slot_of and src_of are wanted, for the
 * block's first product to take the rows where they are.  s is the layer's shape (its dtype is not used). */
moe_status moe_dispatch_q8(const moe_shape *s, const void *x, const float *x_scale, const int32_t *expert_idx,
                           int32_t *counts, int32_t *offsets, int32_t *slot_of, int32_t *src_of, void *xe, float *xe_scale,
                           void *workspace, void *stream);

/* Host, pure.  Bytes of workspace of moe_gated_ffn_q8 (0 if unsupported). */
size_t moe_gated_q8_workspace_bytes(const moe_shape *s);

/* moe_gated_ffn (moe_gated.h) of a MOE_BF16 layer on rows and weights in 8 bits:
 *   G = x Wg[e]^T   U = x Wu[e]^T   H = act(G) * U, rounded to fp16 and held in 8 bits by row   ye = H W2[e]^T, fp16
 *   q13 [E, 2 d_ff, d_model]: rows [0, d_ff) are Wg, [d_ff, 2 d_ff) Wu; q2 [E, d_model, d_ff]; each with its scales
 *   x, x_scale   src_of NULL: expert-major, [moe_max_rows, d_model] and [moe_max_rows]; else [T, d_model] and [T], and
 *                slot i takes the row of token src_of[i] / k (src_of as the dispatch wrote it)
 * d_model and d_ff multiples of 16, at most 65536, and 2 d_ff d_model below 2^31 - 2^26; with src_of T d_model below 2^31 - 2^20.
 * act is as exact as under a 16-bit y of moe_q8_linear.  A value of H past 65504 is infinite, and its row then NaN; below 6.1e-5 values of
 * H are rounded to multiples of 2^-24, so a row of none larger is held more coarsely than its codes would. */
moe_status moe_gated_ffn_q8(const moe_shape *s, const void *x, const float *x_scale, const int32_t *src_of,
                            const int32_t *offsets, const void *q13, const float *scale13, const void *q2,
                            const float *scale2, void *ye, void *workspace, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MOE_Q8_H */
