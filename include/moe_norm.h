/*
 * libmoe -- the step between two blocks of a residual stream: the norm behind a block, its
 * gate and residual scale, the residual sum, and the norm in front of the next block, in one
 * pass over the rows; and the norm in front of the first block alone.  With backward passes.
 *
 *   norm(v)    = w * (v - m) * f + b       f = 1 / sqrt(mean((v - m)^2) + eps); m = mean(v)
 *                                          (MOE_NORM_LAYER) or 0 (MOE_NORM_RMS), per row
 *   before:      next = norm_next(x)
 *   after:       r    = x + scale * gate[g(t)] * norm(z)       rounded to the residual's type
 *                next = norm_next(r)                           of r as it is stored
 *
 * x is the residual stream, z the block's output (what moe_combine wrote, or an attention
 * block's), r the new residual stream, next the next block's input.  g(t) = t / gate_tokens:
 * a row of gates for every gate_tokens rows (a sequence, say; the last group may be short), one
 * for all where gate_tokens is 0.
 *
 * Backward, for a loss whose gradients with respect to r (what does not come through next) and
 * next are dr and dnext; both norms' factors are computed again from r and z:
 *   D      = dr + f_r (u - mean(u) [layer] - rhat mean(u rhat))        u = w_next dnext, rhat = (r - m_r) f_r
 *   dx     = D                                     dw_next = sum_t dnext rhat     db_next = sum_t dnext
 *   a      = scale gate[g(t)] D                    dw = sum_t a zhat              db = sum_t a
 *   dz     = f_z (v - mean(v) [layer] - zhat mean(v zhat))             v = w a, zhat = (z - m_z) f_z
 *   dgate[g] = sum over the rows of g of scale D (w zhat + b)
 * Sums, factors and vector gradients are fp32, in an order that depends on the shape alone.
 *
 * Conventions as in moe.h: device pointers (16-byte aligned), enqueue only, caller-owned buffers,
 * status codes, moe_last_error.  Two buffers may be one: r may be x, and dx may be dr.
 */
#ifndef MOE_NORM_H
#define MOE_NORM_H

#include "moe.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { MOE_NORM_RMS = 0, MOE_NORM_LAYER = 1 } moe_norm_kind;

/* Element types: 0 fp32 (MOE_F32), 1 bf16 (MOE_BF16), 2 fp16 (z only: expert outputs are fp16). */
typedef struct {
    int32_t T;           /* rows, >= 1 */
    int32_t d;           /* row length: a multiple of 8, 8 .. 16384 */
    int32_t kind;        /* moe_norm_kind, of both norms */
    int32_t dtype;       /* next and dnext: 0 or 1 */
    int32_t res;         /* x, r, dr and dx: 0 or 1 */
    int32_t z;           /* z: 0, 1 or 2; dz is fp32 where z is, else bf16 */
    int32_t gate_tokens; /* rows that share a row of gates; 0: all */
    float eps;           /* >= 0 */
    float scale;         /* of the gated norm in the residual sum */
} moe_norm_shape;

/* Host, pure.  Bytes of workspace the backward calls need (the forward calls need none);
 * 0 on an invalid shape. */
size_t moe_norm_workspace_bytes(const moe_norm_shape *n);

/* next [T,d] = norm_next(x [T,d]).  w_next fp32 [d]; b_next fp32 [d] or NULL. */
moe_status moe_norm_before(const moe_norm_shape *n, const void *x, const float *w_next,
                           const float *b_next, void *next, void *stream);

/* dx [T,d] = dr + the norm's input gradient; dw_next fp32 [d], db_next fp32 [d] or NULL:
 * overwritten. */
moe_status moe_norm_before_backward(const moe_norm_shape *n, const void *x, const float *w_next,
                                    const void *dnext, const void *dr, void *dx, float *dw_next,
                                    float *db_next, void *workspace, void *stream);

/* r, next [T,d] from x, z [T,d].  w, w_next fp32 [d]; b, b_next fp32 [d] or NULL;
 * gate fp32 [G,d], G = ceil(T / gate_tokens) or 1, or NULL (all ones). */
moe_status moe_norm_after(const moe_norm_shape *n, const void *x, const void *z, const float *w,
                          const float *b, const float *gate, void *r, const float *w_next,
                          const float *b_next, void *next, void *stream);

/* All gradients, overwritten: dx [T,d] in the residual's type, dz [T,d]; dw, dw_next fp32 [d];
 * db, db_next fp32 [d] or NULL; dgate fp32 [G,d] or NULL.  z, r, w, b, gate, w_next as the forward
 * call had them. */
moe_status moe_norm_after_backward(const moe_norm_shape *n, const void *z, const void *r,
                                   const float *w, const float *b, const float *gate,
                                   const float *w_next, const void *dr, const void *dnext, void *dx,
                                   void *dz, float *dw, float *db, float *dgate, float *dw_next,
                                   float *db_next, void *workspace, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MOE_NORM_H */
