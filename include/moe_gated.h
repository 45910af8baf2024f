/*
 * libmoe -- experts that are gated feed-forward blocks: two projections side by side, the
 * activation of the one times the other, and the projection back.
 *
 *   G = xe Wg[e]     U = xe Wu[e]     H = act(G) * U     ye = H W2[e]         rows of expert e
 *
 * Rows are expert-major as moe_dispatch packs them: expert e owns rows [offsets[e], offsets[e+1]),
 * of which there are at most moe_max_rows(s).  A dense block is a layer of one expert (E = k = 1,
 * capacity = T, offsets {0, T}).  Around it moe_route, moe_dispatch and moe_combine are a gated MoE
 * layer's other parts, and moe_norm.h's calls the step to the next block.
 *
 * The layer's shape is a moe_shape with any of its activations, MOE_ACT_SILU among them; k, T and
 * capacity bound the rows only.  Types as in moe.h: MOE_BF16 layers take xe and the weights in bf16, hold
 * H (and what training keeps) in fp16 and write ye in fp16 (values past 65504 become infinite); MOE_F32 layers are fp32 throughout.
 * Products accumulate in fp32.  Rows at or beyond offsets[E] are neither read nor written.
 *
 * The same block with weights held as 4-bit codes, and one linear map of such weights, are at the end.
 *
 * Conventions as in moe.h: device pointers, 16-byte aligned, enqueue only, caller-owned buffers and
 * workspaces, status codes, moe_last_error.
 */
#ifndef MOE_GATED_H
#define MOE_GATED_H

#include "moe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Host, pure.  Bytes of the packed first projections W13p; the packed W2p has moe_packed_weight_bytes.
 * 0 on an invalid shape. */
size_t moe_gated_packed_bytes(const moe_shape *s);

/* Re-layout of the weights for the kernels: once for serving, in every step for training.
 *   W13 [E, d_model, 2 d_ff]: columns [0, d_ff) are Wg, [d_ff, 2 d_ff) Wu; W2 [E, d_ff, d_model].
 * MOE_BF16: W13p = bf16, each expert transposed, sixteen columns of Wg and the same sixteen of Wu in turn (the
 * last sixteen padded with zeros); W2p = fp16 [E, d_model, d_ff] as moe_pack_weights writes it.
 * MOE_F32: plain copies. */
moe_status moe_pack_gated_weights(const moe_shape *s, const void *W13, const void *W2, void *W13p,
                                  void *W2p, void *stream);

/* Host, pure.  Bytes of workspace of moe_gated_ffn; of one that is given pre and hid (0 if unsupported). */
size_t moe_gated_workspace_bytes(const moe_shape *s);
size_t moe_gated_kept_workspace_bytes(const moe_shape *s);

/* The block.  ye [rows, d_model].  pre, hid: both NULL, or (MOE_BF16) what the backward pass reads:
 * pre fp16 [rows, 2 d_ff] = [G | U], hid fp16 [rows, d_ff] = H, each rounded from fp32 (to infinity past 65504). */
moe_status moe_gated_ffn(const moe_shape *s, const void *xe, const int32_t *offsets,
                         const void *W13p, const void *W2p, void *ye, void *pre, void *hid,
                         void *workspace, void *stream);

/* Host, pure.  Bytes of workspace of moe_gated_ffn_backward; of one that is given pre and hid; 0 if unsupported. */
size_t moe_gated_backward_workspace_bytes(const moe_shape *s);
size_t moe_gated_kept_backward_workspace_bytes(const moe_shape *s);

/*
 * The block's gradients for a loss whose gradient with respect to ye is dye.  MOE_BF16 layers.
 *   dH = dye W2[e]^T     dG = dH * U * act'(G)     dU = dH * act(G)
 *   dxe = dG Wg[e]^T + dU Wu[e]^T     dW13[e] = xe^T [dG | dU]     dW2[e] = H^T dye
 *   xe, offsets, W13p as the forward call had them; W13, W2 in their canonical layouts;
 *   pre, hid   both NULL (the first projections are computed again), or as the forward call kept them
 *   dye        bf16 [rows, d_model]
 *   dxe        bf16 [rows, d_model]; dW13, dW2 bf16 in the weights' layouts: overwritten, zeros for an
 *              expert without rows
 * The products run on bf16 operands (dG, dU and H rounded to bf16) with fp32 sums, each rounded once to its
 * gradient's type.  A G or U past 65504 enters as infinity: with act'(G) and act(G) as their limits, and 0 where dH or act'(G)
 * is 0, so that a closed gate has gradients of 0 whatever its size; else the gradients are not finite.
 */
moe_status moe_gated_ffn_backward(const moe_shape *s, const void *xe, const int32_t *offsets,
                                  const void *W13, const void *W2, const void *W13p, const void *pre,
                                  const void *hid, const void *dye, void *dxe, void *dW13, void *dW2,
                                  void *workspace, void *stream);

/* Which kernel the calls above launch for a GEMM of a block of shape s (0: first projections; 1: second; of the backward
 * pass 2: dH; 3: dxe; 4: dW2; 5: dW13), written to name (host, len bytes, always terminated) as "<kernel> <tile rows>x<tile
 * columns>", with " deep" behind it where five stages of loads are on their way and " tail" where the depth is not taken in whole
 * stages of 64, so that a measurement or a test can say which kernel it ran.  MOE_EINVAL for which outside 0..5, a null name or
 * len == 0; else as the call that launches it. */
moe_status moe_gated_gemm_kernel(const moe_shape *s, int32_t which, char *name, size_t len);

/* ---- weights held as 4-bit codes -------------------------------------------------------------
 *
 *   w[n, k] = (code[n, k] - zero[n, k / group]) * scale[n, k / group]         y[r, n] = sum_k x[r, k] w[e][n, k]
 *
 *   q     uint8 [E, N, K / 2]: the code of k = 2 i in the low four bits of byte i, of 2 i + 1 in the high ones
 *   scale fp16 [E, N, K / group]
 *   zero  uint8 [E, N, K / group], or NULL: 8 throughout
 * group is 32, 64 or 128 and divides K.  Nothing is packed beforehand: the kernels read these as they are.
 */

/* R rows in all, of E experts (1..64) with matrices [N, K]; x: the rows' type, 1 bf16 or 2 fp16. */
typedef struct {
    int32_t R;
    int32_t E;
    int32_t N;
    int32_t K;
    int32_t group;
    int32_t x;
} moe_q4_shape;

/* y fp32 [R, N] = x [R, K] times the rows' expert's matrix; expert e owns rows [offsets[e], offsets[e+1]).
 * Codes and zeros enter the products exactly, scales and sums are fp32: of (code - zero) x for fp16 rows, of (16 + code) x less
 * (16 + zero) x for bf16 rows, whose values may be finite ones of any size (below about 2^-90 they lose digits).  A row with
 * an infinity or NaN has no finite output; the others are untouched. */
moe_status moe_q4_linear(const moe_q4_shape *s, const void *x, const int32_t *offsets, const void *q,
                         const void *scale, const void *zero, float *y, void *stream);

/* Host, pure.  Bytes of workspace of moe_gated_ffn_q4 (0 if unsupported). */
size_t moe_gated_q4_workspace_bytes(const moe_shape *s);

/* moe_gated_ffn of a MOE_BF16 layer with 4-bit weights: q13 [E, 2 d_ff, d_model / 2] (rows [0, d_ff) are Wg's
 * columns, [d_ff, 2 d_ff) Wu's), q2 [E, d_model, d_ff / 2], each with its scales and zeros; d_model and d_ff
 * multiples of group.  xe bf16, ye fp16 [rows, d_model]; the hidden activations are held in fp16. */
moe_status moe_gated_ffn_q4(const moe_shape *s, int32_t group, const void *xe, const int32_t *offsets,
                            const void *q13, const void *scale13, const void *zero13, const void *q2,
                            const void *scale2, const void *zero2, void *ye, void *workspace,
                            void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MOE_GATED_H */
