// What the gated block's translation units share (include/moe_gated.h).
#pragma once

#include "common.h"

namespace moe {

// Packed columns of the two first projections: sixteen of Wg and the same sixteen of Wu in turn.
inline int gated_packed_columns(int d_ff) { return (d_ff + 15) / 16 * 32; }

// In place of a work list: the experts' offsets, and the most rows there can be.
struct DirectTiles {
    const int32_t *offsets = nullptr;
    int E = 0;
    int64_t rows = 0;
};
// Kernels that take it: those of decode steps, and of fp32 layers.
inline bool takes_direct_tiles(const moe_shape &s, const GemmPlan &gp) { return s.dtype == MOE_F32 || (!gp.w4 && gp.bn == 64); }

// ffn.hip: C = H W2p (fp16 operands, bf16 layers; fp32 else), one work list, or, items NULL, direct tiles
moe_status launch_second_gemm(const moe_shape &s, const void *hidden, const void *W2p, void *ye, const GemmPlan &gp,
                              const WorkItem *items, const DirectTiles &direct, hipStream_t st);
// bwd.hip: dW[e] [M][N] = A[rows of e]^T B[rows of e] rounded to bf16; A holds fp16 values where a_f16
void launch_weight_grad_bf16(bool a_f16, const uint16_t *A, const uint16_t *B, uint16_t *C, const int32_t *offsets, int E,
                             int M, int N, int64_t max_rows, int stage, hipStream_t st);
// bwd.hip: whether that runs on 256 x 256 tiles, else on 128 x 128
bool wide_weight_grad_bf16(int E, int M, int N, int64_t max_rows);
// api.hip: the checks that every call makes of its shape
moe_status check_layer_shape(const moe_shape *s);
// api.hip: MOE_EUNSUPPORTED where the shape's activation is the gated block's alone; for the calls whose experts are two plain products
moe_status check_plain_activation(const moe_shape &s);

}  // namespace moe
