// A product of rows and weights in 8 bits: its arguments, and the launch of the kernel for large tiles.
#pragma once

#include "common.h"

namespace moe {

// K: pairs of codes, the "16-bit values" of the expert FFN's loops.  Tiles are found from the experts' offsets.
struct Q8Args {
    const uint16_t *x, *w;
    const float *xs, *ws, *bias;
    const void *r;
    void *y;
    const int32_t *offsets, *row_src;      // row_src: the first product takes row row_src[i] / row_div, of a_rows
    int row_div, a_rows;
    int E, N, K;                           // of a pair of projections N = 2 h
    int h;                                 // else 0
    int act, res, type;                    // act: a moe_act, of a linear map as activation_of has it
    int tiles, entries, share;
};

// The erf form of the GeLU under an fp32 output is an activation of its own.
enum { kGeluErf32 = 8 };
inline int activation_of(int act, bool y32) { return act == MOE_ACT_GELU_ERF && y32 ? kGeluErf32 : act; }

// q8_run.hip: tiles of 256 x 256; pair: the first projections, else the linear map, N a multiple of 4.
// whole: the depth is taken in whole stages of 64, four at least.
void launch_q8_run(bool pair, const Q8Args &a, int64_t entries, bool whole, int stage, hipStream_t st);

}  // namespace moe
