// Rows and weights held in 8 bits (include/moe_q8.h): rows to codes and back, one linear map, the gated feed-forward block,
// and the dispatch of such rows.
//
// Products are of 8-bit whole numbers on the matrix cores, with 32-bit sums: exact, so that no kernel, tile or split of the depth
// changes a sum.  (The 8-bit floating matrix instructions, of the same rate, drop what lies some 2^13 under the largest product
// of an instruction's group: 1.4e-5 of a sum of normally distributed values.)  An instruction takes twice the depth of a 16-bit one
// in the same bytes and cycles, so the loops are the expert FFN's with K in pairs of codes, "16-bit values", throughout.
// The block's hidden rows are rounded to fp16 by the first product's epilogue and held in 8 bits from a pass of their own, since
// a row's scale needs all of the row: 2 + 2 + 1 bytes a value beside the products.
#include "activation.h"
#include "moe_gated.h"
#include "moe_q8.h"
#include "gated.h"
#include "q8.h"
#include "q8_product.h"

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <type_traits>

#include <hip/hip_ext.h>

namespace moe {
namespace {

#include "q8_product_device.h"
#include "gemm_w4_run.h"

constexpr int kMaxDepth = 65536;             // values of a row

// ---------------------------------------------------------------- rows to codes and back
// 16 values of a row as they lie in memory
struct Sixteen {
    float v[16];
    __device__ __forceinline__ void load(const void *row, int type, int col)
    {
        if (type == kF32) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 p = *reinterpret_cast<const f32x4 *>(static_cast<const float *>(row) + col + 4 * q);
#pragma unroll
                for (int c = 0; c < 4; ++c) v[4 * q + c] = p[c];
            }
        } else {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const u32x4 p = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(row) + col + 8 * q);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    v[8 * q + 2 * c] = type == kB16 ? b16_of(p[c], 0) : f16_of(p[c], 0);
                    v[8 * q + 2 * c + 1] = type == kB16 ? b16_of(p[c], 1) : f16_of(p[c], 1);
                }
            }
        }
    }
};

// A row is TPR threads' (a wavefront's, or a block's), NV pieces of 16 values each, and stays in registers between the search for
// its largest magnitude and its codes: read once, written once, bound by memory (fp16 rows: 32768 of 2048 38 us, 5.3 TB/s; 32768 of 8192, a
// block's hidden rows, 126 us, 6.4 TB/s).  rows_end: NULL, or where the number of rows stands, at most R.
template <int TYPE, int TPR, int NV>
__global__ __launch_bounds__(TPR == kWave ? 256 : TPR) void q8_rows_kernel(const void *__restrict__ x, uint32_t *__restrict__ q,
                                                                           float *__restrict__ scale, int64_t R, int K,
                                                                           const int32_t *__restrict__ rows_end)
{
    constexpr int PER = TPR == kWave ? 4 : 1;          // rows of a block at a time
    const int t = threadIdx.x % TPR;
    if (rows_end != nullptr) R = min(R, static_cast<int64_t>(*rows_end));
    __shared__ uint32_t row_most[2][TPR / kWave];
    int turn = 0;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * PER + threadIdx.x / TPR; i < R; i += static_cast<int64_t>(gridDim.x) * PER) {
        const char *row = static_cast<const char *>(x) + i * K * (TYPE == kF32 ? 4 : 2);
        Sixteen p[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) p[v].load(row, TYPE, min((v * TPR + t) * 16, K - 16));
        uint32_t most = 0;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 16; ++e) most = max(most, magnitude(p[v].v[e]));      // (past the row's end: its last piece)
        most = wave_most(most);
        if constexpr (TPR > kWave) {
            if (lane_id() == 0) row_most[turn][threadIdx.x / kWave] = most;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < TPR / kWave; ++w) most = max(most, row_most[turn][w]);
            turn ^= 1;
        }
        const Q8Row held(most);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            int c[16];
            held.codes(p[v].v, c);
            const int col = (v * TPR + t) * 16;
            if (col < K)
                *reinterpret_cast<u32x4 *>(reinterpret_cast<char *>(q) + i * K + col) =
                    (u32x4){pack_codes(c), pack_codes(c + 4), pack_codes(c + 8), pack_codes(c + 12)};
        }
        if (t == 0) scale[i] = held.scale;
    }
}

// A block takes `rows` rows' pieces of 16 codes, whichever row they are of.  Bound by memory: 32768 rows of 2048 to fp16, 0.2 GB, 30.6 us,
// 6.6 TB/s.
template <int TYPE>
__global__ __launch_bounds__(256) void q8_values_kernel(const uint32_t *__restrict__ q, const float *__restrict__ scale, void *__restrict__ x,
                                                        int64_t R, int K, int rows)
{
    const int64_t step = static_cast<int64_t>(gridDim.x) * rows;
    for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * rows; r0 < R; r0 += step) {
        const int per_row = K / 16, pieces = static_cast<int>(min(R - r0, static_cast<int64_t>(rows))) * per_row;
        for (int p = threadIdx.x; p < pieces; p += 256) {
            const int64_t at = r0 * per_row + p;
            const u32x4 c = *(reinterpret_cast<const u32x4 *>(q) + at);
            const float s = scale[r0 + p / per_row];
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = static_cast<float>(static_cast<int8_t>(c[i / 4] >> (i % 4 * 8))) * s;
            if constexpr (TYPE == kF32) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *(reinterpret_cast<f32x4 *>(x) + at * 4 + i) = (f32x4){v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    u32x4 o;
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = pack_16(TYPE, v[8 * i + 2 * e], v[8 * i + 2 * e + 1]);
                    *(reinterpret_cast<u32x4 *>(x) + at * 2 + i) = o;
                }
            }
        }
    }
}

// ---------------------------------------------------------------- few rows per expert
// Bound by the weights' arrival.  A wavefront multiplies tiles of 16 columns (of a pair 16 of each) and at most 32 rows in stages of 128 codes,
// which go through LDS of its own, PD of them on their way, so that nothing is waited for but its own loads.  PD is small, 2 or 3: what is on
// its way comes from many wavefronts on a unit, and each stage more takes LDS from them (4 and 5 were slower).  Where tiles are few, a block's
// four wavefronts share out the stages of one tile (SPLIT), and the whole numbers are added up through LDS at the end; else each has a tile, four side by
// side.  Measured, kernel alone: 1 row, 4096 x 4096, 5.2 us (the latency of a launch and two round trips); 32 rows, 6144 x 4096, 8.3 us, 3.0 TB/s;
// a block's projections for 64 rows of 8 experts, 4096 to 2 x 14336, 137 us, 6.9 TB/s, and back 74 us, 6.3 TB/s; for 2 rows 35 us,
// 6.7 TB/s, and back 20.7, 5.7 TB/s.  Reading alone reaches 7.1 TB/s in 2 GB and 6.3 in 128 MB.
template <bool PAIR, int RT, int PD, bool ONCE, bool SPLIT>
__global__ __launch_bounds__(256) void q8_stream_kernel(Q8Args a)
{
    constexpr int NT = PAIR ? 2 : 1, WAVES = 4, STAGE = (NT + RT) * 2048, LOADS = (NT + RT) * 2;
    const Tiles<16 * RT, (SPLIT ? 16 : 64) * NT> tiles(a.offsets, a.E, a.tiles);
    WorkItem item = tiles[blockIdx.x];
    if (item.expert < 0) return;
    extern __shared__ __attribute__((aligned(16))) char q8_lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 15, oct = lane >> 4;
    if constexpr (!SPLIT) {
        item.n0 += wave * (16 * NT);
        if (item.n0 / NT >= (PAIR ? a.h : a.N)) return;         // (no wavefront waits for another)
    }
    char *const mine = q8_lds + wave * (STAGE * PD);
    const uint32_t dest = lds_address(mine);
    const int rows = item.row1 - item.row0, n0 = item.n0 / NT, width = PAIR ? a.h : a.N;
    const unsigned pitch = static_cast<unsigned>(a.K) * 2u;
    const uint16_t *w0 = a.w + (static_cast<size_t>(item.expert) * a.N + n0) * a.K;
    __amdgpu_buffer_rsrc_t rsw[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
        rsw[t] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(w0 + static_cast<size_t>(t) * a.h * a.K), 0,
                                                   static_cast<unsigned>(min(width - n0, 16)) * pitch, 0x00020000);
    const bool gather = PAIR && a.row_src != nullptr;
    const __amdgpu_buffer_rsrc_t rsx = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t *>(gather ? a.x : a.x + static_cast<size_t>(item.row0) * a.K), 0,
        static_cast<unsigned>(gather ? a.a_rows : rows) * pitch, 0x00020000);
    // a load: eight rows of 128 bytes; lane l lands at row l / 8, place l % 8, where piece place ^ (row / 2 % 8) belongs
    int wsrc[2], xsrc[2 * RT], piece[2];
#pragma unroll
    for (int q = 0; q < 2 * RT; ++q) {
        const int r = q * 8 + (lane >> 3);
        if (q < 2) {
            piece[q] = (lane & 7) ^ ((r >> 1) & 7);
            wsrc[q] = static_cast<int>(r * pitch) + piece[q] * 16;
        }
        const int from = gather ? a.row_src[min(item.row0 + r, item.row1 - 1)] / a.row_div : r;
        xsrc[q] = r < rows ? static_cast<int>(from * pitch) + piece[q & 1] * 16 : 0x7ffffff0;
    }
    const int KT = (a.K + 63) / 64, per = SPLIT ? (KT + WAVES - 1) / WAVES : KT;
    const int s0 = SPLIT ? min(wave * per, KT) : 0, s1 = min(s0 + per, KT);
    // Every block begins elsewhere in its stages: whole numbers' sums are exact in any order, rows of weights are often a power of two bytes
    // apart, and blocks that walk them in step ask few of the memory channels at a time (1 row, 4096 x 4096: 8.1 -> 5.9 us a pass).
    const int turn = __builtin_amdgcn_readfirstlane(s1 > s0 ? static_cast<int>(blockIdx.x * 5u % static_cast<unsigned>(s1 - s0)) : 0);
    // (a piece past the row's end: an offset past every resource reads as zeros)
    auto load = [&](int s, int place) {
        const uint32_t at = dest + place * STAGE;
        const int k = (s + turn < s1 ? s + turn : s + turn - (s1 - s0)) * 128;
        const bool past0 = s >= s1 || k + piece[0] * 16 >= static_cast<int>(pitch), past1 = s >= s1 || k + piece[1] * 16 >= static_cast<int>(pitch);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            load_to_lds_as<ONCE>(rsw[t], past0 ? 0x7ffffff0 : wsrc[0], at + t * 2048, k);
            load_to_lds_as<ONCE>(rsw[t], past1 ? 0x7ffffff0 : wsrc[1], at + t * 2048 + 1024, k);
        }
#pragma unroll
        for (int q = 0; q < 2 * RT; ++q)
            load_to_lds(rsx, (q & 1 ? past1 : past0) ? 0x7ffffff0 : xsrc[q], at + NT * 2048 + q * 1024, k);
    };
    i32x4 acc[NT][RT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[t][j] = (i32x4){0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < PD; ++p) load(s0 + p, p);
    int place = 0;
    for (int s = s0; s < s1; ++s) {
        MOE_VMCNT((PD - 1) * LOADS);
        lds_handover();
        const char *at = mine + place * STAGE;
        u32x4 w[NT][2], x[RT][2];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int f = fr * 128 + (((p * 4 + oct) ^ ((fr >> 1) & 7)) << 4);
#pragma unroll
            for (int t = 0; t < NT; ++t) w[t][p] = *reinterpret_cast<const u32x4 *>(at + t * 2048 + f);
#pragma unroll
            for (int j = 0; j < RT; ++j) x[j][p] = *reinterpret_cast<const u32x4 *>(at + NT * 2048 + j * 2048 + f);
        }
        MOE_LGKM0();
        lds_handover();
        load(s + PD, place);
        place = place == PD - 1 ? 0 : place + 1;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < RT; ++j)
                    acc[t][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, w[t][p]), __builtin_bit_cast(i32x4, x[j][p]),
                                                                     acc[t][j], 0, 0, 0);
    }
    MOE_VMCNT(0);
    MOE_MATRIX_RESULTS();
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < RT; ++j) asm volatile("" : "+v"(acc[t][j]));
    if constexpr (SPLIT) {
        // sums of the wavefronts: [wave][tile][lane] of four numbers
        __syncthreads();
        i32x4 *const sums = reinterpret_cast<i32x4 *>(q8_lds);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < RT; ++j) sums[((j * NT + t) * WAVES + wave) * 64 + lane] = acc[t][j];
        __syncthreads();
        if (wave >= RT) return;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            i32x4 s = sums[(wave * NT + t) * WAVES * 64 + lane];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s += sums[((wave * NT + t) * WAVES + w) * 64 + lane];
            acc[t][0] = s;
        }
    }
#pragma unroll
    for (int jj = 0; jj < (SPLIT ? 1 : RT); ++jj) {
        const int j = SPLIT ? wave : jj, row = j * 16 + fr, n = n0 + oct * 4;
        if (row >= rows || n >= width) continue;
        float v[NT][4];
        const float xs = row_scale(a, item.row0 + row);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const i32x4 s = acc[t][jj];
            float cs[4];
            column_scales(a.ws + static_cast<size_t>(item.expert) * a.N + t * a.h, n, width, cs);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float in = static_cast<float>(s[c]) * xs;
                if constexpr (PAIR) v[t][c] = in * cs[c];
                else v[t][c] = __builtin_fmaf(in, cs[c], a.bias != nullptr ? a.bias[static_cast<size_t>(item.expert) * a.N + min(n + c, a.N - 1)] : 0.0f);
            }
        }
        const size_t at = static_cast<size_t>(item.row0 + row);
        const ActForm form(a.act);
        auto activated = [&](auto act) {
#pragma unroll
            for (int c = 0; c < 4; ++c) v[0][c] = activate<decltype(act)::value>(form, v[0][c]) * (PAIR ? v[NT - 1][c] : 1.0f);
        };
        if constexpr (PAIR) with_activation<MOE_ACT_GELU_ERF, MOE_ACT_SILU>(a.act, activated);
        else with_activation<MOE_ACT_GELU_ERF, kGeluErf32, MOE_ACT_IDENTITY>(a.act, activated);
        if constexpr (PAIR) {
            store_hidden(a, at, n, v[0]);
        } else if (a.N % 4 == 0) {
            const WayOut<4> out(a, item.row0, item.row1, n);
            typename WayOut<4>::Residual r;
            out.ask(row, r);
#pragma unroll
            for (int c = 0; c < 4; ++c) v[0][c] += out.value(r, c);
            out.leave(row, v[0]);
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const WayOut<1> out(a, item.row0, item.row1, n + c);
                typename WayOut<1>::Residual r;
                out.ask(row, r);
                const float u[1] = {v[0][c] + out.value(r, 0)};
                out.leave(row, u);
            }
        }
    }
}

// ---------------------------------------------------------------- tiles of 128 x 128, one for a block
// Some rows and a long depth: five stages on their way, one block to a compute unit, bound by the weights' arrival, or where tiles are fewer than
// units by a tile's chain of stages, 0.4 to 0.5 us each.  Sums leave through LDS, so that y and r are met in whole lines of a row.
// Measured, kernel alone: 64 rows, 32000 x 4096, fp32 out, 27 us, 5.2 TB/s; 1003 uneven rows of 5 experts, 1999 x 1008, silu, bias and an fp32
// residual, 17 us; of 2000 columns 15.6.
template <bool PAIR, bool KTAIL, bool ONCE>
__global__ __launch_bounds__(256, 1) void q8_tile_kernel(Q8Args a)
{
    constexpr int BM = 128, BN = 128;
    constexpr bool DEEP = true;
    constexpr int F16 = kI8Operands;
    constexpr bool TILE_IN = false, TILE_PAIR = false, W_PAIR = PAIR, W_ONCE = ONCE;
    constexpr int tile_pitch = 0, pair_at = 0;
    const uint16_t *const tile_in = nullptr;
    const uint16_t *const A = a.x, *const W = a.w;
    const int N = a.N, K = a.K, pair_h = a.h, row_div = a.row_div, a_rows = a.a_rows;
    const int32_t *const row_src = PAIR ? a.row_src : nullptr;
    const Tiles<BM, BN> items(a.offsets, a.E, a.tiles);
    // scales and biases are on their way through the stages
    const WorkItem mine = items[blockIdx.x];
    if (mine.expert < 0) return;
    constexpr int TM_ = BM / 32;
    const int l = lane_id(), wm_ = threadIdx.x / kWave & 1, wn_ = __builtin_amdgcn_readfirstlane(threadIdx.x / (2 * kWave));
    int source[TM_];
    float xs[TM_];
#pragma unroll
    for (int j = 0; j < TM_; ++j) {
        source[j] = min(mine.row0 + wm_ * 64 + j * 16 + (l & 15), mine.row1 - 1);
        if (row_src != nullptr) source[j] = row_src[source[j]];
        else xs[j] = a.xs[source[j]];
    }
    // a lane's columns on the way out: four of the wavefront's 64 (of a pair too), as far as rows begin at whole dwords and no four lie across a
    // row's end; else one (1003 uneven rows of 5 experts, 1999 x 1008, silu, bias and an fp32 residual: one a lane everywhere 19.2 us a pass, so 16.8)
    const bool dwords = N % 2 == 0 || (a.type == kF32 && (a.r == nullptr || a.res == kF32));
    const bool fours = PAIR || N % 4 == 0 || (dwords && mine.n0 + wn_ * 64 + 64 <= N);
    const int col = PAIR ? l % 8 * 4 : fours ? l % 16 * 4 : l, width = PAIR ? pair_h : N;
    const int n = PAIR ? mine.n0 / 2 + wn_ * 32 + col : mine.n0 + wn_ * 64 + col;
    const float *const ws = a.ws + static_cast<size_t>(mine.expert) * N;
    const float *const other = PAIR ? ws + pair_h : a.bias != nullptr ? a.bias + static_cast<size_t>(mine.expert) * N : nullptr;
    float cs[4], cb[4] = {0.0f, 0.0f, 0.0f, 0.0f};       // (cb: of a pair the second's scales)
    column_scales(ws, n, width, cs);
    if (other != nullptr) column_scales(other, n, width, cb);
#include "gemm_w4_body.inc"

    // the wavefront's 64 rows of 64 columns (of a pair 32 of each), 32 bytes of row padding
    constexpr int PITCH = 256 + 32;
    char *const patch = lds + wave * 64 * PITCH;
    if (row_src != nullptr) {
#pragma unroll
        for (int j = 0; j < TM; ++j) xs[j] = a.xs[source[j] / row_div];
    }
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            f32x4 v;
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = sum_of(acc[i][j][c]) * xs[j];
            *reinterpret_cast<f32x4 *>(patch + (j * 16 + fr) * PITCH + (i * 16 + oct * 4) * 4) = v;
        }
    lds_handover();
    const ActForm form(a.act);
    // sixteen rows' residuals are on their way together
    auto leave_sums = [&](auto perc, auto actc) {
        constexpr int PER = decltype(perc)::value, ROWS = PER;
        const WayOut<PER> out(a, item.row0 + wm * 64, item.row1, n);
        typename WayOut<PER>::Residual r[16 / ROWS];
#pragma unroll 1
        for (int row0 = 0; row0 < 64; row0 += 16) {
            const int in = PER == 4 ? lane / 16 : 0;
#pragma unroll
            for (int it = 0; it < 16 / ROWS; ++it) out.ask(row0 + it * ROWS + in, r[it]);
#pragma unroll
            for (int it = 0; it < 16 / ROWS; ++it) {
                const char *const at = patch + (row0 + it * ROWS + in) * PITCH + col * 4;
                float v[PER];
                if constexpr (PER == 4) {
                    const f32x4 s = *reinterpret_cast<const f32x4 *>(at);
#pragma unroll
                    for (int c = 0; c < 4; ++c) v[c] = s[c];
                } else {
                    v[0] = *reinterpret_cast<const float *>(at);
                }
#pragma unroll
                for (int c = 0; c < PER; ++c)
                    v[c] = activate<decltype(actc)::value>(form, __builtin_fmaf(v[c], cs[c], cb[c])) + out.value(r[it], c);
                out.leave(row0 + it * ROWS + in, v);
            }
        }
    };
    const int left = rows - wm * 64;                      // of the wavefront's rows
    const size_t row0 = static_cast<size_t>(item.row0) + wm * 64;
    auto way = [&](auto actc) {
        constexpr int ACT = decltype(actc)::value;
        if constexpr (PAIR) {
            const int at = col / 16 * 32 + col % 16;
            if (n >= width) return;
#pragma unroll
            for (int it = 0; it < 8; ++it) {
                const int row = it * 8 + lane / 8;
                const f32x4 g = *reinterpret_cast<const f32x4 *>(patch + row * PITCH + at * 4);
                const f32x4 u = *reinterpret_cast<const f32x4 *>(patch + row * PITCH + at * 4 + 64);
                float v[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] = activate<ACT>(form, g[c] * cs[c]) * (u[c] * cb[c]);
                if (row < left) store_hidden(a, row0 + row, n, v);
            }
        } else if (fours) {
            leave_sums(std::integral_constant<int, 4>{}, actc);
        } else {
            leave_sums(std::integral_constant<int, 1>{}, actc);
        }
    };
    if constexpr (PAIR) with_activation<MOE_ACT_GELU_ERF, MOE_ACT_SILU>(a.act, way);
    else with_activation<MOE_ACT_GELU_ERF, kGeluErf32, MOE_ACT_SILU, MOE_ACT_IDENTITY>(a.act, way);
}

// ---------------------------------------------------------------- tiles of 128 x 128, a share of them for a block
// As the kernels of q8_run.hip, two blocks to a compute unit: products of a few hundred tiles, and of a short depth, whose tiles are mostly
// beginnings and ends.  Each operand's byte is multiplied half as often as in a 256 x 256 tile; a stage takes 1.0 us for the unit's two tiles, there
// 1.3 for one of four times the area.  Measured, kernel alone: 8192 rows of 16 experts, 768 x 2048, 23 us, 1.12 POP/s
// (6000 uneven rows of the same 25.0 us, in tiles of 256 x 256 30.8); 6002 uneven rows of 13 experts, 1008 x 2608, 34 us.
// WHOLE: N is a multiple of four, and a lane takes four columns of a row on the way out; else one, of 64.
template <bool WHOLE, bool KTAIL, bool ONCE>
__global__ __launch_bounds__(256, 2) void q8_small_run_kernel(Q8Args a)
{
    constexpr int BM = 128, BN = 128, TM = 4;
    const Tiles<BM, BN> items(a.offsets, a.E, a.tiles);
    const ActForm form(a.act);
    struct Columns {
        float xs[TM];
        float ws[4], bias[4];
    };
    w4_run<kI8Operands, KTAIL, BM, 0, false, BN, ONCE>(a.x, a.w, items, nullptr, a.entries, a.share, a.N, a.K, nullptr, 1, 0,
        [&](const WorkItem &item, int wn, int) {
            Columns c;
            const int lane = lane_id(), wm = threadIdx.x / kWave & 1;
#pragma unroll
            for (int j = 0; j < TM; ++j) c.xs[j] = a.xs[min(item.row0 + wm * (BM / 2) + j * 16 + (lane & 15), item.row1 - 1)];
            const size_t first = static_cast<size_t>(item.expert) * a.N;
            const int n = item.n0 + wn * 64 + (WHOLE ? lane % 16 * 4 : lane);
#pragma unroll
            for (int e = 0; e < 4; ++e) c.bias[e] = 0.0f;
            column_scales(a.ws + first, n, a.N, c.ws);
            if (a.bias != nullptr) column_scales(a.bias + first, n, a.N, c.bias);
            return c;
        },
        [&](auto &acc, const Columns &ahead, const WorkItem &item, const W4Place<BM, BN> &place, auto landed) {
            const int lane = place.lane;
            constexpr int PER = WHOLE ? 4 : 1, ROWS = PER;      // columns of a lane, rows of a step
            const WayOut<PER> out(a, item.row0 + place.wm * (BM / 2), item.row1, item.n0 + place.wn * 64 + (WHOLE ? lane % 16 * 4 : lane));
            const int in = WHOLE ? lane / 16 : 0;
            // (sixteen rows' residuals are on their way from the step before, of single columns, which are more, from the step's start)
            constexpr int TURNS = WHOLE ? 2 : 1;
            typename WayOut<PER>::Residual r[TURNS][16 / ROWS];
            auto ask = [&](int j) {
#pragma unroll
                for (int it = 0; it < 16 / ROWS; ++it) out.ask(j * 16 + it * ROWS + in, r[j % TURNS][it]);
            };
            if constexpr (WHOLE) ask(0);
            static_for<TM>([&](auto jc) {
                constexpr int j = decltype(jc)::value;
                lds_handover();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x4 v;
#pragma unroll
                    for (int c = 0; c < 4; ++c) v[c] = sum_of(acc[i][j][c]) * ahead.xs[j];
                    // (a row's 16-byte pieces XOR-swizzled with the row)
                    *reinterpret_cast<f32x4 *>(place.patch + place.fr * 256 + (((i * 4 + place.oct) ^ place.fr) << 4)) = v;
                }
                MOE_SB();
                if constexpr (j == 0) landed();
                if constexpr (!WHOLE) ask(j);
                else if constexpr (j + 1 < TM) ask(j + 1);
                lds_handover();
                MOE_SB();
                with_activation<MOE_ACT_GELU_ERF, kGeluErf32, MOE_ACT_IDENTITY>(a.act, [&](auto act) {
#pragma unroll
                    for (int it = 0; it < 16 / ROWS; ++it) {
                        const int row = it * ROWS + in;
                        float v[PER];
                        if constexpr (WHOLE) {
                            const f32x4 s = *reinterpret_cast<const f32x4 *>(place.patch + row * 256 + ((lane % 16 ^ row) << 4));
#pragma unroll
                            for (int c = 0; c < 4; ++c) v[c] = s[c];
                        } else {
                            v[0] = *reinterpret_cast<const float *>(place.patch + row * 256 + ((lane / 4 ^ row) << 4) + lane % 4 * 4);
                        }
#pragma unroll
                        for (int c = 0; c < PER; ++c)
                            v[c] = activate<decltype(act)::value>(form, __builtin_fmaf(v[c], ahead.ws[c], ahead.bias[c])) + out.value(r[j % TURNS][it], c);
                        out.leave(j * 16 + row, v);
                    }
                });
            });
        });
}

// The block's first projections.
template <bool KTAIL, bool ONCE>
__global__ __launch_bounds__(256, 2) void q8_gated_small_run_kernel(Q8Args a)
{
    constexpr int BM = 128, BN = 128, TM = 4;
    const Tiles<BM, BN> items(a.offsets, a.E, a.tiles);
    const ActForm form(a.act);
    struct Scales {
        float xs[TM];
        float gs[2][4], us[2][4];
    };
    w4_run<kI8Operands, KTAIL, BM, 0, true, BN, ONCE>(a.x, a.w, items, nullptr, a.entries, a.share, a.N, a.K, a.row_src, a.row_div, a.a_rows,
        [&](const WorkItem &item, int wn, int oct) {
            Scales c;
            const int lane = lane_id(), wm = threadIdx.x / kWave & 1;
            int from[TM];
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                from[j] = min(item.row0 + wm * (BM / 2) + j * 16 + (lane & 15), item.row1 - 1);
                if (a.row_src != nullptr) from[j] = a.row_src[from[j]];
            }
#pragma unroll
            for (int j = 0; j < TM; ++j) c.xs[j] = a.xs[a.row_src != nullptr ? from[j] / a.row_div : from[j]];
            const float *gs = a.ws + static_cast<size_t>(item.expert) * a.N;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int n = min(item.n0 / 2 + wn * 32 + p * 16 + oct * 4, a.h - 4);      // (h is a multiple of 16)
                const f32x4 g = *reinterpret_cast<const f32x4 *>(gs + n), u = *reinterpret_cast<const f32x4 *>(gs + a.h + n);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    c.gs[p][e] = g[e];
                    c.us[p][e] = u[e];
                }
            }
            return c;
        },
        [&](auto &acc, const Scales &ahead, const WorkItem &item, const W4Place<BM, BN> &place, auto landed) {
            const int lane = place.lane, row0 = item.row0 + place.wm * (BM / 2), left = item.row1 - row0;
            const int col = item.n0 / 2 + place.wn * 32 + lane % 4 * 8;
            static_for<TM>([&](auto jc) {
                constexpr int j = decltype(jc)::value;
                lds_handover();
                with_activation<MOE_ACT_GELU_ERF, MOE_ACT_SILU>(a.act, [&](auto act) {
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        f16x4 o;
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const float g = sum_of(acc[2 * p][j][c]) * ahead.xs[j] * ahead.gs[p][c];
                            const float u = sum_of(acc[2 * p + 1][j][c]) * ahead.xs[j] * ahead.us[p][c];
                            o[c] = to_f16(activate<decltype(act)::value>(form, g) * u);
                        }
                        *reinterpret_cast<f16x4 *>(place.at(p, 0)) = o;
                    }
                });
                MOE_SB();
                if constexpr (j == 0) landed();
                lds_handover();
                MOE_SB();
                // 16 rows of 32 columns, four lanes to a row
                const int row = lane / 4;
                const u32x4 q = *reinterpret_cast<const u32x4 *>(place.patch + row * 256 + ((lane % 4 ^ row) << 4));
                if (j * 16 + row < left && col < a.h)
                    *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.y) + static_cast<size_t>(row0 + j * 16 + row) * a.h + col) = q;
            });
        },
        a.h);
}

// ---------------------------------------------------------------- dispatch
// codes and scales of the tokens to their slots; a wavefront owns a token, whose codes are read once however many slots it has.  Bound by memory:
// 32768 tokens of 2048 to two of 32 experts each, 0.2 GB, take the dispatch from 10.1 to 41.4 us, 6.4 TB/s; 64 of 4096 from 9.6 to 12.9, a launch.
__global__ __launch_bounds__(256) void q8_scatter_kernel(const u32x4 *__restrict__ x, const float *__restrict__ xs,
                                                         const int32_t *__restrict__ slot_of, u32x4 *__restrict__ xe,
                                                         float *__restrict__ xes, int T, int k, int vec, int max_rows)
{
    const int lane = lane_id();
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / kWave; t < T; t += static_cast<int64_t>(gridDim.x) * 4) {
        int slot = lane < k ? slot_of[t * k + lane] : -1;
        if (slot >= max_rows) slot = -1;
        if (slot >= 0) xes[slot] = xs[t];
        for (int c = lane; c - lane < vec; c += kWave) {
            const u32x4 v = x[t * vec + min(c, vec - 1)];
            for (int j = 0; j < k; ++j) {
                const int to = __shfl(slot, j);
                if (to >= 0 && c < vec) xe[static_cast<size_t>(to) * vec + c] = v;
            }
        }
    }
}

// ---------------------------------------------------------------- host side
void launch_rows(int64_t R, int K, int type, const void *x, void *q, float *scale, const int32_t *rows_end, hipStream_t st)
{
    using std::integral_constant;
    auto with_type = [&](auto ty) {
        auto launch = [&](auto tpr, auto nv) {
            constexpr int TPR = decltype(tpr)::value, PER = TPR == kWave ? 4 : 1;
            const unsigned grid = static_cast<unsigned>(std::min<int64_t>((R + PER - 1) / PER, 1 << 20));
            hipLaunchKernelGGL((q8_rows_kernel<decltype(ty)::value, TPR, decltype(nv)::value>), dim3(grid), dim3(TPR == kWave ? 256 : TPR),
                               0, st, x, static_cast<uint32_t *>(q), scale, R, K, rows_end);
        };
        // Many rows: a wavefront each, without a barrier, as far as its registers go (fp16, K = 2048, 2048 / 8192 / 32768 rows 6.5 / 12.9 /
        // 38 us, by blocks of 256 threads 6.9 / 17 / 57; three pieces a lane, 6002 rows of 2608, 15.6 where the blocks take 14).
        if (R >= 2048 && K > 1024 && K <= 2048) launch(integral_constant<int, 64>{}, integral_constant<int, 2>{});
        else if (K <= 1024) launch(integral_constant<int, 64>{}, integral_constant<int, 1>{});
        else if (K <= 4096) launch(integral_constant<int, 256>{}, integral_constant<int, 1>{});
        else if (K <= 8192) launch(integral_constant<int, 256>{}, integral_constant<int, 2>{});
        else if (K <= 16384) launch(integral_constant<int, 512>{}, integral_constant<int, 2>{});
        else launch(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    };
    if (type == kF32) with_type(integral_constant<int, kF32>{});
    else if (type == kB16) with_type(integral_constant<int, kB16>{});
    else with_type(integral_constant<int, kF16>{});
}

// The kernel of a product of `rows` rows of E experts, by what each would take, us: the weights' arrival, the bytes that pass through LDS, and the
// rounds of tiles with their stages, whichever is longest.  The numbers are fitted to sweeps of the kernels over 111 products (1 to 16384 rows, 1
// to 64 experts, 768 to 32000 columns, depths of 512 to 14336; profiles/eight_bit_product_kernels_sweep.txt): the kernel chosen takes 1.024 times the
// fastest one's time on average and more than 1.1 times in six.  The worst are 1.45 and 1.47, where uneven experts of some 96 rows get tiles of
// 256 x 256: one row tile is counted for each, 256 tiles in a round, and an expert of more than 256 rows makes it two (1536 rows of 16 experts,
// 768 to 4096 columns, 38.1 us, in 128 x 128 26.3).
struct Q8Plan {
    int bm, bn;                            // tile; bm 16 or 32: the kernel for few rows
    bool deep, split;
};
Q8Plan plan_product(int64_t rows, int E, int columns, int K)
{
    const double depth = 2.0 * K, stages = (K + 63) / 64, used = E * (1.0 - std::pow(1.0 - 1.0 / E, static_cast<double>(rows)));
    const double weights = used * columns * depth;                      // bytes
    // tiles of bm rows: one of every expert while they are a good deal emptier than a tile, else half of one too many
    auto few = [&](int bm) { return rows * 8 <= static_cast<int64_t>(bm) * E * 3; };
    auto row_tiles = [&](int bm) {
        if (E == 1) return static_cast<double>((rows + bm - 1) / bm);
        return few(bm) ? used : std::max(used, static_cast<double>(rows) / bm + E / 2.0);
    };
    // how often `tiles` go round a chip that holds at_once of them (many: the shares even out)
    auto rounds = [](double tiles, double at_once) { return tiles > 3.0 * at_once ? tiles / at_once : std::ceil(tiles / at_once); };
    Q8Plan best{0, 0, false, false};
    double least = 1e30;
    auto offer = [&](double us, Q8Plan p) {
        if (us < least) {
            least = us;
            best = p;
        }
    };
    for (int bm : {16, 32}) {
        const double groups = row_tiles(bm) * ((columns + 15) / 16), bytes = groups * (16 + bm) * depth;
        // (few blocks of four tiles side by side: the stages of a unit that has one, two or three of them)
        const double side = groups / 4 <= 768 ? std::ceil(groups / 4 / 256) : 0.0;
        const double stage = bm == 16 ? std::max(0.33, 0.28 * side) : std::max(0.42, 0.39 * side);
        offer(4.0 + std::max({weights / 6.0e6, bytes / 14.5e6, groups / 768 * 4.5, 0.42 / 4 * stages}), {bm, 0, false, true});
        offer(4.0 + std::max({weights / 6.9e6, bytes / 19.5e6, groups / 768 / 4 * (2.5 + 0.7 * stages), stage * stages}), {bm, 0, false, false});
    }
    const double t128 = row_tiles(128) * ((columns + 127) / 128), t256 = row_tiles(256) * ((columns + 255) / 256);
    const double deep = (E == 1 || few(128) ? row_tiles(128) : static_cast<double>(rows) / 128 + E) * ((columns + 127) / 128);
    if (K >= 320) offer(std::max(6.0 + weights / 6.4e6, deep <= 256 ? 6.0 + 0.45 * stages : rounds(deep, 256) * (9.0 + 0.5 * stages)), {128, 128, true, false});
    offer(std::max(6.0 + weights / 6e6, t128 <= 256 ? 8.0 + 0.42 * stages : 3.0 + rounds(t128, 512) * (8.0 + stages)), {128, 128, false, false});
    offer(std::max(6.0 + weights / 6e6, 4.0 + rounds(t256, 256) * (8.0 + 1.3 * stages)), {256, 256, false, false});
    return best;
}

// How a product is launched.  once: weights that one tile of rows reads, and more of them (of all experts, whichever have rows) than 64 MiB, a quarter of
// the last level of cache, go past the caches.  us kept / past, with 1.2 GB of other weights between two calls and, in brackets, of the same
// weights again: 1 row, 34 MB 10.1 / 9.2 (6.5 / 6.7), 67 MB 15.1 / 13.3 (12.6 / 11.7), 134 MB 27.3 / 24.6 (21.0 / 21.7); 64 rows, 50 MB 24.3 / 23.3
// (19.8 / 21.8), 67 MB 25.9 / 23.9 (20.4 / 22.8), 134 MB 31.5 / 28.0 (26.4 / 27.1).  So below the line what a program's next call may find again stays.
constexpr int64_t kKeptBytes = 64 << 20, kMostTiles = 1 << 23;
struct Q8Launch {
    Q8Plan plan;
    int tiles;
    int64_t entries;
    bool once, whole;                      // whole: the form that takes the depth in whole stages, without a tail
};
Q8Launch plan_launch(bool pair, int64_t rows, int E, int N, int K, int h)
{
    Q8Launch l;
    const int columns = pair ? gated_packed_columns(h) : N;
    auto tile = [&] {
        const int bn = l.plan.bm <= 32 ? (pair ? 2 : 1) * (l.plan.split ? 16 : 64) : l.plan.bn;
        l.tiles = (columns + bn - 1) / bn;
        l.entries = tile_entries(rows, E, l.plan.bm, l.tiles);
    };
    l.plan = plan_product(rows, E, columns, K);
    if (!pair && l.plan.bn == 256 && N % 4 != 0) l.plan = {128, 128, false, false};
    tile();
    if (l.entries >= kMostTiles && l.plan.bn != 256) {          // (a block for every tile would be too many)
        l.plan = {128, 128, false, false};
        tile();
    }
    // (tiles of 32 rows that share out their depth are for fewer weights)
    l.once = rows <= static_cast<int64_t>(l.plan.bm) * E && 2ll * E * N * K > kKeptBytes && !(l.plan.bm == 32 && l.plan.split);
    // those whose loads run on from tile to tile need four stages
    l.whole = K % 64 == 0 && (l.plan.bm <= 32 || l.plan.deep || K >= 256);
    return l;
}
void product_kernel_name(bool pair, const Q8Launch &l, char *name, size_t len)
{
    const Q8Plan &p = l.plan;
    const bool few = p.bm <= 32;
    const char *kernel = few ? "q8_stream_kernel" : p.deep ? "q8_tile_kernel" : p.bn == 128 ? (pair ? "q8_gated_small_run_kernel" : "q8_small_run_kernel")
                                                                                 : (pair ? "q8_gated_run_kernel" : "q8_run_kernel");
    std::snprintf(name, len, "%s %dx%d%s%s%s%s", kernel, p.bm, few ? (pair ? 32 : 16) : p.bn, few && p.split ? " split" : "", p.deep ? " deep" : "",
                  l.once && p.bn != 256 ? " once" : "", l.whole || few ? "" : " tail");
}

template <bool PAIR>
void launch_product(Q8Args a, int64_t rows, int stage, hipStream_t st)
{
    const Q8Launch l = plan_launch(PAIR, rows, a.E, a.N, a.K, a.h);
    a.tiles = l.tiles;
    a.entries = static_cast<int>(l.entries);
    if (l.plan.bm <= 32) {
        using std::integral_constant;
        auto stream = [&](auto rt, auto once, auto split) {
            constexpr int RT = decltype(rt)::value, PD = PAIR ? 2 : RT == 1 ? 3 : 2;
            launch_product_kernel<q8_stream_kernel<PAIR, RT, PD, decltype(once)::value, decltype(split)::value>>(
                a, l.entries, static_cast<size_t>(4) * PD * ((PAIR ? 2 : 1) + RT) * 2048, stage, st);
        };
        const integral_constant<int, 1> sixteen;
        const integral_constant<int, 2> thirty_two;
        const std::true_type yes;
        const std::false_type no;
        if (l.plan.bm == 16 && l.plan.split) l.once ? stream(sixteen, yes, yes) : stream(sixteen, no, yes);
        else if (l.plan.bm == 16) l.once ? stream(sixteen, yes, no) : stream(sixteen, no, no);
        else if (l.plan.split) stream(thirty_two, no, yes);
        else l.once ? stream(thirty_two, yes, no) : stream(thirty_two, no, no);
        return;
    }
    if (l.plan.bn == 256) return launch_q8_run(PAIR, a, l.entries, l.whole, stage, st);
    auto launch = [&](auto tail, auto oncec) {
        constexpr bool TAIL = decltype(tail)::value, ONCE = decltype(oncec)::value;
        if (l.plan.deep) {
            launch_product_kernel<q8_tile_kernel<PAIR, TAIL, ONCE>>(a, l.entries, kW4Lds, stage, st);
            return;
        }
        constexpr int units = 2 * kRunUnits;
        a.share = std::max(1, std::min(w4_run_share(128, a.K), parts_of(a.entries, units)));
        const int blocks = w4_run_blocks(a.entries, a.share, units);
        if constexpr (PAIR) launch_product_kernel<q8_gated_small_run_kernel<TAIL, ONCE>>(a, blocks, w4_lds(128, 128), stage, st);
        else if (a.N % 4 == 0) launch_product_kernel<q8_small_run_kernel<true, TAIL, ONCE>>(a, blocks, w4_lds(128, 128), stage, st);
        else launch_product_kernel<q8_small_run_kernel<false, TAIL, ONCE>>(a, blocks, w4_lds(128, 128), stage, st);
    };
    if (l.whole && l.once) launch(std::false_type{}, std::true_type{});
    else if (l.whole) launch(std::false_type{}, std::false_type{});
    else if (l.once) launch(std::true_type{}, std::true_type{});
    else launch(std::true_type{}, std::false_type{});
}

bool known_type(int type) { return type >= kF32 && type <= kF16; }

moe_status check_rows(const char *call, int64_t R, int K, int type)
{
    if (R < 1 || K < 1 || !known_type(type)) {
        set_error("%s: R and K must be >= 1 and the type 0 (fp32), 1 (bf16) or 2 (fp16)", call);
        return MOE_EINVAL;
    }
    if (K % 16 != 0 || K > kMaxDepth || R > (1ll << 40) / K) {
        set_error("%s: K = %d must be a multiple of 16 up to %d, and R K at most 2^40", call, K, kMaxDepth);
        return MOE_EUNSUPPORTED;
    }
    return MOE_OK;
}

moe_status check_tiles(const char *call, int64_t rows, int E, int columns)
{
    if (tile_entries(rows, E, 128, (columns + 127) / 128) < kMostTiles) return MOE_OK;
    set_error("%s: %lld rows of %d columns are more than 2^23 tiles of 128 x 128", call, static_cast<long long>(rows), columns);
    return MOE_EUNSUPPORTED;
}

moe_status check_q8_block(const moe_shape *s)
{
    const moe_status rc = check_layer_shape(s);
    if (rc != MOE_OK) return rc;
    if (s->dtype != MOE_BF16) {
        set_error("moe_gated_ffn_q8: bf16 layers only");
        return MOE_EUNSUPPORTED;
    }
    if (s->d_model % 16 != 0 || s->d_ff % 16 != 0 || s->d_model > kMaxDepth || s->d_ff > kMaxDepth ||
        2ll * s->d_ff * s->d_model >= (1ll << 31) - (1 << 26) || moe_max_rows(s) >= 1ll << 30) {
        set_error("moe_gated_ffn_q8: d_model and d_ff multiples of 16 up to %d, 2 d_ff d_model below 2^31 - 2^26, rows below 2^30", kMaxDepth);
        return MOE_EUNSUPPORTED;
    }
    return check_tiles("moe_gated_ffn_q8", moe_max_rows(s), s->E, std::max(s->d_model, 2 * s->d_ff));
}

moe_status check_linear(const moe_q8_shape *s)
{
    if (s == nullptr) {
        set_error("moe_q8_linear: shape is NULL");
        return MOE_EINVAL;
    }
    if (s->R < 1 || s->E < 1 || s->N < 1 || s->K < 1 || !known_type(s->res) || !known_type(s->y) || s->act < MOE_ACT_GELU_ERF ||
        s->act > MOE_ACT_SILU) {
        set_error("moe_q8_linear: R, E, N, K must be >= 1, res and y 0 (fp32), 1 (bf16) or 2 (fp16), act a moe_act");
        return MOE_EINVAL;
    }
    if (s->E > kMaxExperts || s->N >= 1 << 21 || s->K % 16 != 0 || s->K > kMaxDepth || s->R >= 1 << 30) {
        set_error("moe_q8_linear: at most %d experts, N below 2^21, K a multiple of 16 up to %d, R below 2^30", kMaxExperts, kMaxDepth);
        return MOE_EUNSUPPORTED;
    }
    return check_tiles("moe_q8_linear", s->R, s->E, s->N);
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" {

moe_status moe_q8_rows(int64_t R, int32_t K, int32_t type, const void *x, void *q, float *scale, void *stream)
{
    const moe_status rc = check_rows("moe_q8_rows", R, K, type);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE_PTR(x);
    MOE_REQUIRE_PTR(q);
    MOE_REQUIRE_PTR(scale);
    launch_rows(R, K, type, x, q, scale, nullptr, static_cast<hipStream_t>(stream));
    MOE_TRY_HIP(hipGetLastError());
    return MOE_OK;
}

moe_status moe_q8_values(int64_t R, int32_t K, int32_t type, const void *q, const float *scale, void *x, void *stream)
{
    const moe_status rc = check_rows("moe_q8_values", R, K, type);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE_PTR(q);
    MOE_REQUIRE_PTR(scale);
    MOE_REQUIRE_PTR(x);
    const int rows = std::max(1, 1024 / (K / 16));
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>((R + rows - 1) / rows, 1 << 20));
    auto launch = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, static_cast<hipStream_t>(stream), static_cast<const uint32_t *>(q), scale, x, R, K, rows);
    };
    if (type == kF32) launch(q8_values_kernel<kF32>);
    else if (type == kB16) launch(q8_values_kernel<kB16>);
    else launch(q8_values_kernel<kF16>);
    MOE_TRY_HIP(hipGetLastError());
    return MOE_OK;
}

moe_status moe_q8_linear(const moe_q8_shape *s, const void *x, const float *x_scale, const int32_t *offsets, const void *w,
                         const float *w_scale, const float *bias, const void *r, void *y, void *stream)
{
    const moe_status rc = check_linear(s);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE_PTR(x);
    MOE_REQUIRE_PTR(x_scale);
    MOE_REQUIRE_PTR(offsets);
    MOE_REQUIRE_PTR(w);
    MOE_REQUIRE_PTR(w_scale);
    MOE_OPTIONAL_PTR(bias);
    MOE_OPTIONAL_PTR(r);
    MOE_REQUIRE_PTR(y);
    if (r == y && s->res != s->y) {
        set_error("moe_q8_linear: r may be y where their types are the same");
        return MOE_EINVAL;
    }
    Q8Args a = {};
    a.x = static_cast<const uint16_t *>(x);
    a.xs = x_scale;
    a.w = static_cast<const uint16_t *>(w);
    a.ws = w_scale;
    a.bias = bias;
    a.r = r;
    a.y = y;
    a.offsets = offsets;
    a.row_div = 1;
    a.E = s->E;
    a.N = s->N;
    a.K = s->K / 2;
    a.act = activation_of(s->act, s->y == kF32);
    a.res = s->res;
    a.type = s->y;
    launch_product<false>(a, s->R, -1, static_cast<hipStream_t>(stream));
    MOE_TRY_HIP(hipGetLastError());
    return MOE_OK;
}

moe_status moe_q8_linear_kernel(const moe_q8_shape *s, char *name, size_t len)
{
    if (name == nullptr || len == 0) {
        set_error("moe_q8_linear_kernel: name is NULL or has no room");
        return MOE_EINVAL;
    }
    const moe_status rc = check_linear(s);
    if (rc != MOE_OK) return rc;
    product_kernel_name(false, plan_launch(false, s->R, s->E, s->N, s->K / 2, 0), name, len);
    return MOE_OK;
}

moe_status moe_gated_q8_kernel(const moe_shape *s, int32_t which, char *name, size_t len)
{
    if (name == nullptr || len == 0 || which < 0 || which > 1) {
        set_error("moe_gated_q8_kernel: which must be 0 or 1, and name have room");
        return MOE_EINVAL;
    }
    const moe_status rc = check_q8_block(s);
    if (rc != MOE_OK) return rc;
    const int64_t R = moe_max_rows(s);
    product_kernel_name(which == 0, which == 0 ? plan_launch(true, R, s->E, 2 * s->d_ff, s->d_model / 2, s->d_ff) : plan_launch(false, R, s->E, s->d_model, s->d_ff / 2, 0),
                        name, len);
    return MOE_OK;
}

moe_status moe_dispatch_q8(const moe_shape *s, const void *x, const float *x_scale, const int32_t *expert_idx,
                           int32_t *counts, int32_t *offsets, int32_t *slot_of, int32_t *src_of, void *xe, float *xe_scale,
                           void *workspace, void *stream)
{
    const moe_status rc = check_layer_shape(s);
    if (rc != MOE_OK) return rc;
    if (s->d_model % 16 != 0) {
        set_error("moe_dispatch_q8: d_model = %d must be a multiple of 16", s->d_model);
        return MOE_EUNSUPPORTED;
    }
    MOE_REQUIRE_PTR(x);
    MOE_REQUIRE_PTR(x_scale);
    MOE_REQUIRE_PTR(expert_idx);
    MOE_REQUIRE_PTR(counts);
    MOE_REQUIRE_PTR(offsets);
    MOE_REQUIRE_PTR(slot_of);
    MOE_REQUIRE_PTR(src_of);
    MOE_OPTIONAL_PTR(xe);
    MOE_OPTIONAL_PTR(xe_scale);
    if ((xe == nullptr) != (xe_scale == nullptr)) {
        set_error("moe_dispatch_q8: xe and xe_scale come together");
        return MOE_EINVAL;
    }
    MOE_REQUIRE_PTR(workspace);
    Workspace w;
    layout_workspace(*s, 1, 1, workspace, &w);
    hipStream_t st = static_cast<hipStream_t>(stream);
    prof_begin(kStagePlan, st);
    const moe_status plan = launch_plan(*s, expert_idx, counts, offsets, slot_of, src_of, w, false, 0, st);
    prof_end(kStagePlan, st);
    if (plan != MOE_OK) return plan;
    if (xe != nullptr) {
        prof_begin(kStageScatter, st);
        hipLaunchKernelGGL(q8_scatter_kernel, dim3(std::min(parts_of(s->T, 4), 1 << 20)), dim3(256), 0, st, static_cast<const u32x4 *>(x), x_scale, slot_of,
                           static_cast<u32x4 *>(xe), xe_scale, s->T, s->k, s->d_model / 16, static_cast<int>(moe_max_rows(s)));
        prof_end(kStageScatter, st);
        MOE_TRY_HIP(hipGetLastError());
    }
    return MOE_OK;
}

size_t moe_gated_q8_workspace_bytes(const moe_shape *s)
{
    if (check_q8_block(s) != MOE_OK) return 0;
    const size_t R = static_cast<size_t>(moe_max_rows(s));
    return align_up(R * s->d_ff * 2, 256) + align_up(R * s->d_ff, 256) + align_up(R * 4, 256);
}

moe_status moe_gated_ffn_q8(const moe_shape *s, const void *x, const float *x_scale, const int32_t *src_of,
                            const int32_t *offsets, const void *q13, const float *scale13, const void *q2,
                            const float *scale2, void *ye, void *workspace, void *stream)
{
    const moe_status rc = check_q8_block(s);
    if (rc != MOE_OK) return rc;
    if (src_of != nullptr && static_cast<int64_t>(s->T) * s->d_model >= (1ll << 31) - (1 << 20)) {
        set_error("moe_gated_ffn_q8: with src_of T d_model has to be below 2^31 - 2^20; moe_dispatch_q8 moves the rows");
        return MOE_EUNSUPPORTED;
    }
    MOE_REQUIRE_PTR(x);
    MOE_REQUIRE_PTR(x_scale);
    MOE_OPTIONAL_PTR(src_of);
    MOE_REQUIRE_PTR(offsets);
    MOE_REQUIRE_PTR(q13);
    MOE_REQUIRE_PTR(scale13);
    MOE_REQUIRE_PTR(q2);
    MOE_REQUIRE_PTR(scale2);
    MOE_REQUIRE_PTR(ye);
    MOE_REQUIRE_PTR(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const size_t R = static_cast<size_t>(moe_max_rows(s));
    char *const hidden = static_cast<char *>(workspace), *const codes = hidden + align_up(R * s->d_ff * 2, 256);
    float *const scales = reinterpret_cast<float *>(codes + align_up(R * s->d_ff, 256));
    Q8Args a = {};
    a.x = static_cast<const uint16_t *>(x);
    a.xs = x_scale;
    a.w = static_cast<const uint16_t *>(q13);
    a.ws = scale13;
    a.y = hidden;
    a.offsets = offsets;
    a.row_src = src_of;
    a.row_div = s->k;
    a.a_rows = s->T;
    a.E = s->E;
    a.N = 2 * s->d_ff;
    a.K = s->d_model / 2;
    a.h = s->d_ff;
    a.act = s->act;
    launch_product<true>(a, static_cast<int64_t>(R), kStageGemm1, st);
    launch_rows(static_cast<int64_t>(R), s->d_ff, kF16, hidden, codes, scales, offsets + s->E, st);
    Q8Args b = {};
    b.x = reinterpret_cast<const uint16_t *>(codes);
    b.xs = scales;
    b.w = static_cast<const uint16_t *>(q2);
    b.ws = scale2;
    b.y = ye;
    b.offsets = offsets;
    b.row_div = 1;
    b.E = s->E;
    b.N = s->d_model;
    b.K = s->d_ff / 2;
    b.act = MOE_ACT_IDENTITY;
    b.type = kF16;
    launch_product<false>(b, static_cast<int64_t>(R), kStageGemm2, st);
    MOE_TRY_HIP(hipGetLastError());
    return MOE_OK;
}

}  // extern "C"
