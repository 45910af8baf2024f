// The gated feed-forward block on expert-major rows (include/moe_gated.h):
//   H = act(xe Wg) * (xe Wu), ye = H W2, and its backward pass.
//
// Forward: one grouped GEMM over the packed first projections, in which sixteen columns of Wg and the same sixteen of Wu
// take turns, so that a lane's accumulators hold a gate and the value that it gates: the activation and the product are
// the epilogue, and G and U go to memory only where a backward pass will read them.  The second GEMM is the expert FFN's.
// Backward: dH = dye W2^T with G and U brought into LDS behind its last stages, dG and dU its epilogue; dxe = [dG | dU] W13^T,
// one product over 2 d_ff; the weight gradients are the expert FFN's kernels, rounded to bf16.
// H is rounded to fp16, since the second product's operands are of 16 bits: 2^-11 of a value where bf16 is off by 2^-8 (the block's
// output 2.9e-4 root mean square from 64-bit results where fp32 throughout and one rounding of the output are 2.1e-4), for a
// largest value of 65504.  What is kept for the backward pass, G, U and H, is rounded to fp16 for the same reason and to half the bytes;
// dG, dU and, as an operand, H to bf16, whose range gradients need and which all operands of a product share: 2.4e-3 where one rounding
// of the gradients alone is 1.7e-3.
// The loops are the expert FFN's: tiles of 256 columns on gemm_w4_run.h's, 128 x 128 on gemm_w4_body.inc's, decode steps
// straight from global memory.
#include "activation.h"
#include "block_tile.h"
#include "gated.h"
#include "moe_gated.h"

#include <algorithm>
#include <cstdio>

#include <hip/hip_ext.h>

#include <type_traits>

namespace moe {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;

#include "gemm_w4.h"
#include "gemm_w4_run.h"

__device__ __forceinline__ void store_f16x4(char *p, const float (&v)[4])
{
    f16x4 h;
#pragma unroll
    for (int c = 0; c < 4; ++c) h[c] = static_cast<_Float16>(v[c]);
    *reinterpret_cast<f16x4 *>(p) = h;
}
__device__ __forceinline__ void store_bf16x4(char *p, const float (&v)[4])
{
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    u32x2 o;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        bf16x2 b;
        b[0] = static_cast<__bf16>(v[2 * c]);
        b[1] = static_cast<__bf16>(v[2 * c + 1]);
        o[c] = __builtin_bit_cast(uint32_t, b);
    }
    *reinterpret_cast<u32x2 *>(p) = o;
}

// ---------------------------------------------------------------- first projections, tiles of 256 packed columns
// Bound by the matrix cores at the clock that their energy leaves, as the expert FFN's: 32768 rows, 32 experts, 2048 x 8192,
// 256 x 256 tiles, 1745 us, 1260 TFLOP/s (a vendor library's dense product of that size 1200); keeping G, U and H for the backward
// pass, 16384 rows, 8 experts, 2048 x 5632, 596 us, 1269 TFLOP/s.
// R of a wavefront's rows, from `r` on, as they lie in the patch's rows 16 part .. (W4Place): PIECES 16-byte pieces of 8
// columns each, to columns col0 + 8 piece of `out`; of 16 pieces the last eight go pair_at columns further on.
template <int BM, int R, int PIECES>
__device__ __forceinline__ void leave_gated(const W4Place<BM> &place, uint16_t *out, int pitch, int pair_at, int col0, int h,
                                            int row0, int row1, int part)
{
    constexpr int ROWS = 64 / PIECES;
    // (a row past the tile's or a column past h lies past the resource)
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        out + static_cast<size_t>(row0) * pitch, 0, static_cast<unsigned>(max(row1 - row0, 0)) * pitch * 2u, 0x00020000);
    const int piece = place.lane % PIECES, lane_row = place.lane / PIECES, col = col0 + piece % 8 * 8;
    const int first = col < h ? (lane_row * pitch + col + (piece >= 8 ? pair_at : 0)) * 2 : 0x7ff00000;
    const int step = col < h ? ROWS * pitch * 2 : 0;
    lds_handover();
    MOE_SB();
#pragma unroll
    for (int it = 0; it < R / ROWS; ++it) {
        const int row = it * ROWS + lane_row;
        const u32x4 q = *reinterpret_cast<const u32x4 *>(place.patch + (part * 16 + row) * 256 + ((piece ^ (row & 15)) << 4));
        __builtin_amdgcn_raw_buffer_store_b128(q, rs, first + it * step, 0, 0);
        if (it % 4 == 3) MOE_SB();
    }
    lds_handover();
}

// acc[2 p] and acc[2 p + 1] of a lane: gate and value of the same four columns
template <int ACT, bool KEEP, bool KTAIL, int BM>
__global__ __launch_bounds__(256, 1) void gated_run_kernel(
    const uint16_t *__restrict__ A, const uint16_t *__restrict__ W, uint16_t *__restrict__ H, uint16_t *__restrict__ Pre,
    const WorkItem *__restrict__ items, int entries, int share, int N, int K, int h)
{
    struct None {};
    w4_run<false, KTAIL, BM, 0>(A, W, items, nullptr, entries, share, N, K, nullptr, 1, 0, [](const WorkItem &, int, int) { return None{}; },
        [&](auto &acc, const None &, const WorkItem &item, const W4Place<BM> &place, auto landed) {
            const int col0 = item.n0 / 2 + place.wn * 64;
            // 16 rows at a time: gates and values through the patch's first sixteen rows, H through the last
            // sixteen (of 128 x 256 tiles, which have sixteen, through the same)
            constexpr int HPART = W4Place<BM>::UR == 32 && KEEP ? 1 : 0;
#pragma unroll
            for (int j = 0; j < W4Place<BM>::TM; ++j) {
                const int row0 = item.row0 + place.wm * (BM / 2) + j * 16;
                if constexpr (KEEP) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                        store_f16x4(place.at((i & 1) * 4 + (i >> 1), 0), v);
                        if (i % 4 == 3) MOE_SB();
                    }
                    if (j == 0) landed();
                    leave_gated<BM, 16, 16>(place, Pre, 2 * h, h, col0, h, row0, item.row1, 0);
                }
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    float v[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) v[c] = gate_value<ACT>(acc[2 * p][j][c]) * acc[2 * p + 1][j][c];
                    store_f16x4(place.at(p, HPART), v);
                    if (p % 2 == 1) MOE_SB();
                }
                if (!KEEP && j == 0) landed();
                leave_gated<BM, 16, 8>(place, H, h, 0, col0, h, row0, item.row1, HPART);
            }
        });
}

// ---------------------------------------------------------------- first projections, 128 x 128 tiles
// For some hundred rows per expert, bound by bytes into LDS; with five stages on their way (DEEP) for fewer, bound by the weights'
// arrival: the block of 8 experts, 2048 x 5632, 48 rows each, 142 us, 3.9 TB/s (128 x 256 tiles 150, 256 x 256 164).
template <int ACT, bool KEEP, bool KTAIL, bool DEEP>
__global__ __launch_bounds__(256, DEEP ? 1 : 2) void gated_tile_kernel(
    const uint16_t *__restrict__ A, const uint16_t *__restrict__ W, uint16_t *__restrict__ H, uint16_t *__restrict__ Pre,
    const WorkItem *__restrict__ items, int N, int K, int h)
{
    constexpr int BM = 128, BN = 128;
    constexpr bool F16 = false, TILE_IN = false, TILE_PAIR = false, W_PAIR = false, W_ONCE = false;
    constexpr int tile_pitch = 0, pair_at = 0, row_div = 1, a_rows = 0, pair_h = 0;
    const uint16_t *const tile_in = nullptr;
    const int32_t *const row_src = nullptr;
#include "gemm_w4_body.inc"

    // the wavefront's 64 rows of 32 gates and 32 values, or of 32 hidden values: 16 bytes of row padding
    constexpr int PITCH = 128 + 16;
    char *const patch = lds + wave * 64 * PITCH;
    const int rbase = item.row0 + wm * 64, hcol = n0 / 2 + wn * 32;
#pragma unroll
    for (int pass = KEEP ? 0 : 1; pass < 2; ++pass) {      // pass 0: G and U, 1: H
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                char *const at = patch + (j * 16 + fr) * PITCH + (p * 16 + 4 * oct) * 2;
                float v[4], u[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    u[c] = acc[2 * p + 1][j][c];
                    v[c] = pass == 0 ? acc[2 * p][j][c] : gate_value<ACT>(acc[2 * p][j][c]) * u[c];
                }
                store_f16x4(at, v);
                if (pass == 0) store_f16x4(at + 64, u);
                if (j == TM / 2 - 1) MOE_SB();
            }
            MOE_SB();
        }
        MOE_LGKM0();
        __builtin_amdgcn_wave_barrier();
        auto leave = [&](auto piecesc, uint16_t *out, int pitch) {
            constexpr int PIECES = decltype(piecesc)::value, ROWS = 64 / PIECES;
            const int piece = lane % PIECES, col = hcol + piece % 4 * 8;
#pragma unroll 8
            for (int it = 0; it < 64 / ROWS; ++it) {
                const int rr = it * ROWS + lane / PIECES, r = rbase + rr;
                const u32x4 q = *reinterpret_cast<const u32x4 *>(patch + rr * PITCH + piece * 16);
                if (r < item.row1 && col < h)
                    *reinterpret_cast<u32x4 *>(out + static_cast<size_t>(r) * pitch + col + (piece >= 4 ? h : 0)) = q;
            }
        };
        if (pass == 0) {
            leave(std::integral_constant<int, 8>{}, Pre, 2 * h);
            MOE_LGKM0();
            __builtin_amdgcn_wave_barrier();
        } else {
            leave(std::integral_constant<int, 4>{}, H, h);
        }
    }
}

// ---------------------------------------------------------------- first projections, few rows per expert
// As grouped_gemm_stream_kernel of the expert FFN: a wavefront takes its fragments straight from global memory, here of 32
// packed columns (sixteen gates and their values) and at most 32 rows, PD stages of 64 on their way; the block finds its tile
// from the offsets.  32 rows, 16 experts, 768 x 2048: 15.8 us, 6.4 TB/s of weights (a list of tiles made first: 3 us and a launch
// more).
template <int ACT, bool KEEP, bool KTAIL>
__global__ __launch_bounds__(64, 2) void gated_stream_kernel(
    const uint16_t *__restrict__ A, const uint16_t *__restrict__ W, _Float16 *__restrict__ H, _Float16 *__restrict__ Pre,
    const int32_t *__restrict__ offsets, int E, int N, int K, int h)
{
    WorkItem item;
    if (!block_tile<32>(offsets, E, N / 32, blockIdx.x, item.expert, item.row0, item.row1, item.n0)) return;
    const int rows = item.row1 - item.row0, nw = item.n0 * 32;
    const int lane = threadIdx.x, fr = lane & 15, oct = lane >> 4;
    const int KT = (K + 63) / 64;
    const uint16_t *wp[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)         // (N is a multiple of 32)
        wp[t] = W + (static_cast<size_t>(item.expert) * N + nw + t * 16 + fr) * K + oct * 8;

    auto body = [&](auto rt, auto pd) {
        constexpr int RT = decltype(rt)::value, PD = decltype(pd)::value;
        const uint16_t *ap[RT];
#pragma unroll
        for (int j = 0; j < RT; ++j)
            ap[j] = A + static_cast<size_t>(item.row0 + min(j * 16 + fr, rows - 1)) * K + oct * 8;
        u32x4 wr[PD][2][2], ar[PD][RT][2];
        // (no branches around the loads: a piece past K is read from inside the row, and zeroed when multiplied)
        auto load = [&](auto u, int s) {
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                int k0 = s * 64 + p * 32;
                if constexpr (KTAIL) k0 = min(k0, K - 8 - oct * 8);
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    wr[decltype(u)::value][t][p] = *reinterpret_cast<const u32x4 *>(wp[t] + k0);
#pragma unroll
                for (int j = 0; j < RT; ++j)
                    ar[decltype(u)::value][j][p] = *reinterpret_cast<const u32x4 *>(ap[j] + k0);
            }
        };
        f32x4 acc[2][RT];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int j = 0; j < RT; ++j) acc[t][j] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
        auto use = [&](auto u, auto tail, int s) {
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const bool past = KTAIL && decltype(tail)::value && s * 64 + p * 32 + oct * 8 >= K;
                const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const u32x4 w = past ? zero : wr[decltype(u)::value][t][p];
#pragma unroll
                    for (int j = 0; j < RT; ++j) {
                        const u32x4 a = past ? zero : ar[decltype(u)::value][j][p];
                        acc[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, a), acc[t][j], 0, 0, 0);
                    }
                }
            }
        };
        static_for<PD>([&](auto u) { load(u, min(decltype(u)::value, KT - 1)); });
        int s = 0;
        for (; s + 2 * PD <= KT; s += PD)
            static_for<PD>([&](auto u) {
                use(u, std::false_type{}, 0);
                load(u, s + decltype(u)::value + PD);
                __builtin_amdgcn_sched_barrier(0);
            });
        for (; s < KT; s += PD)                      // the last stages: fewer than two rounds
            static_for<PD>([&](auto u) {
                if (s + decltype(u)::value < KT) use(u, std::true_type{}, s + decltype(u)::value);
                if (s + decltype(u)::value + PD < KT) load(u, s + decltype(u)::value + PD);
            });

        // acc[t][j][c]: gate (t = 0) or value of hidden column nw / 2 + 4 oct + c, row row0 + 16 j + fr
        const int n = nw / 2 + 4 * oct;
        if (n >= h) return;
#pragma unroll
        for (int j = 0; j < RT; ++j) {
            if (j * 16 + fr >= rows) continue;
            const size_t r = static_cast<size_t>(item.row0 + j * 16 + fr);
            float v[4], g[4], u[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                g[c] = acc[0][j][c];
                u[c] = acc[1][j][c];
                v[c] = gate_value<ACT>(g[c]) * u[c];
            }
            if constexpr (KEEP) {
                store_f16x4(reinterpret_cast<char *>(Pre + r * 2 * h + n), g);
                store_f16x4(reinterpret_cast<char *>(Pre + r * 2 * h + h + n), u);
            }
            store_f16x4(reinterpret_cast<char *>(H + r * h + n), v);
        }
    };
    using std::integral_constant;
    if (rows <= 16)
        body(integral_constant<int, 1>{}, integral_constant<int, 6>{});
    else
        body(integral_constant<int, 2>{}, integral_constant<int, 4>{});
}

// ---------------------------------------------------------------- fp32 layers
template <int ACT>
__device__ __forceinline__ float gate_value_f32(float v)
{
    if constexpr (ACT == MOE_ACT_SILU) return v / (1.0f + expf(-v));
    else if constexpr (ACT == MOE_ACT_GELU_ERF) return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
    else if constexpr (ACT == MOE_ACT_GELU_TANH) return 0.5f * v * (1.0f + tanhf(0.7978845608028654f * (v + 0.044715f * v * v * v)));
    else if constexpr (ACT == MOE_ACT_RELU) return fmaxf(v, 0.0f);
    else return v;
}

// H = act(A Wg) * (A Wu), W13 canonical [E, K, 2 h]: as grouped_gemm_f32_kernel of the expert FFN, with a second set of
// weight columns.  Tiles of 32 TM rows x 32 hidden columns, four wavefronts of 16 TM x 16, on the fp32 matrix instruction.  512 rows,
// 4 experts, 128 x 256: 5.3 us, most of it a launch's latency (tiles from the offsets; behind a list of them 3 us more); 4096 rows,
// one expert, 1024 x 2560, the block 106 TFLOP/s.
template <int ACT, int TM>
__global__ __launch_bounds__(256) void gated_f32_kernel(const float *__restrict__ A, const float *__restrict__ B,
                                                        float *__restrict__ H, const int32_t *__restrict__ offsets, int E, int h, int K)
{
    WorkItem tile;
    if (!block_tile<32 * TM>(offsets, E, (h + 31) / 32, blockIdx.x, tile.expert, tile.row0, tile.row1, tile.n0)) return;
    const int n0 = tile.n0 * 32;
    constexpr int BM = 32 * TM, BN = 32, BK = 32, PD = 4, LDA = BK + 4, LDB = BN + 4;
    __shared__ __attribute__((aligned(16))) float As[2][BM * LDA];
    __shared__ __attribute__((aligned(16))) float Bs[2][2][BK * LDB];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave & 1, wn = wave >> 1, r16 = lane & 15, kq = lane >> 4;
    const int KT = (K + BK - 1) / BK;
    const size_t N = 2 * static_cast<size_t>(h);

    const int a_row = tid / 8, a_k = tid % 8 * 4, b_k = tid / 8, b_n = tid % 8 * 4;
    const float *a_src[TM];
#pragma unroll
    for (int m = 0; m < TM; ++m) a_src[m] = A + static_cast<size_t>(min(tile.row0 + a_row + 32 * m, tile.row1 - 1)) * K;
    const float *b_src = B + static_cast<size_t>(tile.expert) * K * N + min(n0 + b_n, h - 4);   // (columns past h are not stored)
    f32x4 ar[PD][TM], br[PD][2];
    // (no branches around the loads: what lies past K is read from inside and zeroed on its way into LDS)
    auto load = [&](auto slot, int s) {
        constexpr int u = decltype(slot)::value;
#pragma unroll
        for (int m = 0; m < TM; ++m) ar[u][m] = *reinterpret_cast<const f32x4 *>(a_src[m] + min(s * BK + a_k, K - 4));
#pragma unroll
        for (int t = 0; t < 2; ++t)
            br[u][t] = *reinterpret_cast<const f32x4 *>(b_src + static_cast<size_t>(min(s * BK + b_k, K - 1)) * N + t * h);
    };
    f32x4 acc[2][TM];
#pragma unroll
    for (int m = 0; m < TM; ++m) acc[0][m] = acc[1][m] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    auto stage = [&](auto slot, int s) {
        constexpr int u = decltype(slot)::value, buf = u & 1;
        const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int m = 0; m < TM; ++m) *reinterpret_cast<f32x4 *>(&As[buf][(a_row + 32 * m) * LDA + a_k]) = s * BK + a_k < K ? ar[u][m] : zero;
#pragma unroll
        for (int t = 0; t < 2; ++t)
            *reinterpret_cast<f32x4 *>(&Bs[buf][t][b_k * LDB + b_n]) = s * BK + b_k < K ? br[u][t] : zero;
        load(slot, min(s + PD, KT - 1));         // (past the last stage: loaded again, never used)
        // LDS writes only are waited for: the loads stay in flight across the barrier
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int c = 0; c < BK; c += 16) {
            f32x4 af[TM];
#pragma unroll
            for (int m = 0; m < TM; ++m)
                af[m] = *reinterpret_cast<const f32x4 *>(&As[buf][((wm * TM + m) * 16 + r16) * LDA + c + 4 * kq]);
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const float w = Bs[buf][t][(c + 4 * kq + q) * LDB + wn * 16 + r16];
#pragma unroll
                    for (int m = 0; m < TM; ++m) acc[t][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(w, af[m][q], acc[t][m], 0, 0, 0);
                }
        }
    };
    static_for<PD>([&](auto u) { load(u, min(decltype(u)::value, KT - 1)); });
    int s0 = 0;
    for (; s0 + PD <= KT; s0 += PD) static_for<PD>([&](auto u) { stage(u, s0 + decltype(u)::value); });
    static_for<PD>([&](auto u) {
        if (s0 + decltype(u)::value < KT) stage(u, s0 + decltype(u)::value);
    });
    // acc[t][m][c]: column n0 + wn * 16 + 4 kq + c, row row0 + (wm * TM + m) * 16 + r16
    const int n = n0 + wn * 16 + 4 * kq;
    if (n >= h) return;
#pragma unroll
    for (int m = 0; m < TM; ++m) {
        const int r = tile.row0 + (wm * TM + m) * 16 + r16;
        if (r >= tile.row1) return;
        f32x4 o;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = gate_value_f32<ACT>(acc[0][m][c]) * acc[1][m][c];
        *reinterpret_cast<f32x4 *>(H + static_cast<size_t>(r) * h + n) = o;
    }
}

// ---------------------------------------------------------------- backward: dH and through the gate
// a b, and 0 where either is 0 and the other infinite
__device__ __forceinline__ float times_or_zero(float a, float b)
{
    float v = 0.0f;
#if defined(__HIP_DEVICE_COMPILE__)
    asm("v_mul_legacy_f32 %0, %1, %2" : "=v"(v) : "v"(a), "v"(b));
#endif
    return v;
}

// C tile dH = dye W2^T; out = [dG | dU] = [dH U act'(G) | dH act(G)], both bf16, G and U from pre [rows, 2 h].  G and U come
// into LDS behind the last stages, 32 rows of a wavefront's part at a time, and are turned into dG and dU in their places; of
// 256 x 256 tiles the rows from 64 on follow while the first ones are computed.  16384 rows, 8 experts, 2048 x 5632: 399 us alone,
// 947 TFLOP/s: per 256 x 256 tile of 32 stages 512 KiB come in and go out behind the loop.
template <int ACT, bool KTAIL, int BM>
__global__ __launch_bounds__(256, BM == 128 ? 2 : 1) void gated_dh_kernel(
    const uint16_t *__restrict__ A, const uint16_t *__restrict__ W, const uint16_t *__restrict__ pre, uint16_t *__restrict__ out,
    const WorkItem *__restrict__ items, int N, int K)
{
    constexpr int BN = BM;
    constexpr bool F16 = false, TILE_IN = true, TILE_PAIR = true, DEEP = false, W_PAIR = false, W_ONCE = false;
    constexpr int row_div = 1, a_rows = 0, pair_h = 0;
    const int32_t *const row_src = nullptr;
    const uint16_t *const tile_in = pre;
    const int tile_pitch = 2 * N, pair_at = N;
#include "gemm_w4_body.inc"

    constexpr int LPR = BN / 16, RPI = 64 / LPR, LINES = 32 / RPI;
    const int rbase = item.row0 + wm * (BM / 2), ncol = n0 + wn * (BN / 2) + lane % LPR * 8;
    const int pair[2][2] = {{ua, uw}, {ua1, uw1}};
    static_for<BM / 64>([&](auto uc) {                // rows 32 u .. of the wavefront's part
        constexpr int u = decltype(uc)::value;
        // What may be on its way behind this pair: the pair behind it, and the stores of the pairs before.
        if constexpr (u == 0) MOE_VMCNT(2 * TILE_LOADS);
        else if constexpr (BM == 128) MOE_VMCNT(2 * LINES);
        else if constexpr (u == 1) MOE_VMCNT(2 * TILE_LOADS + 2 * LINES);
        else if constexpr (u == 2) MOE_VMCNT(2 * TILE_LOADS + 4 * LINES);
        else MOE_VMCNT(4 * LINES);
        char *const gp = lds + pair[u & 1][0] + wave * (W_UNIT / 4), *const up = lds + pair[u & 1][1] + wave * (W_UNIT / 4);
#pragma unroll
        for (int jj = 0; jj < 2; ++jj) {
            const int j = 2 * u + jj, row = jj * 16 + fr;
            f16x4 g[TN], v[TN];
            auto place = [&](int i) { return row * BN + (((2 * i + (oct >> 1)) ^ tile_key(row)) << 4) + (oct & 1) * 8; };
#pragma unroll
            for (int i = 0; i < TN; ++i) {
                g[i] = *reinterpret_cast<const f16x4 *>(gp + place(i));
                v[i] = *reinterpret_cast<const f16x4 *>(up + place(i));
            }
#pragma unroll
            for (int i = 0; i < TN; ++i) {
                float dg[4], du[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float value, slope;
                    gate_value_and_slope<ACT>(static_cast<float>(g[i][c]), value, slope);
                    // (0 times what fp16 has made infinite is 0, as it is with the value itself)
                    const float dh = acc[i][j][c];
                    dg[c] = times_or_zero(dh * slope, static_cast<float>(v[i][c]));
                    du[c] = times_or_zero(dh, value);
                }
                store_bf16x4(gp + place(i), dg);
                store_bf16x4(up + place(i), du);
                if (i % 2 == 1) MOE_SB();   // a few accumulator registers at a time leave the AGPRs
            }
        }
        __builtin_amdgcn_wave_barrier();
        u32x4 line[2][LINES];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int it = 0; it < LINES; ++it) {
                const int rr = it * RPI + lane / LPR;
                line[t][it] = *reinterpret_cast<const u32x4 *>((t == 0 ? gp : up) + rr * BN + ((lane % LPR ^ tile_key(rr)) << 4));
            }
        if constexpr (BM == 256 && u < 2) {
            // (the places are free when they have been read)
            MOE_LGKM0();
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int at = wm * (BM / 2) + (u + 2) * 32, from = t * pair_at, col0 = n0 + wn * (BN / 2);
                const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
                    const_cast<uint16_t *>(tile_in) + static_cast<size_t>(item.row0 + min(at, rows - 1)) * tile_pitch + from + min(col0, N - 8), 0,
                    static_cast<unsigned>(at < rows && col0 < N ? ((rows - at) * tile_pitch - from - col0) * 2 : 0), 0x00020000);
#pragma unroll
                for (int q = 0; q < TILE_LOADS; ++q) load_to_lds(rs, t_src[q], w_dest + pair[u & 1][t] + q * 1024, 0);
            }
        }
        MOE_SB();
        // (stores whose rows or columns lie outside are issued too, past the resource, so that their number is known)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int row0 = rbase + u * 32;
            const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
                out + static_cast<size_t>(row0) * tile_pitch + t * pair_at, 0,
                static_cast<unsigned>(max((item.row1 - row0) * tile_pitch - t * pair_at, 0)) * 2u, 0x00020000);
#pragma unroll
            for (int it = 0; it < LINES; ++it) {
                const int rr = it * RPI + lane / LPR;
                __builtin_amdgcn_raw_buffer_store_b128(line[t][it], rs, ncol < N ? (rr * tile_pitch + ncol) * 2 : 0x7ff00000, 0, 0);
            }
        }
        MOE_SB();
    });
}

// ---------------------------------------------------------------- backward: dxe
// C [rows, N] bf16 = A W^T, A = [dG | dU].  16384 rows, 8 experts, N = 2048, K = 11264, 128 x 256 tiles: 850 us alone, 889 TFLOP/s (544 tiles of
// 256 x 256 are two rounds and a bit); the weight gradients beside it fill the last one.
template <bool KTAIL, int BM>
__global__ __launch_bounds__(256, 1) void rows_bf16_run_kernel(
    const uint16_t *__restrict__ A, const uint16_t *__restrict__ W, uint16_t *__restrict__ C, const WorkItem *__restrict__ items,
    int entries, int share, int N, int K)
{
    struct None {};
    w4_run<false, KTAIL, BM, 0>(A, W, items, nullptr, entries, share, N, K, nullptr, 1, 0, [](const WorkItem &, int, int) { return None{}; },
        [&](auto &acc, const None &, const WorkItem &item, const W4Place<BM> &place, auto landed) {
            constexpr int R = W4Place<BM>::UR;
#pragma unroll
            for (int r = 0; r < BM / 2; r += R) {
#pragma unroll
                for (int j = r / 16; j < (r + R) / 16; ++j) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                        store_bf16x4(place.at(i, j - r / 16), v);
                        if (i % 4 == 3) MOE_SB();
                    }
                }
                if (r == 0) landed();
                place.template leave<R>(C, item, r, 0, N);
            }
        });
}

template <bool KTAIL, bool DEEP>
__global__ __launch_bounds__(256, DEEP ? 1 : 2) void rows_bf16_tile_kernel(
    const uint16_t *__restrict__ A, const uint16_t *__restrict__ W, uint16_t *__restrict__ C, const WorkItem *__restrict__ items,
    int N, int K)
{
    constexpr int BM = 128, BN = 128;
    constexpr bool F16 = false, TILE_IN = false, TILE_PAIR = false, W_PAIR = false, W_ONCE = false;
    constexpr int tile_pitch = 0, pair_at = 0, row_div = 1, a_rows = 0, pair_h = 0;
    const uint16_t *const tile_in = nullptr;
    const int32_t *const row_src = nullptr;
#include "gemm_w4_body.inc"

    constexpr int PITCH = BN + 16, LPR = BN / 16, RPI = 64 / LPR;
    char *const patch = lds + wave * (BM / 2) * PITCH;
    const int rbase = item.row0 + wm * (BM / 2), ncol = n0 + wn * (BN / 2) + lane % LPR * 8;
#pragma unroll
    for (int i = 0; i < TN; ++i) {
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            store_bf16x4(patch + (j * 16 + fr) * PITCH + (i * 16 + 4 * oct) * 2, v);
        }
        MOE_SB();
    }
    MOE_LGKM0();
    __builtin_amdgcn_wave_barrier();
#pragma unroll 8
    for (int it = 0; it < BM / 2 / RPI; ++it) {
        const int rr = it * RPI + lane / LPR, r = rbase + rr;
        const u32x4 q = *reinterpret_cast<const u32x4 *>(patch + rr * PITCH + lane % LPR * 16);
        if (r < item.row1 && ncol < N) *reinterpret_cast<u32x4 *>(C + static_cast<size_t>(r) * N + ncol) = q;
    }
}

// ---------------------------------------------------------------- weight packing
// out[e][column n of in, packed][k] = in[e][k][n], 64 x 64 tiles through LDS.  GATED: n in [0, 2 h), columns n and h + n are
// sixteen apart, padding columns zeros; else out[e][n][k], from bf16 to fp16.
// Bound by HBM: 16 bytes per lane both ways.  8 experts, 2048 x 11264: 178 us, 4.2 TB/s; rows of 2000 bytes (K = 1000) 3.4.
template <bool GATED>
__global__ __launch_bounds__(256) void gated_pack_kernel(const uint16_t *__restrict__ in, uint16_t *__restrict__ out, int K,
                                                         int N, int NP)
{
    constexpr int PITCH = 66;                      // (33 words: a column's elements fall into different banks)
    __shared__ uint16_t tile[64 * PITCH];
    const size_t expert = blockIdx.z;
    const int k0 = blockIdx.y * 64, p0 = blockIdx.x * 64;
    // packed column p (of 64 from p0 on) -> column of the matrix, -1: padding
    auto column = [&](int p) {
        if constexpr (!GATED) return p < N ? p : -1;
        const int h = N / 2, b = p / 32, c = b * 16 + p % 16;
        return c < h ? c + (p % 32 < 16 ? 0 : h) : -1;
    };
    const uint16_t *src = in + expert * K * N;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int v = threadIdx.x + 256 * q, kk = v / 8, pp = v % 8 * 8, n = column(p0 + pp);
        u32x4 w = {0u, 0u, 0u, 0u};                // (eight packed columns are eight of the matrix's)
        if (n >= 0 && k0 + kk < K) w = *reinterpret_cast<const u32x4 *>(src + static_cast<size_t>(k0 + kk) * N + n);
#pragma unroll
        for (int c = 0; c < 4; ++c) *reinterpret_cast<uint32_t *>(&tile[kk * PITCH + pp + 2 * c]) = w[c];
    }
    __syncthreads();
    uint16_t *dst = out + expert * K * NP;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int v = threadIdx.x + 256 * q, pp = v / 8, kk = v % 8 * 8;
        if (p0 + pp >= NP || k0 + kk >= K) continue;
        u32x4 w;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            uint32_t lo = tile[(kk + 2 * c) * PITCH + pp], hi = tile[(kk + 2 * c + 1) * PITCH + pp];
            if constexpr (!GATED) {
                lo = __builtin_bit_cast(uint16_t, static_cast<_Float16>(bf16_to_f32(static_cast<uint16_t>(lo))));
                hi = __builtin_bit_cast(uint16_t, static_cast<_Float16>(bf16_to_f32(static_cast<uint16_t>(hi))));
            }
            w[c] = lo | (hi << 16);
        }
        *reinterpret_cast<u32x4 *>(dst + static_cast<size_t>(p0 + pp) * K + k0 + kk) = w;
    }
}

// ---------------------------------------------------------------- host side
// Tile of a row-grouped GEMM on these kernels.  few: the kernel for decode steps is there, and few rows mean that the weights'
// arrival bounds the launch (first projections); mid: that of 128 x 256 tiles.
//  * Decode kernel / 128 x 128 tiles, us of the whole block, 16 experts 768 x 2048, 8 of 2048 x 5632, 64 of 512 x 1376, 4 of 4096 x
//    2048: 5 rows per expert 29 / 32, 118 / 124, 48 / 52, 37 / 46, 8 rows 31 / 33, 122 / 127, 57 / 55, 39 / 47, 16 rows 36 / 36, 140 / 135,
//    65 / 56, 47 / 46.  Of experts whose rows are uneven (popularity by 1 / rank) the line lies lower: 6 rows 33 / 34 and 121 / 125, 8 rows
//    42 / 38 and 132 / 131, 10 rows 42 / 38 and 140 / 136.  While its blocks are few it holds longer: one expert 1024 x 2816, 32 rows 17 /
//    22, 48 rows 33 / 31.
//  * Up to 64 rows per expert, K = 2048, five stages of 128 x 128 on their way / the general choice: 16 rows 135 / 146, 32 139 / 160, 64
//    146 / 158, 128 170 / 174, 256 233 / 224; uneven rows, 20 133 / 143, 64 137 / 148; K = 768 40 / 36, K = 1024 119 / 112.
//  * Else the expert FFN's choice, from no fewer rows than one tile has (one expert, 128 rows: 47 -> 32).
GemmPlan plan_gated(int64_t rows, int E, int N, int K, bool few, bool mid, int64_t max_rows)
{
    GemmPlan gp;
    if (few && (rows <= 7 * static_cast<int64_t>(E) ||
                (rows <= 32 * static_cast<int64_t>(E) && rows * ((N + 127) / 128) <= 2000))) {
        gp.bm = 32;
        gp.bn = 64;
        gp.concurrent = 128;
    } else if (mid && (few_long_tiles(rows, E, N, K) || (few && K >= 1920 && rows <= 64 * static_cast<int64_t>(E)))) {
        gp.bm = gp.bn = 128;
        gp.concurrent = 32;
        gp.w4 = gp.deep = true;
    } else {
        choose_w4_tile(std::max<int64_t>(rows, 256), E, N, K, &gp);
        if (!mid && gp.bm != gp.bn) {
            gp.bn = 128;
            gp.concurrent = 64;
        }
    }
    gp.tiles_n = (N + gp.bn - 1) / gp.bn;
    gp.max_row_tiles = static_cast<int32_t>((max_rows + gp.bm - 1) / gp.bm + E);
    gp.max_items = work_list_entries(gp);
    return gp;
}

// Whether the form of a tile kernel that takes its depth in whole stages of 64 serves (with loads that run on from tile to
// tile, also four of them at least); else that with a tail.
bool whole_stages(const GemmPlan &gp, int K) { return K % 64 == 0 && (gp.bn != 256 || K >= 256); }

struct GatedWorkspace {
    Workspace lists;           // work lists of the two GEMMs, and (last) the hidden activations
    size_t bytes, kept_bytes;  // kept_bytes: where the caller keeps those
};
void layout_gated(const moe_shape &s, void *base, GatedWorkspace *w)
{
    const int64_t R = moe_max_rows(&s);
    char *p = static_cast<char *>(base);
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char *at = p + off;
        off += align_up(bytes, 256);
        return at;
    };
    w->lists = Workspace{};
    const bool f32 = s.dtype == MOE_F32;
    if (f32) {
        w->lists.gp[0].max_items = 0;          // (both GEMMs find their tiles from the offsets)
    } else {
        w->lists.gp[0] = plan_gated(R, s.E, gated_packed_columns(s.d_ff), s.d_model, true, true, R);
    }
    w->lists.gp[1] = choose_gemm_plan(s, 1, 1, s.T);
    for (int g = 0; g < 2; ++g)
        w->lists.items[g] = reinterpret_cast<WorkItem *>(take(sizeof(WorkItem) * w->lists.gp[g].max_items));
    w->kept_bytes = off;
    w->lists.hidden = take(static_cast<size_t>(R) * s.d_ff * (f32 ? 4 : 2));
    w->bytes = off;
}

struct GatedBwdWorkspace {
    Workspace lists, again;    // of dH and dxe; of the first projections, computed again
    uint16_t *dGU, *pre, *hid; // [R][2 h], [R][2 h], [R][h]
    size_t bytes, kept_bytes;  // kept_bytes: without what only first projections computed again need, which lies last
};
void layout_gated_bwd(const moe_shape &s, void *base, GatedBwdWorkspace *w)
{
    const int64_t R = moe_max_rows(&s);
    char *p = static_cast<char *>(base);
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char *at = p + off;
        off += align_up(bytes, 256);
        return at;
    };
    w->lists = w->again = Workspace{};
    w->lists.gp[0] = plan_gated(R, s.E, s.d_ff, s.d_model, false, false, R);
    w->lists.gp[1] = plan_gated(R, s.E, s.d_model, 2 * s.d_ff, false, true, R);
    w->again.gp[0] = plan_gated(R, s.E, gated_packed_columns(s.d_ff), s.d_model, true, true, R);
    w->again.gp[1] = w->lists.gp[1];
    for (int g = 0; g < 2; ++g)
        w->lists.items[g] = reinterpret_cast<WorkItem *>(take(sizeof(WorkItem) * w->lists.gp[g].max_items));
    const size_t Rh = static_cast<size_t>(R) * s.d_ff;
    w->dGU = reinterpret_cast<uint16_t *>(take(Rh * 4));
    w->kept_bytes = off;
    w->again.items[0] = reinterpret_cast<WorkItem *>(take(sizeof(WorkItem) * w->again.gp[0].max_items));
    w->again.items[1] = w->lists.items[1];
    w->pre = reinterpret_cast<uint16_t *>(take(Rh * 4));
    w->hid = reinterpret_cast<uint16_t *>(take(Rh * 2));
    w->bytes = off;
}

template <typename Kernel, typename... Args>
void launch_timed(Kernel kern, int grid, int threads, size_t lds, int stage, hipStream_t st, Args... args)
{
    hipEvent_t t0, t1;
    prof_kernel_events(stage, &t0, &t1);
    hipExtLaunchKernelGGL(kern, dim3(grid), dim3(threads), lds, st, t0, t1, 0, args...);
}

// f(activation)
template <typename F>
void with_activation(int act, F f)
{
    using std::integral_constant;
    switch (act) {
    case MOE_ACT_GELU_ERF: f(integral_constant<int, MOE_ACT_GELU_ERF>{}); break;
    case MOE_ACT_GELU_TANH: f(integral_constant<int, MOE_ACT_GELU_TANH>{}); break;
    case MOE_ACT_RELU: f(integral_constant<int, MOE_ACT_RELU>{}); break;
    case MOE_ACT_SILU: f(integral_constant<int, MOE_ACT_SILU>{}); break;
    default: f(integral_constant<int, MOE_ACT_IDENTITY>{});
    }
}

// H (and pre) of a bf16 layer
template <int ACT, bool KEEP>
void launch_first(const moe_shape &s, const uint16_t *xe, const uint16_t *W13p, uint16_t *H, uint16_t *pre, const GemmPlan &gp,
                  const WorkItem *items, const DirectTiles &direct, hipStream_t st)
{
    const int N = gated_packed_columns(s.d_ff), K = s.d_model, h = s.d_ff;
    if (!gp.w4) {
        auto kern = K % 64 == 0 ? gated_stream_kernel<ACT, KEEP, false> : gated_stream_kernel<ACT, KEEP, true>;
        launch_timed(kern, block_tile_grid(direct.rows, direct.E, 32, N / 32), 64, 0, kStageGemm1, st, xe, W13p,
                     reinterpret_cast<_Float16 *>(H), reinterpret_cast<_Float16 *>(pre), direct.offsets, direct.E, N, K, h);
        return;
    }
    auto shape = [&](auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        static PerDeviceOnce once[4];
        const int share = w4_run_share(gp.bm, K), blocks = w4_run_blocks(gp.max_items, share);
        auto run = [&](auto kern, PerDeviceOnce &o) {
            o.raise_lds(reinterpret_cast<const void *>(kern), static_cast<int>(kW4RunLds));
            launch_timed(kern, blocks, 256, kW4RunLds, kStageGemm1, st, xe, W13p, H, pre, items, gp.max_items, share, N, K, h);
        };
        auto tile = [&](auto kern, PerDeviceOnce &o, size_t lds) {
            o.raise_lds(reinterpret_cast<const void *>(kern), static_cast<int>(lds));
            launch_timed(kern, gp.max_items, 256, lds, kStageGemm1, st, xe, W13p, H, pre, items, N, K, h);
        };
        if (gp.bm == 256) run(gated_run_kernel<ACT, KEEP, TAIL, 256>, once[0]);
        else if (gp.bn == 256) run(gated_run_kernel<ACT, KEEP, TAIL, 128>, once[1]);
        else if (gp.deep) tile(gated_tile_kernel<ACT, KEEP, TAIL, true>, once[2], kW4Lds);
        else tile(gated_tile_kernel<ACT, KEEP, TAIL, false>, once[3], w4_lds(128, 128));
    };
    if (whole_stages(gp, K)) shape(std::false_type{});
    else shape(std::true_type{});
}

// fp32 tiles of 64 rows where they are a few per compute unit (32 / 64 rows a tile, us of the block: 896 tiles 124 / 128, 470 86 / 100, 1280
// 169 / 158, 1400 58 / 56, 2496 236 / 227, 5120 659 / 610).
bool tall_f32_tiles(int64_t rows, int E, int d_ff) { return (rows / 64 + E / 2) * ((d_ff + 31) / 32) >= 1200; }

void launch_first_gemm(const moe_shape &s, const void *xe, const void *W13p, void *H, void *pre, const GemmPlan &gp,
                       const WorkItem *items, const DirectTiles &direct, hipStream_t st)
{
    with_activation(s.act, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        auto f32 = [&](auto tmc) {
            constexpr int TM = decltype(tmc)::value;
            launch_timed(gated_f32_kernel<ACT, TM>, block_tile_grid(direct.rows, direct.E, 32 * TM, (s.d_ff + 31) / 32), 256, 0,
                         kStageGemm1, st, static_cast<const float *>(xe), static_cast<const float *>(W13p), static_cast<float *>(H),
                         direct.offsets, direct.E, s.d_ff, s.d_model);
        };
        if (s.dtype == MOE_F32 && tall_f32_tiles(direct.rows, direct.E, s.d_ff))
            f32(std::integral_constant<int, 2>{});
        else if (s.dtype == MOE_F32)
            f32(std::integral_constant<int, 1>{});
        else if (pre != nullptr)
            launch_first<ACT, true>(s, static_cast<const uint16_t *>(xe), static_cast<const uint16_t *>(W13p),
                                    static_cast<uint16_t *>(H), static_cast<uint16_t *>(pre), gp, items, direct, st);
        else
            launch_first<ACT, false>(s, static_cast<const uint16_t *>(xe), static_cast<const uint16_t *>(W13p),
                                     static_cast<uint16_t *>(H), nullptr, gp, items, direct, st);
    });
}

void launch_dh(const moe_shape &s, const uint16_t *dye, const uint16_t *W2, const uint16_t *pre, uint16_t *dGU,
               const GemmPlan &gp, const WorkItem *items, hipStream_t st)
{
    const int N = s.d_ff, K = s.d_model;
    with_activation(s.act, [&](auto act) {
        auto launch = [&](auto tail, auto bm) {
            constexpr int BM = decltype(bm)::value;
            auto kern = gated_dh_kernel<decltype(act)::value, decltype(tail)::value, BM>;
            constexpr size_t lds = w4_lds(BM, BM);
            static PerDeviceOnce once;
            once.raise_lds(reinterpret_cast<const void *>(kern), static_cast<int>(lds));
            launch_timed(kern, gp.max_items, 256, lds, kStageBwdDP, st, dye, W2, pre, dGU, items, N, K);
        };
        auto shape = [&](auto tail) {
            if (gp.bm == 256) launch(tail, std::integral_constant<int, 256>{});
            else launch(tail, std::integral_constant<int, 128>{});
        };
        if (K % 64 == 0) shape(std::false_type{});
        else shape(std::true_type{});
    });
}

void launch_dxe(const moe_shape &s, const uint16_t *dGU, const uint16_t *W13, uint16_t *dxe, const GemmPlan &gp,
                const WorkItem *items, hipStream_t st)
{
    const int N = s.d_model, K = 2 * s.d_ff;
    auto shape = [&](auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        static PerDeviceOnce once[4];
        const int share = w4_run_share(gp.bm, K), blocks = w4_run_blocks(gp.max_items, share);
        auto run = [&](auto kern, PerDeviceOnce &o) {
            o.raise_lds(reinterpret_cast<const void *>(kern), static_cast<int>(kW4RunLds));
            launch_timed(kern, blocks, 256, kW4RunLds, kStageBwdDxe, st, dGU, W13, dxe, items, gp.max_items, share, N, K);
        };
        auto tile = [&](auto kern, PerDeviceOnce &o, size_t lds) {
            o.raise_lds(reinterpret_cast<const void *>(kern), static_cast<int>(lds));
            launch_timed(kern, gp.max_items, 256, lds, kStageBwdDxe, st, dGU, W13, dxe, items, N, K);
        };
        if (gp.bm == 256) run(rows_bf16_run_kernel<TAIL, 256>, once[0]);
        else if (gp.bn == 256) run(rows_bf16_run_kernel<TAIL, 128>, once[1]);
        else if (gp.deep) tile(rows_bf16_tile_kernel<TAIL, true>, once[2], kW4Lds);
        else tile(rows_bf16_tile_kernel<TAIL, false>, once[3], w4_lds(128, 128));
    };
    if (whole_stages(gp, K)) shape(std::false_type{});
    else shape(std::true_type{});
}

// Everything that the calls below take: a gated row is 2 d_ff values, and the kernels' byte offsets inside a tile's 256 rows
// are 32 bits.
moe_status check_gated(const moe_shape *s, bool training)
{
    const moe_status rc = check_layer_shape(s);
    if (rc != MOE_OK) return rc;
    if (s->d_ff >= 1 << 20 || s->d_model >= 1 << 20) {
        set_error("gated block: d_model and d_ff below 2^20 (got %d, %d)", s->d_model, s->d_ff);
        return MOE_EUNSUPPORTED;
    }
    if (moe_max_rows(s) >= (1ll << 31) - 256) {
        set_error("gated block: %lld rows do not fit 31 bits", static_cast<long long>(moe_max_rows(s)));
        return MOE_EUNSUPPORTED;
    }
    if (training && s->dtype != MOE_BF16) {
        set_error("gated block: its backward pass and what it keeps are for bf16 layers");
        return MOE_EUNSUPPORTED;
    }
    return MOE_OK;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" {

size_t moe_gated_packed_bytes(const moe_shape *s)
{
    if (check_gated(s, false) != MOE_OK) return 0;
    const size_t per = static_cast<size_t>(s->E) * s->d_model;
    return s->dtype == MOE_F32 ? per * s->d_ff * 8 : per * gated_packed_columns(s->d_ff) * 2;
}

moe_status moe_pack_gated_weights(const moe_shape *s, const void *W13, const void *W2, void *W13p, void *W2p, void *stream)
{
    const moe_status rc = check_gated(s, false);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE_PTR(W13);
    MOE_REQUIRE_PTR(W2);
    MOE_REQUIRE_PTR(W13p);
    MOE_REQUIRE_PTR(W2p);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int d = s->d_model, h = s->d_ff;
    if (s->dtype == MOE_F32) {
        const size_t one = static_cast<size_t>(s->E) * d * h * 4;
        MOE_TRY_HIP(hipMemcpyAsync(W13p, W13, 2 * one, hipMemcpyDeviceToDevice, st));
        MOE_TRY_HIP(hipMemcpyAsync(W2p, W2, one, hipMemcpyDeviceToDevice, st));
        return MOE_OK;
    }
    const int NP = gated_packed_columns(h);
    hipLaunchKernelGGL(gated_pack_kernel<true>, dim3(ceil_div(NP, 64), ceil_div(d, 64), s->E), dim3(256), 0, st,
                       static_cast<const uint16_t *>(W13), static_cast<uint16_t *>(W13p), d, 2 * h, NP);
    hipLaunchKernelGGL(gated_pack_kernel<false>, dim3(ceil_div(d, 64), ceil_div(h, 64), s->E), dim3(256), 0, st,
                       static_cast<const uint16_t *>(W2), static_cast<uint16_t *>(W2p), h, d, d);
    MOE_TRY_HIP(hipGetLastError());
    return MOE_OK;
}

size_t moe_gated_workspace_bytes(const moe_shape *s)
{
    if (check_gated(s, false) != MOE_OK) return 0;
    GatedWorkspace w;
    layout_gated(*s, nullptr, &w);
    return w.bytes;
}

size_t moe_gated_kept_workspace_bytes(const moe_shape *s)
{
    if (check_gated(s, true) != MOE_OK) return 0;
    GatedWorkspace w;
    layout_gated(*s, nullptr, &w);
    return w.kept_bytes;
}

moe_status moe_gated_ffn(const moe_shape *s, const void *xe, const int32_t *offsets, const void *W13p, const void *W2p,
                         void *ye, void *pre, void *hid, void *workspace, void *stream)
{
    moe_status rc = check_gated(s, pre != nullptr || hid != nullptr);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE_PTR(xe);
    MOE_REQUIRE_PTR(offsets);
    MOE_REQUIRE_PTR(W13p);
    MOE_REQUIRE_PTR(W2p);
    MOE_REQUIRE_PTR(ye);
    MOE_OPTIONAL_PTR(pre);
    MOE_OPTIONAL_PTR(hid);
    MOE_REQUIRE_PTR(workspace);
    if ((pre == nullptr) != (hid == nullptr)) {
        set_error("moe_gated_ffn: pre and hid come together (both or neither)");
        return MOE_EINVAL;
    }
    GatedWorkspace w;
    layout_gated(*s, workspace, &w);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const DirectTiles direct{offsets, s->E, moe_max_rows(s)};
    const bool direct1 = takes_direct_tiles(*s, w.lists.gp[1]);
    if (!takes_direct_tiles(*s, w.lists.gp[0]) || !direct1) {
        prof_begin(kStageTiles, st);
        rc = launch_items(*s, 1, 1, offsets, nullptr, w.lists, st);
        prof_end(kStageTiles, st);
        if (rc != MOE_OK) return rc;
    }
    void *H = hid != nullptr ? hid : w.lists.hidden;
    launch_first_gemm(*s, xe, W13p, H, pre, w.lists.gp[0], w.lists.items[0], direct, st);
    return launch_second_gemm(*s, H, W2p, ye, w.lists.gp[1], direct1 ? nullptr : w.lists.items[1], direct, st);
}

size_t moe_gated_backward_workspace_bytes(const moe_shape *s)
{
    if (check_gated(s, true) != MOE_OK) return 0;
    GatedBwdWorkspace w;
    layout_gated_bwd(*s, nullptr, &w);
    return w.bytes;
}

size_t moe_gated_kept_backward_workspace_bytes(const moe_shape *s)
{
    if (check_gated(s, true) != MOE_OK) return 0;
    GatedBwdWorkspace w;
    layout_gated_bwd(*s, nullptr, &w);
    return w.kept_bytes;
}

moe_status moe_gated_gemm_kernel(const moe_shape *s, int32_t which, char *name, size_t len)
{
    if (name == nullptr || len == 0 || which < 0 || which > 5) {
        set_error("moe_gated_gemm_kernel: which must be in 0..5, name a buffer");
        return MOE_EINVAL;
    }
    const moe_status rc = check_gated(s, which > 1);
    if (rc != MOE_OK) return rc;
    const int64_t R = moe_max_rows(s);
    const int d = s->d_model, h = s->d_ff, NP = gated_packed_columns(h);
    auto put = [&](const char *kernel, int bm, int bn, const char *form) { std::snprintf(name, len, "%s %dx%d%s", kernel, bm, bn, form); };
    auto tiles = [&](const char *run, const char *tile, const GemmPlan &gp, int K) {
        const char *form = whole_stages(gp, K) ? gp.deep ? " deep" : "" : gp.deep ? " deep tail" : " tail";
        put(gp.bn == 256 ? run : tile, gp.bm, gp.bn, form);
    };
    if (which == 0 && s->dtype == MOE_F32) {
        put("gated_f32_kernel", tall_f32_tiles(R, s->E, h) ? 64 : 32, 32, "");
    } else if (which == 0) {
        const GemmPlan gp = plan_gated(R, s->E, NP, d, true, true, R);
        if (gp.w4) tiles("gated_run_kernel", "gated_tile_kernel", gp, d);
        else put("gated_stream_kernel", 32, 32, d % 64 == 0 ? "" : " tail");
    } else if (which == 1 && s->dtype == MOE_F32) {
        const GemmPlan gp = choose_gemm_plan(*s, 1, 1, s->T);
        put("grouped_gemm_f32_kernel", gp.bm, gp.bn, "");
    } else if (which == 1) {
        expert_gemm_kernel_name(*s, 1, name, len);
    } else if (which == 2) {
        const GemmPlan gp = plan_gated(R, s->E, h, d, false, false, R);
        put("gated_dh_kernel", gp.bm, gp.bn, d % 64 == 0 ? "" : " tail");
    } else if (which == 3) {
        const GemmPlan gp = plan_gated(R, s->E, d, 2 * h, false, true, R);
        tiles("rows_bf16_run_kernel", "rows_bf16_tile_kernel", gp, 2 * h);
    } else {
        const int M = which == 4 ? h : d, N = which == 4 ? d : 2 * h;
        if (wide_weight_grad_bf16(s->E, M, N, R)) put("wgrad_w4_kernel", 256, 256, "");
        else put("wgrad_gemm_kernel", 128, 128, "");
    }
    return MOE_OK;
}

moe_status moe_gated_ffn_backward(const moe_shape *s, const void *xe, const int32_t *offsets, const void *W13, const void *W2,
                                  const void *W13p, const void *pre, const void *hid, const void *dye, void *dxe, void *dW13,
                                  void *dW2, void *workspace, void *stream)
{
    moe_status rc = check_gated(s, true);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE_PTR(xe);
    MOE_REQUIRE_PTR(offsets);
    MOE_REQUIRE_PTR(W13);
    MOE_REQUIRE_PTR(W2);
    MOE_REQUIRE_PTR(W13p);
    MOE_OPTIONAL_PTR(pre);
    MOE_OPTIONAL_PTR(hid);
    MOE_REQUIRE_PTR(dye);
    MOE_REQUIRE_PTR(dxe);
    MOE_REQUIRE_PTR(dW13);
    MOE_REQUIRE_PTR(dW2);
    MOE_REQUIRE_PTR(workspace);
    if ((pre == nullptr) != (hid == nullptr)) {
        set_error("moe_gated_ffn_backward: pre and hid come together (both or neither)");
        return MOE_EINVAL;
    }
    GatedBwdWorkspace w;
    layout_gated_bwd(*s, workspace, &w);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t R = moe_max_rows(s);
    const int d = s->d_model, h = s->d_ff;
    rc = launch_items(*s, 1, 1, offsets, nullptr, w.lists, st);
    if (rc != MOE_OK) return rc;
    if (pre == nullptr) {
        // (writes the second list again, as it is)
        rc = launch_items(*s, 1, 1, offsets, nullptr, w.again, st);
        if (rc != MOE_OK) return rc;
        launch_first_gemm(*s, xe, W13p, w.hid, w.pre, w.again.gp[0], w.again.items[0], DirectTiles{offsets, s->E, R}, st);
        pre = w.pre;
        hid = w.hid;
    }
    const uint16_t *xeb = static_cast<const uint16_t *>(xe), *dyeb = static_cast<const uint16_t *>(dye);
    auto hidden_grads = [&]() {
        launch_dh(*s, dyeb, static_cast<const uint16_t *>(W2), static_cast<const uint16_t *>(pre), w.dGU, w.lists.gp[0],
                  w.lists.items[0], st);
    };
    auto input_grads = [&]() {
        launch_dxe(*s, w.dGU, static_cast<const uint16_t *>(W13), static_cast<uint16_t *>(dxe), w.lists.gp[1], w.lists.items[1], st);
    };
    auto weight_grad2 = [&](hipStream_t q) {
        launch_weight_grad_bf16(true, static_cast<const uint16_t *>(hid), dyeb, static_cast<uint16_t *>(dW2), offsets, s->E, h, d,
                                R, kStageBwdWgrad2, q);
    };
    auto weight_grad1 = [&](hipStream_t q) {
        launch_weight_grad_bf16(false, xeb, w.dGU, static_cast<uint16_t *>(dW13), offsets, s->E, d, 2 * h, R, kStageBwdWgrad1, q);
    };
    std::unique_lock<std::mutex> enqueue;
    // (Half as much work again as a plain layer of these sizes.  us of forward and backward pass in order / beside each other, rows
    // spread evenly (by 1 / rank), by rows x d_model x d_ff: 4e8 87 / 91 (88 / 89), 1.1e9 107 / 110 (113 / 119), 1.5e9 107 / 112 (123 / 128),
    // 1.6e9 148 / 142 (182 / 178); above the line, which lies at 1.8e9: 5.9e9 184 / 174, 6.4e9 240 / 240 (322 / 284), 1.6e10 545 / 456 (733 / 600),
    // 1.9e11 3213 / 3160 (4547 / 4306), 4e11 6997 / 6956 (12297 / 11999); past it, at 4.7e11: 5.5e11 8490 / 8696 (14358 / 14405), 1.9e12 28493 /
    // 29609.)
    SideStream *side = lend_side_stream(1.5 * static_cast<double>(R) * d * h, st, enqueue);
    if (side == nullptr) {
        hidden_grads();
        input_grads();
        weight_grad2(st);
        weight_grad1(st);
        MOE_TRY_HIP(hipGetLastError());
        return MOE_OK;
    }
    // dW2 beside dH, dW13 beside dxe
    auto enqueue_both = [&]() -> moe_status {
        MOE_TRY_HIP(hipEventRecord(side->dispatched, st));
        MOE_TRY_HIP(hipStreamWaitEvent(side->stream, side->dispatched, 0));
        hidden_grads();
        weight_grad2(side->stream);
        MOE_TRY_HIP(hipEventRecord(side->hidden, st));
        MOE_TRY_HIP(hipStreamWaitEvent(side->stream, side->hidden, 0));
        input_grads();
        weight_grad1(side->stream);
        return MOE_OK;
    };
    rc = enqueue_both();
    // (joined also after a failure part-way)
    hipError_t je = hipEventRecord(side->joined, side->stream);
    if (je == hipSuccess) je = hipStreamWaitEvent(st, side->joined, 0);
    if (rc != MOE_OK) return rc;
    if (je != hipSuccess) return hip_fail(je, "joining the side stream");
    MOE_TRY_HIP(hipGetLastError());
    return MOE_OK;
}

}  // extern "C"
