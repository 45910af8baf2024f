// Tiles of 256 x 256 of products of rows and weights in 8 bits (include/moe_q8.h): the linear map and the gated block's first
// projections on the loop of gemm_w4_run.h.
// Both epilogues pass their values through the wavefront's patch (W4Place), without a branch.
// Bound by the matrix cores, whose rate depends on what they multiply: 16384 x 4096 x 4096 2.4 to 2.6 POP/s of random codes (3.2 of zeros), 8192^3 2.8
// (3.6); instructions alone, from registers, reach 3.6 of random codes.  A stage of 64 x 2 codes takes 1.3 us.  Tiles of a short depth are bound by
// their epilogue: of a pair 2050 vector instructions, 256 of them exponentials and reciprocals, beside a single wavefront per SIMD, 5 us
// (8192 rows of 16 experts, 768 to 2 x 2048, 48 us, 1.07 POP/s; 32768 rows of 32 experts, 2048 to 2 x 8192, 960 to 1090 us, 2.0 to 2.3 POP/s).
#include "activation.h"
#include "gated.h"
#include "moe_q8.h"
#include "q8_product.h"

#include <algorithm>
#include <type_traits>

#include <hip/hip_ext.h>

namespace moe {
namespace {

#include "q8_product_device.h"
#include "gemm_w4_run.h"

constexpr int BM = 256, TM = BM / 32;

// The linear map.  Y32: y is fp32; RES: there is a residual, whose loads are kAhead steps of 16 rows and 64 columns ahead: all units
// reach their tiles' ends together, and wait for memory there (16384 x 4096 x 4096, GELU, bias, residual and y bf16: without the residual
// 247 us, two steps ahead 276; with a GeLU of two instructions less 242, one step ahead 275, two 268, three, with 20 registers spilled instead of
// up to 7, 273).
constexpr int kAhead = 2;
template <int ACT, bool Y32, bool RES, bool KTAIL>
__global__ __launch_bounds__(256, 1) void q8_run_kernel(Q8Args a)
{
    const Tiles<BM, 256> items(a.offsets, a.E, a.tiles);
    const ActForm form(a.act);
    struct Columns {                       // the tile's rows' scales; a lane's four columns of each half's 64
        float xs[TM];
        float ws[2][4], bias[2][4];
    };
    w4_run<kI8Operands, KTAIL, BM, 0>(a.x, a.w, items, nullptr, a.entries, a.share, a.N, a.K, nullptr, 1, 0,
        [&](const WorkItem &item, int wn, int) {
            Columns c;
            const int lane = lane_id(), wm = threadIdx.x / kWave & 1;
#pragma unroll
            for (int j = 0; j < TM; ++j) c.xs[j] = a.xs[min(item.row0 + wm * (BM / 2) + j * 16 + (lane & 15), item.row1 - 1)];
            const float *ws = a.ws + static_cast<size_t>(item.expert) * a.N;
            const float *bias = a.bias != nullptr ? a.bias + static_cast<size_t>(item.expert) * a.N : ws;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int n = min(item.n0 + wn * 128 + half * 64 + lane % 16 * 4, a.N - 4);
                const f32x4 s = *reinterpret_cast<const f32x4 *>(ws + n), b = *reinterpret_cast<const f32x4 *>(bias + n);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    c.ws[half][e] = s[e];
                    c.bias[half][e] = a.bias != nullptr ? b[e] : 0.0f;
                }
            }
            return c;
        },
        [&](auto &acc, const Columns &ahead, const WorkItem &item, const W4Place<BM> &place, auto landed) {
            const int lane = place.lane, row0 = item.row0 + place.wm * (BM / 2), n0 = item.n0 + place.wn * 128;
            const bool wide = a.res == kF32;
            // (a row past the tile's or a column past N lies past the resources; of the residual's two, which are of its two sizes, one is empty)
            const size_t first = static_cast<size_t>(row0) * a.N;
            // (the wavefront's 128 rows at most: 2^28 values, so that what lies past N lies past these)
            const unsigned values = static_cast<unsigned>(min(max(item.row1 - row0, 0), BM / 2)) * static_cast<unsigned>(a.N);
            const __amdgpu_buffer_rsrc_t ry = __builtin_amdgcn_make_buffer_rsrc(static_cast<char *>(a.y) + first * (Y32 ? 4 : 2), 0,
                                                                                values * (Y32 ? 4u : 2u), 0x00020000);
            char *const rbase = static_cast<char *>(const_cast<void *>(a.r)) + first * (wide ? 4 : 2);
            const __amdgpu_buffer_rsrc_t r32 = __builtin_amdgcn_make_buffer_rsrc(rbase, 0, wide ? values * 4u : 0u, 0x00020000);
            const __amdgpu_buffer_rsrc_t r16 = __builtin_amdgcn_make_buffer_rsrc(rbase, 0, wide ? 0u : values * 2u, 0x00020000);
            const int n = n0 + lane % 16 * 4, step4 = 4 * a.N;
            // value of the lane's first row in 16 rows `j`, half `half`; four rows on is step4 further
            auto at_of = [&](int j, int half) { return n + half * 64 < a.N ? (j * 16 + lane / 16) * a.N + n + half * 64 : 0x1ff00000; };
            u32x4 rw[kAhead][4];
            u32x2 rh[kAhead][4];
            auto ask = [&](auto stepc) {
                constexpr int step = decltype(stepc)::value, turn = step % kAhead;
                int at = at_of(step / 2, step % 2);
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    rw[turn][it] = __builtin_amdgcn_raw_buffer_load_b128(r32, at * 4, 0, 0);
                    rh[turn][it] = __builtin_amdgcn_raw_buffer_load_b64(r16, at * 2, 0, 0);
                    at += step4;
                }
            };
            if constexpr (RES) static_for<kAhead>(ask);
            static_for<2 * TM>([&](auto stepc) {
                constexpr int step = decltype(stepc)::value, j = step / 2, half = step % 2, turn = step % kAhead;
                lds_handover();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x4 v;
#pragma unroll
                    for (int c = 0; c < 4; ++c) v[c] = sum_of(acc[half * 4 + i][j][c]) * ahead.xs[j];
                    // (a row's 16-byte pieces XOR-swizzled with the row)
                    *reinterpret_cast<f32x4 *>(place.patch + place.fr * 256 + (((i * 4 + place.oct) ^ place.fr) << 4)) = v;
                }
                MOE_SB();
                if constexpr (step == 0) landed();
                lds_handover();
                MOE_SB();
                float v[4][4];
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const int row = it * 4 + lane / 16;
                    const f32x4 s = *reinterpret_cast<const f32x4 *>(place.patch + row * 256 + ((lane % 16 ^ row) << 4));
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        v[it][c] = activate<ACT>(form, __builtin_fmaf(s[c], ahead.ws[half][c], ahead.bias[half][c]));
                        if constexpr (RES)
                            v[it][c] += wide ? __uint_as_float(rw[turn][it][c])
                                             : a.res == kF16 ? f16_of(rh[turn][it][c / 2], c % 2) : b16_of(rh[turn][it][c / 2], c % 2);
                    }
                    if (it % 2 == 1) MOE_SB();
                }
                // (y may be r: what is asked for is of other rows or columns than what is stored)
                if constexpr (RES && step + kAhead < 2 * TM) ask(std::integral_constant<int, step + kAhead>{});
                int at = at_of(j, half);
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    if constexpr (Y32) {
                        const u32x4 o = {__float_as_uint(v[it][0]), __float_as_uint(v[it][1]), __float_as_uint(v[it][2]), __float_as_uint(v[it][3])};
                        __builtin_amdgcn_raw_buffer_store_b128(o, ry, at * 4, 0, 0);
                    } else {
                        const u32x2 h = {pack_16(kF16, v[it][0], v[it][1]), pack_16(kF16, v[it][2], v[it][3])};
                        const u32x2 b = {pack_16(kB16, v[it][0], v[it][1]), pack_16(kB16, v[it][2], v[it][3])};
                        __builtin_amdgcn_raw_buffer_store_b64(a.type == kF16 ? h : b, ry, at * 2, 0, 0);
                    }
                    at += step4;
                }
                MOE_SB();
            });
        });
}

// The block's first projections: acc[2 p] and acc[2 p + 1] of a lane are gate and value of the same four columns.
template <int ACT, bool KTAIL>
__global__ __launch_bounds__(256, 1) void q8_gated_run_kernel(Q8Args a)
{
    const Tiles<BM, 256> items(a.offsets, a.E, a.tiles);
    const ActForm form(a.act);
    struct Scales {
        float xs[TM];
        float gs[4][4], us[4][4];
    };
    w4_run<kI8Operands, KTAIL, BM, 0, true>(a.x, a.w, items, nullptr, a.entries, a.share, a.N, a.K, a.row_src, a.row_div, a.a_rows,
        [&](const WorkItem &item, int wn, int oct) {
            Scales c;
            const int lane = lane_id(), wm = threadIdx.x / kWave & 1;
            const int32_t *src = a.row_src != nullptr ? a.row_src : a.offsets;
            const int div = a.row_src != nullptr ? a.row_div : 1;
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                const int row = min(item.row0 + wm * (BM / 2) + j * 16 + (lane & 15), item.row1 - 1);
                const int from = src[a.row_src != nullptr ? row : 0] / div;
                c.xs[j] = a.xs[a.row_src != nullptr ? from : row];
            }
            const float *gs = a.ws + static_cast<size_t>(item.expert) * a.N;
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const int n = min(item.n0 / 2 + wn * 64 + p * 16 + oct * 4, a.h - 4);      // (h is a multiple of 16)
                const f32x4 g = *reinterpret_cast<const f32x4 *>(gs + n), u = *reinterpret_cast<const f32x4 *>(gs + a.h + n);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    c.gs[p][e] = g[e];
                    c.us[p][e] = u[e];
                }
            }
            return c;
        },
        [&](auto &acc, const Scales &ahead, const WorkItem &item, const W4Place<BM> &place, auto landed) {
            const int row0 = item.row0 + place.wm * (BM / 2), col = item.n0 / 2 + place.wn * 64 + place.lane % 8 * 8;
            const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
                static_cast<uint16_t *>(a.y) + static_cast<size_t>(row0) * a.h, 0,
                static_cast<unsigned>(max(item.row1 - row0, 0)) * static_cast<unsigned>(a.h) * 2u, 0x00020000);
            int at = col < a.h ? (place.lane / 8 * a.h + col) * 2 : 0x7f000000;
            const int step8 = col < a.h ? 16 * a.h : 0;
            static_for<TM>([&](auto jc) {
                constexpr int j = decltype(jc)::value;
                lds_handover();
                static_for<4>([&](auto pc) {
                    constexpr int p = decltype(pc)::value;
                    f16x4 o;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float g = sum_of(acc[2 * p][j][c]) * ahead.xs[j] * ahead.gs[p][c];
                        const float u = sum_of(acc[2 * p + 1][j][c]) * ahead.xs[j] * ahead.us[p][c];
                        o[c] = to_f16(activate<ACT>(form, g) * u);
                        if constexpr (ACT == kForm) MOE_SB();      // (four at a time spill registers)
                    }
                    *reinterpret_cast<f16x4 *>(place.at(p, 0)) = o;
                    MOE_SB();
                });
                if constexpr (j == 0) landed();
                // 16 rows of 64 columns, eight to a row's line
                lds_handover();
                MOE_SB();
#pragma unroll
                for (int it = 0; it < 2; ++it) {
                    const int row = it * 8 + place.lane / 8;
                    const u32x4 q = *reinterpret_cast<const u32x4 *>(place.patch + row * 256 + ((place.lane % 8 ^ row) << 4));
                    __builtin_amdgcn_raw_buffer_store_b128(q, rs, at, 0, 0);
                    at += step8;
                }
                MOE_SB();
            });
        },
        a.h);
}

}  // namespace

void launch_q8_run(bool pair, const Q8Args &args, int64_t entries, bool whole, int stage, hipStream_t st)
{
    Q8Args a = args;
    a.share = w4_run_share(BM, a.K);
    const int blocks = w4_run_blocks(static_cast<int>(entries), a.share);
    auto with_tail = [&](auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        if (pair) {
            with_activation<MOE_ACT_GELU_ERF, MOE_ACT_SILU>(a.act, [&](auto act) {
                launch_product_kernel<q8_gated_run_kernel<decltype(act)::value, TAIL>>(a, blocks, kW4RunLds, stage, st);
            });
            return;
        }
        auto launch = [&](auto y32, auto actc) {
            constexpr bool Y32 = decltype(y32)::value;
            constexpr int ACT = decltype(actc)::value;
            if (a.r != nullptr) launch_product_kernel<q8_run_kernel<ACT, Y32, true, TAIL>>(a, blocks, kW4RunLds, stage, st);
            else launch_product_kernel<q8_run_kernel<ACT, Y32, false, TAIL>>(a, blocks, kW4RunLds, stage, st);
        };
        if (a.type == kF32) with_activation<kGeluErf32, MOE_ACT_IDENTITY>(a.act, [&](auto act) { launch(std::true_type{}, act); });
        else with_activation<MOE_ACT_GELU_ERF, MOE_ACT_IDENTITY>(a.act, [&](auto act) { launch(std::false_type{}, act); });
    };
    if (whole) with_tail(std::false_type{});
    else with_tail(std::true_type{});
}

}  // namespace moe
