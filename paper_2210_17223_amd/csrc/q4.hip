// Products with weights held as 4-bit codes with group scales and zeros (include/moe_gated.h): one linear map, and the
// gated feed-forward block on them.
//
// The codes go from memory into registers and from there into the matrix instruction: eight codes of a lane become eight
// 16-bit numbers in place, by masks and an exponent (the conversion of narrow integers by their place in a number's digits that
// Kim, Henry, Fahim and Hassan Awadalla give in "Who Says Elephants Can't Run", 2022): in bf16 2^-16 (16 + q), in fp16
// 1024 + q.  Products and sums over a group are then exact but for fp32's roundings, and a group's sum is scaled in fp32:
//   bf16   sum (q - z) x = sum (16 + q) x - (16 + z) sum x, with sum x from one more matrix instruction against ones
//          (shared by all of a wavefront's columns).  16 is the least that an exponent can add: the code is then the first
//          four of the seven digits behind the point.  Against 128 + q, whose code is the last four and needs no shift for one
//          of its four pairs, sums that cancel keep three more bits, for one instruction in eight of the widening.
//          Codes and ones are over 2^16, which the result is multiplied by, since bf16 rows have fp32's range and a group's 128
//          terms of up to 31 x (and 271 sum x: zeros are bytes) would pass it from |x| = 1e34 on.
//   fp16   q - z by one packed subtraction (exact), no correction
#include "activation.h"
#include "block_tile.h"
#include "gated.h"
#include "moe_gated.h"

#include <algorithm>
#include <type_traits>
#include <utility>

#include <hip/hip_ext.h>

namespace moe {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;

#include "gemm_w4.h"

enum { kXBf16 = 1, kXF16 = 2 };
enum { kOutF32 = 0, kOutF16, kOutGated };

template <int... I, typename F>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F f)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void unrolled(F f)
{
    each_of(std::make_integer_sequence<int, N>{}, f);
}

// Eight codes of a dword, c0 lowest, as eight 16-bit numbers in the order c0 c4 c1 c5 c2 c6 c3 c7.  exponent: exponent_of<XT>()
// in a vector register (an instruction takes one constant, and masking and setting the exponent is one instruction then).
template <int XT>
__device__ __forceinline__ uint32_t exponent_of()
{
    uint32_t e = XT == kXBf16 ? 0x39803980u : 0x64006400u;
    asm volatile("" : "+v"(e));
    return e;
}
constexpr uint32_t kOnes = 0x37803780u;   // two times 2^-16 in bf16
template <int XT>
constexpr float kBack = XT == kXBf16 ? 65536.0f : 1.0f;
template <int XT>
__device__ __forceinline__ u32x4 widen(uint32_t w, uint32_t exponent, f16x2 minus, f16x2 minus16)
{
    if constexpr (XT == kXBf16) {
        auto part = [&](uint32_t v) { return (v & 0x00780078u) | exponent; };
        return (u32x4){part(w << 3), part(w >> 1), part(w >> 5), part(w >> 9)};
    } else {
        // low four bits of a byte: 1024 + q; high: 1024 + 16 q, a sixteenth of which is 64 + q
        const f16x2 sixteenth = {static_cast<_Float16>(0.0625f), static_cast<_Float16>(0.0625f)};
        auto low = [&](uint32_t v) {
            return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, (v & 0x000f000fu) | exponent) + minus);
        };
        auto high = [&](uint32_t v) {
            return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (v & 0x00f000f0u) | exponent),
                                                                          sixteenth, minus16));
        };
        return (u32x4){low(w), high(w), low(w >> 8), high(w >> 8)};
    }
}
// eight values of x in that order
__device__ __forceinline__ u32x4 reorder(const u32x4 &v)
{
    return (u32x4){__builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[2], v[0], 0x07060302u),
                   __builtin_amdgcn_perm(v[3], v[1], 0x05040100u), __builtin_amdgcn_perm(v[3], v[1], 0x07060302u)};
}
template <int XT>
__device__ __forceinline__ f32x4 multiply(const u32x4 &x, const u32x4 &w, const f32x4 &c)
{
    if constexpr (XT == kXBf16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, w), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, w), c, 0, 0, 0);
}

// Four dwords of a lane, 32 codes of its column from k = 32 oct on, to the order in which one instruction's k lie in one
// group (oct = lane / 16): of 128 nothing to do; of 64 the halves of the wavefront exchange, of 32 also the rows of a half.
// Dword j then holds eight codes from k_of<G>(j, oct) on.
template <int G>
__device__ __forceinline__ void regroup(u32x4 &w)
{
    auto swap32 = [](uint32_t &a, uint32_t &b) {
        const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
        a = r[0];
        b = r[1];
    };
    auto swap16 = [](uint32_t &a, uint32_t &b) {
        const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
        a = r[0];
        b = r[1];
    };
    uint32_t v[4] = {w[0], w[1], w[2], w[3]};
    if constexpr (G < 128) {
        swap32(v[0], v[2]);
        swap32(v[1], v[3]);
    }
    if constexpr (G < 64) {
        swap16(v[0], v[1]);
        swap16(v[2], v[3]);
    }
    w = (u32x4){v[0], v[1], v[2], v[3]};
}
template <int G>
__device__ __forceinline__ int k_of(int j, int oct)
{
    if constexpr (G == 128) return oct * 32 + j * 8;
    else if constexpr (G == 64) return (j >> 1) * 64 + (oct & 1) * 32 + (oct >> 1) * 16 + (j & 1) * 8;
    else return j * 32 + oct * 8;
}

template <int BYTES>
struct Run {                               // BYTES consecutive bytes, from an address of any alignment
    uint32_t w[(BYTES + 3) / 4];
    __device__ __forceinline__ void load(const void *p)
    {
        if constexpr (BYTES == 2) {
            uint16_t v;
            __builtin_memcpy(&v, p, 2);
            w[0] = v;
        } else {
            __builtin_memcpy(w, p, BYTES);
        }
    }
    __device__ __forceinline__ void set16(int i, uint32_t v) { w[i / 2] = i % 2 == 0 ? v : w[i / 2] | (v << 16); }
    __device__ __forceinline__ void set8(int i, uint32_t v) { w[i / 4] = i % 4 == 0 ? v : w[i / 4] | (v << (i % 4 * 8)); }
    // what the lanes of quarter Q of the wavefront hold, in all of them (of the same place in their quarters)
    template <int Q>
    __device__ __forceinline__ Run quarter() const
    {
        Run out;
#pragma unroll
        for (int i = 0; i < (BYTES + 3) / 4; ++i) {
            const auto h = __builtin_amdgcn_permlane32_swap(w[i], w[i], false, false);
            const uint32_t v = h[Q / 2];
            const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
            out.w[i] = r[Q % 2];
        }
        return out;
    }
    __device__ __forceinline__ float half(int i) const
    {
        return static_cast<float>(__builtin_bit_cast(f16x2, w[i / 2])[i % 2]);
    }
    __device__ __forceinline__ uint32_t byte(int i) const { return (w[i / 4] >> (i % 4 * 8)) & 0xffu; }
};

struct Q4Args {
    const uint16_t *x;
    const int32_t *offsets;
    const uint8_t *q, *zero;
    const uint16_t *scale;
    void *out;
    int E, N, K, kind, act;                // kind kOut...; kOutGated: N = 2 h rows of codes, out [rows, h]
    int tiles;                             // column tiles of an expert
    const float *row_scale;                // of the block's first product on many rows: what x was divided by
    bool reorder_out;                      // kOutGated: out in the codes' order, for the second product
};

__device__ __forceinline__ float gated_by(int act, float g, float u)
{
    switch (act) {
    case MOE_ACT_GELU_ERF: return gate_value<MOE_ACT_GELU_ERF>(g) * u;
    case MOE_ACT_GELU_TANH: return gate_value<MOE_ACT_GELU_TANH>(g) * u;
    case MOE_ACT_RELU: return gate_value<MOE_ACT_RELU>(g) * u;
    case MOE_ACT_SILU: return gate_value<MOE_ACT_SILU>(g) * u;
    default: return g * u;
    }
}

// ---------------------------------------------------------------- few rows per expert
// The time is that of streaming the codes once.  A block owns 16 NT columns of one expert, its wavefronts share out the
// depth in steps of 256 (a 128-byte line of every column's codes) and add up through LDS in a fixed order; rows are taken XR at
// a time.
// What bounded it first was the address unit, which takes a cycle for every 64 bytes that four neighbouring lanes do not
// share, and neighbouring lanes hold neighbouring columns (or rows of x): 64 cycles for each KiB, and x is four loads beside
// one of codes, the scales and zeros two more (64 rows, 8 experts of 4096 x 14336, group 64: busy for 81 % of 180 us).  So
// x and the codes are loaded line by line, pass through the wavefront's own LDS, x in the codes' order, and are read from there
// as the instruction wants them; and of scales and zeros a lane loads one of four steps, which the quarters of the wavefront
// then hand round.
// Loads are waited for in the order of their issue: x of the next step goes out before the codes of the one behind it.
// 2 rows, 8 experts, 4096 x 14336, group 128, the block's two products: 25 + 14 us, 5 TB/s of codes from the caches' side, 3.8 where
// none are left there; 64 rows, group 64 with zeros, 194 to 200 us a pass, 3.9 TB/s, the issue of vector instructions beside the loads.
// KTAIL: K is not a multiple of 256.
template <int XT, int G, bool ZEROS, int NT, int XR, bool KTAIL>
__global__ __launch_bounds__(512) void q4_stream_kernel(Q4Args a)
{
    constexpr int GROUPS = 256 / G, PER = 4 / (128 / G);     // groups of a step; dwords of 128 k and one group
    constexpr int XP = XR / 2, PITCH = 528, CODES = 144;     // pieces of x per lane; bytes of a row of x, of codes in LDS
    const int expert = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles;
    const int r0 = a.offsets[expert], r1 = a.offsets[expert + 1];
    if (r0 >= r1) return;
    const int lane = lane_id(), fr = lane & 15, oct = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
    // [waves] of a step's x and codes, and then of the sums [NT][4][64]
    constexpr int XS = XR * PITCH, OWN = XS + NT * 16 * CODES;
    static_assert(OWN >= NT * 1024, "the sums lie there, too");
    extern __shared__ __attribute__((aligned(16))) char shared[];
    char *const own = shared + wave * OWN;
    const bool gated = a.kind == kOutGated;
    const int half = gated ? NT / 2 : NT, width = gated ? a.N / 2 : a.N, col0 = tile * half * 16;
    const int KG = a.K / G, KB = a.K / 2;
    // group t's first row of codes, and the rows it has (past the last column: one, again)
    auto first_row = [&](int t) {
        return static_cast<size_t>(expert) * a.N + min(col0 + t % half * 16, width - 1) + (t >= half ? width : 0);
    };
    auto rows_of = [&](int t) { return min(max(width - col0 - t % half * 16, 1), 16); };
    const uint32_t exponent = exponent_of<XT>();
    // codes: lane l loads 16 bytes of row l / 8 of each eight
    const int q_at = (lane >> 3) * KB + (lane & 7) * 16;
    char *const q_to = own + XS + (lane >> 3) * CODES + (lane & 7) * 16;
    const char *const q_from = own + XS + fr * CODES + oct * 16;
    unsigned g_at[NT];                                       // the lane's row of groups
#pragma unroll
    for (int t = 0; t < NT; ++t) g_at[t] = static_cast<unsigned>(min(fr, rows_of(t) - 1)) * KG;
    const int steps = a.K / 256;
    const int s0 = steps * wave / waves, s1 = steps * (wave + 1) / waves;
    // x: lane l loads 16 bytes of row l / 32 of each two
    const int x_at = (lane >> 5) * a.K * 2 + (lane & 31) * 16;
    char *const x_to = own + (lane >> 5) * PITCH + (lane & 31) * 16;
    const char *const x_from = own + fr % XR * PITCH;

    for (int row0 = r0; row0 < r1; row0 += XR) {
        // (rows past the expert's last one: zeros that no load fetches)
        const __amdgpu_buffer_rsrc_t rsx = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint16_t *>(a.x) + static_cast<size_t>(row0) * a.K, 0, static_cast<unsigned>(min(r1 - row0, XR)) * a.K * 2u, 0x00020000);
        f32x4 total[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) total[t] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
        u32x4 code[2][NT][2], xr[XP];
        Run<GROUPS * 2> sc[2][NT];                           // of the step s0 + 4 c + oct, for two c
        Run<GROUPS> zr[2][NT];
        auto load_x = [&](int s) {
#pragma unroll
            for (int i = 0; i < XP; ++i)
                xr[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsx, x_at + i * 4 * a.K, s * 512, 0));
        };
        auto load_codes = [&](auto uc, int s) {
            constexpr int u = decltype(uc)::value;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
                    const_cast<uint8_t *>(a.q) + first_row(t) * KB + s * 128, 0, static_cast<unsigned>(max(rows_of(t) * KB - s * 128, 0)), 0x00020000);
#pragma unroll
                for (int b = 0; b < 2; ++b)
                    code[u][t][b] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, q_at + b * 8 * KB, 0, 0));
            }
        };
        auto load_scales = [&](auto cc, int s) {             // of the steps s .. s + 3
            constexpr int c = decltype(cc)::value;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const unsigned at = g_at[t] + static_cast<unsigned>(min(s + oct, s1 - 1)) * GROUPS;
                sc[c][t].load(reinterpret_cast<const char *>(a.scale + first_row(t) * KG) + at * 2u);
                if constexpr (ZEROS) zr[c][t].load(a.zero + first_row(t) * KG + at);
            }
        };
        auto codes_into_lds = [&](auto uc) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int b = 0; b < 2; ++b) *reinterpret_cast<u32x4 *>(q_to + (t * 2 + b) * 8 * CODES) = code[decltype(uc)::value][t][b];
        };
        auto x_into_lds = [&]() {
#pragma unroll
            for (int i = 0; i < XP; ++i) *reinterpret_cast<u32x4 *>(x_to + i * 2 * PITCH) = reorder(xr[i]);
        };
        // the step's sums, with scales s and zeros z (every lane's own)
        auto use = [&](auto &s, auto &z) {
            const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
            const u32x4 ones = {kOnes, kOnes, kOnes, kOnes};
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                u32x4 xf[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) xf[j] = *reinterpret_cast<const u32x4 *>(x_from + (b * 128 + k_of<G>(j, oct)) * 2);
                f32x4 xsum[GROUPS / 2];
                if constexpr (XT == kXBf16) {
#pragma unroll
                    for (int g = 0; g < GROUPS / 2; ++g) {
                        xsum[g] = none;
#pragma unroll
                        for (int j = 0; j < PER; ++j) xsum[g] = multiply<XT>(xf[g * PER + j], ones, xsum[g]);
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    u32x4 w = *reinterpret_cast<const u32x4 *>(q_from + t * 16 * CODES + b * 64);
                    regroup<G>(w);
#pragma unroll
                    for (int g = 0; g < GROUPS / 2; ++g) {
                        const float sv = s[t].half(b * (GROUPS / 2) + g);
                        const float zv = ZEROS ? static_cast<float>(z[t].byte(b * (GROUPS / 2) + g)) : 8.0f;
                        const _Float16 m1 = static_cast<_Float16>(-1024.0f - zv), m16 = static_cast<_Float16>(-64.0f - zv);
                        f32x4 part = none;
#pragma unroll
                        for (int j = 0; j < PER; ++j)
                            part = multiply<XT>(xf[g * PER + j],
                                                widen<XT>(w[g * PER + j], exponent, (f16x2){m1, m1}, (f16x2){m16, m16}), part);
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            float v = part[c];
                            if constexpr (XT == kXBf16) v = __builtin_fmaf(-16.0f - zv, xsum[g][c], v);
                            total[t][c] = __builtin_fmaf(sv, v, total[t][c]);
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);           // (half a step's numbers at a time)
            }
        };
        using std::integral_constant;
        if (s0 < s1) {
            // (past the last step: the last one again, never used)
            load_scales(integral_constant<int, 0>{}, s0);
            load_codes(integral_constant<int, 0>{}, s0);
            load_x(s0);
            load_codes(integral_constant<int, 1>{}, min(s0 + 1, s1 - 1));
            for (int s = s0; s < s1; s += 8) {
                unrolled<8>([&](auto ic) {
                    constexpr int i = decltype(ic)::value, c = i / 4;
                    if (s + i >= s1) return;
                    lds_handover();
                    x_into_lds();
                    codes_into_lds(integral_constant<int, i % 2>{});
                    load_x(min(s + i + 1, s1 - 1));
                    load_codes(integral_constant<int, i % 2>{}, min(s + i + 2, s1 - 1));
                    if constexpr (i % 4 == 0) load_scales(integral_constant<int, 1 - c>{}, min(s + i + 4, s1 - 1));
                    Run<GROUPS * 2> mine[NT];
                    Run<GROUPS> zeros[NT];
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        mine[t] = sc[c][t].template quarter<i % 4>();
                        if constexpr (ZEROS) zeros[t] = zr[c][t].template quarter<i % 4>();
                    }
                    lds_handover();
                    use(mine, zeros);
                });
            }
        }
        if constexpr (KTAIL) {
            // what is left of K, in the last wavefront: groups past it have no scale, codes and x past it read as zeros
            // or the next row's codes against zeros
            if (wave == waves - 1) {
                Run<GROUPS * 2> mine[NT];
                Run<GROUPS> zeros[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) {
                        const bool there = steps * GROUPS + g < KG;
                        const unsigned at = g_at[t] + min(steps * GROUPS + g, KG - 1);
                        mine[t].set16(g, there ? (a.scale + first_row(t) * KG)[at] : 0u);
                        if constexpr (ZEROS) zeros[t].set8(g, (a.zero + first_row(t) * KG)[at]);
                    }
                }
                load_codes(integral_constant<int, 0>{}, steps);
#pragma unroll
                for (int i = 0; i < XP; ++i)
                    xr[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                        rsx, steps * 256 + (lane & 31) * 8 < a.K ? x_at + i * 4 * a.K + steps * 512 : 0x7ffffff0, 0, 0));
                lds_handover();
                x_into_lds();
                codes_into_lds(integral_constant<int, 0>{});
                lds_handover();
                use(mine, zeros);
            }
        }

        // total[t][c]: row row0 + 4 oct + c, column fr of group t
        // (over x, whose reads are through)
        lds_handover();
        float *mine = reinterpret_cast<float *>(own);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c) mine[(t * 4 + c) * 64 + lane] = total[t][c] * kBack<XT>;
        __syncthreads();
        const int rows = min(r1 - row0, XR), cols = half * 16;
        auto add_up = [&](int row, int t, int n) {
            const int at = (t * 4 + row % 4) * 64 + row / 4 * 16 + n;
            float v = 0.0f;
            for (int w = 0; w < waves; ++w) v += reinterpret_cast<const float *>(shared + w * OWN)[at];
            return v;
        };
        for (int i = threadIdx.x; i < rows * cols; i += blockDim.x) {
            const int row = i / cols, c = i % cols;
            if (col0 + c >= width) continue;
            const size_t at = static_cast<size_t>(row0 + row) * width + col0 + c;
            const float v = add_up(row, c / 16, c % 16);
            if (gated) static_cast<_Float16 *>(a.out)[at] = static_cast<_Float16>(gated_by(a.act, v, add_up(row, c / 16 + half, c % 16)));
            else if (a.kind == kOutF16) static_cast<_Float16 *>(a.out)[at] = static_cast<_Float16>(v);
            else static_cast<float *>(a.out)[at] = v;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- many rows per expert
// Row of the expert's codes that lies in row i of a tile's 128, of wavefronts of TN column groups each: of a gated tile half of
// a wavefront's groups are gates, half the values of the same columns.
template <int TN>
__device__ __forceinline__ int tile_code_row(bool gated, int i, int col0, int width)
{
    if (!gated) return min(col0 + i, width - 1);
    const int w = i / (16 * TN), t = i / 16 % TN;
    return min(col0 + w * (8 * TN) + t % (TN / 2) * 16 + i % 16, width - 1) + (t >= TN / 2 ? width : 0);
}
// Where element e of eight lies in the codes' order
__device__ __forceinline__ int widened_place(int e) { return (e & ~7) | (e & 3) << 1 | (e >> 2 & 1); }

// LDS of the tile kernels' four wavefronts that work on a stage together
constexpr int tile_lds(int bm, int bn, int group)
{
    return bm * 272 + bn * 80 + 128 / group * bn * 8;
}
constexpr int ready_lds(int bm, int bn, int group)
{
    const int stages = 2 * bm * 256 + bn * 64 + 128 / group * bn * 8, tile = bm * (bn + 8) * 2;
    return stages > tile ? stages : tile;
}
// Where KS times NT threads share out a tile's depth, stage by stage in turn: the first NT add up all sums, in a fixed
// order (through LDS, behind a barrier after its last use).  False: not one of them.
template <int KS, int NT, int TN, int TM>
__device__ __forceinline__ bool join(f32x4 (&total)[TN][TM], char *shared, int pitch, int part_of, int tid)
{
    if constexpr (KS > 1) {
        if (part_of > 0) {
            f32x4 *const out = reinterpret_cast<f32x4 *>(shared + part_of * pitch) + tid;
#pragma unroll
            for (int i = 0; i < TN * TM; ++i) out[i * NT] = total[i / TM][i % TM];
        }
        __syncthreads();
        if (part_of > 0) return false;
#pragma unroll
        for (int p = 1; p < KS; ++p) {
            const f32x4 *const in = reinterpret_cast<const f32x4 *>(shared + p * pitch) + tid;
#pragma unroll
            for (int i = 0; i < TN * TM; ++i) {
                const f32x4 v = in[i * NT];
#pragma unroll
                for (int c = 0; c < 4; ++c) total[i / TM][i % TM][c] += v[c];
            }
        }
    }
    return true;
}

// The linear map on tiles of BM rows x BN columns: of 128 columns four wavefronts of 64 x 64 (BM = 128), 64 x 32 or 32 x 32, of
// 32 columns one.  Stages of 128: x (in the codes' order), codes, scales and zeros of the next one are on their way in registers
// while this one, in LDS, is multiplied; KS times as many wavefronts, or several blocks, of a compute unit take turns at that.  A
// group's sums have accumulators of their own; behind the group they are scaled into the totals, four instructions for each tile
// of 16 x 16 and group beside its G / 32 matrix instructions (and in bf16 four more for the zeros).  Each wavefront widens its own
// columns' codes, seven instructions for eight of them, which feed BM / 32 matrix instructions: bound by the issue of vector
// instructions, and with few tiles by the compute units that have none.  4096 x 4096, group 128: 64 rows 12 us, 160 rows 20 us,
// 1000 rows 63 us (530 TFLOP/s); 8192 x 8192, 300 rows 91 us, from fp16 6000 rows 1047 us (770 TFLOP/s).
template <int XT, int G, bool ZEROS, int BM, int BN, int KS>
__global__ __launch_bounds__(2 * BN * KS, KS == 4 && BN == 128 ? 4 : 2) void q4_tile_kernel(Q4Args a)
{
    constexpr int NT = 2 * BN, WM = BM / 64 > 1 ? 2 : 1, WN = NT / kWave / WM, TM = BM / WM / 16, TN = BN / 16 / WN;
    constexpr int GS = 128 / G, PER = 4 / GS;                // groups of a stage, dwords of 128 k and one group
    constexpr int XPITCH = 272, QPITCH = 80;                 // bytes of a row in LDS
    constexpr int XV = BM * 16 / NT;                         // 16-byte pieces of x per thread and stage
    constexpr int Q_AT = BM * XPITCH, S_AT = Q_AT + BN * QPITCH;
    static_assert(KS == 1 || tile_lds(BM, BN, G) >= BM * BN * 4, "the sums lie there, too");
    extern __shared__ __attribute__((aligned(16))) char all_shared[];
    const int part_of = __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
    char *const shared = all_shared + part_of * tile_lds(BM, BN, G);
    const int tid = threadIdx.x % NT, lane = tid & 63, fr = lane & 15, oct = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % WM, wn = wave / WM;
    const int width = a.N, KG = a.K / G, KB = a.K / 2;

    int expert, row0, row1, col0;
    if (!block_tile<BM>(a.offsets, a.E, a.tiles, blockIdx.x, expert, row0, row1, col0)) return;
    col0 *= BN;

    // staging: piece p = tid + NT q; x: row p / 16 of the tile, codes: row p / 4
    const __amdgpu_buffer_rsrc_t rsx = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t *>(a.x) + static_cast<size_t>(row0) * a.K, 0, static_cast<unsigned>(row1 - row0) * a.K * 2u, 0x00020000);
    auto code_row = [&](int i) { return min(col0 + i, width - 1); };
    const uint8_t *q_src[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int p = tid + NT * q;
        q_src[q] = a.q + (static_cast<size_t>(expert) * a.N + code_row(p / 4)) * KB;
    }
    const size_t g_row = (static_cast<size_t>(expert) * a.N + code_row(tid % BN)) * KG;   // threads < BN: scales, others: zeros
    u32x4 xr[XV], qr[2];
    Run<GS * 2> gr;
    auto load = [&](int s) {
#pragma unroll
        for (int q = 0; q < XV; ++q) {
            // (offsets are unsigned: 128 rows of 2^24 values are nearly 2^32 bytes, and what lies past K lies past those)
            const unsigned p = tid + NT * q, k = s * 128 + p % 16 * 8, K = a.K;
            xr[q] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsx, k < K ? (p / 16 * K + k) * 2 : 0xfffffff0u, 0, 0));
        }
#pragma unroll
        for (int q = 0; q < 2; ++q)
            qr[q] = *reinterpret_cast<const u32x4 *>(q_src[q] + min(s * 64 + (tid + NT * q) % 4 * 16, KB - 16));
        if (tid < BN) {
            if (s * GS + GS <= KG) {
                gr.load(a.scale + g_row + s * GS);
            } else {
#pragma unroll
                for (int g = 0; g < GS; ++g) gr.set16(g, s * GS + g < KG ? a.scale[g_row + min(s * GS + g, KG - 1)] : 0u);
            }
        } else if (ZEROS) {
#pragma unroll
            for (int g = 0; g < GS; ++g) gr.set16(g, a.zero[g_row + min(s * GS + g, KG - 1)]);
        }
    };
    auto place = [&]() {
#pragma unroll
        for (int q = 0; q < XV; ++q) {
            const int p = tid + NT * q;
            *reinterpret_cast<u32x4 *>(shared + p / 16 * XPITCH + p % 16 * 16) = reorder(xr[q]);
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int p = tid + NT * q;
            *reinterpret_cast<u32x4 *>(shared + Q_AT + p / 4 * QPITCH + p % 4 * 16) = qr[q];
        }
        // [group][BN] pairs of scale and zero
#pragma unroll
        for (int g = 0; g < GS; ++g) {
            float *to = reinterpret_cast<float *>(shared + S_AT) + (g * BN + tid % BN) * 2;
            if (tid < BN) to[0] = gr.half(g);
            else to[1] = ZEROS ? static_cast<float>((gr.w[g / 2] >> (g % 2 * 16)) & 0xffu) : 8.0f;
        }
    };
    f32x4 total[TN][TM];
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int r = 0; r < TM; ++r) total[t][r] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t exponent = exponent_of<XT>();
    auto multiply_stage = [&]() {
        const char *const xb = shared + (wm * (BM / WM) + fr) * XPITCH, *const qb = shared + Q_AT + (wn * TN * 16 + fr) * QPITCH + oct * 16;
        const float *const sb = reinterpret_cast<const float *>(shared + S_AT) + (wn * TN * 16 + fr) * 2;
        const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
        const u32x4 ones = {kOnes, kOnes, kOnes, kOnes};
        u32x4 code[TN];
#pragma unroll
        for (int t = 0; t < TN; ++t) {
            code[t] = *reinterpret_cast<const u32x4 *>(qb + t * 16 * QPITCH);
            regroup<G>(code[t]);
        }
#pragma unroll
        for (int gt = 0; gt < GS * (TN / 2); ++gt) {             // two column groups at a time
            const int g = gt / (TN / 2), t0 = gt % (TN / 2) * 2;
            f32x4 part[2][TM], xsum[TM];
            float sv[2], zv[2];
            f16x2 m1[2], m16[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const float2 v = *reinterpret_cast<const float2 *>(sb + (g * BN + (t0 + t) * 16) * 2);
                sv[t] = v.x;
                zv[t] = v.y;
                const _Float16 one = static_cast<_Float16>(-1024.0f - v.y), sixteen = static_cast<_Float16>(-64.0f - v.y);
                m1[t] = (f16x2){one, one};
                m16[t] = (f16x2){sixteen, sixteen};
            }
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                u32x4 xf[TM];
#pragma unroll
                for (int r = 0; r < TM; ++r) xf[r] = *reinterpret_cast<const u32x4 *>(xb + r * 16 * XPITCH + k_of<G>(g * PER + j, oct) * 2);
                if constexpr (XT == kXBf16) {
#pragma unroll
                    for (int r = 0; r < TM; ++r) xsum[r] = multiply<XT>(xf[r], ones, j == 0 ? none : xsum[r]);
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const u32x4 w = widen<XT>(code[t0 + t][g * PER + j], exponent, m1[t], m16[t]);
#pragma unroll
                    for (int r = 0; r < TM; ++r) part[t][r] = multiply<XT>(xf[r], w, j == 0 ? none : part[t][r]);
                }
                __builtin_amdgcn_sched_barrier(0);           // (32 k's numbers at a time)
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < TM; ++r)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float v = part[t][r][c];
                        if constexpr (XT == kXBf16) v = __builtin_fmaf(-16.0f - zv[t], xsum[r][c], v);
                        total[t0 + t][r][c] = __builtin_fmaf(sv[t], v, total[t0 + t][r][c]);
                    }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const int stages = (a.K + 127) / 128, turns = (stages + KS - 1) / KS;
    load(part_of);
    for (int i = 0; i < turns; ++i) {
        place();
        __syncthreads();
        load(min(i + 1, turns - 1) * KS + part_of);          // (the last one again, never used; past K: zeros)
        multiply_stage();
        __syncthreads();
    }
    if (!join<KS, NT>(total, all_shared, tile_lds(BM, BN, G), part_of, tid)) return;

    // total[t][r][c]: row wm * BM / WM + 16 r + 4 oct + c of the tile, column (wn * TN + t) * 16 + fr: sixteen columns of four
    // rows per instruction, 64 bytes each
    const int rows = row1 - row0;
#pragma unroll
    for (int r = 0; r < TM; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int row = wm * (BM / WM) + r * 16 + oct * 4 + c;
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                const int col = col0 + (wn * TN + t) * 16 + fr;
                if (row < rows && col < width)
                    static_cast<float *>(a.out)[static_cast<size_t>(row0 + row) * width + col] = total[t][r][c] * kBack<XT>;
            }
        }
}

// The rows of a block's first product, ready for the kernel below: fp16, in the codes' order, each row divided by a power of two
// such that its largest value is at most 2^15 (bf16's eight digits are then exact down to 2^-29 of it, and below that off by
// less than fp32 sums of such rows round).  A wavefront per row (a grid holds fewer than 2^32 threads: past 2^22 rows it takes
// several).
__global__ __launch_bounds__(256) void q4_rows_kernel(const uint16_t *__restrict__ x, const int32_t *__restrict__ offsets, int E,
                                                      _Float16 *__restrict__ out, float *__restrict__ row_scale, int K)
{
    const int lane = lane_id();
    const unsigned rows = max(offsets[E], 0);
    for (unsigned row = blockIdx.x * 4 + threadIdx.x / kWave; row < rows; row += gridDim.x * 4) {
        const uint16_t *src = x + static_cast<size_t>(row) * K;
        float most = 0.0f;
        for (int k = lane * 8; k < K; k += kWave * 8) {
            const u32x4 v = *reinterpret_cast<const u32x4 *>(src + k);
#pragma unroll
            for (int c = 0; c < 4; ++c)
                most = fmaxf(most, fmaxf(fabsf(__uint_as_float(v[c] << 16)), fabsf(__uint_as_float(v[c] & 0xffff0000u))));
        }
#pragma unroll
        for (int m = kWave / 2; m > 0; m >>= 1) most = fmaxf(most, __shfl_xor(most, m));
        // 2^15 / 2^ceil(log2 most), within fp32's range of normal numbers; a row of zeros or without a largest value as it is
        const int e = static_cast<int>(__float_as_uint(most) >> 23 & 0xff) - 127;
        const bool plain = most == 0.0f || e == 128;
        const int shift = plain ? 0 : min(max(14 - e, -126), 126);
        const float by = __uint_as_float(static_cast<uint32_t>(shift + 127) << 23);
        if (lane == 0) row_scale[row] = __uint_as_float(static_cast<uint32_t>(127 - shift) << 23);
        for (int k = lane * 8; k < K; k += kWave * 8) {
            const u32x4 v = reorder(*reinterpret_cast<const u32x4 *>(src + k));
            u32x4 o;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float lo = __uint_as_float(v[c] << 16) * by, hi = __uint_as_float(v[c] & 0xffff0000u) * by;
                const f16x2 h = {static_cast<_Float16>(lo), static_cast<_Float16>(hi)};
                o[c] = __builtin_bit_cast(uint32_t, h);
            }
            *reinterpret_cast<u32x4 *>(out + static_cast<size_t>(row) * K + k) = o;
        }
    }
}

// The tile kernel for rows that are ready, fp16 in the codes' order; tiles, wavefronts and parts as above.  They go from memory
// straight into LDS, one stage ahead, two places in turn; of a row's sixteen 16-byte pieces the one that quarter o of a
// wavefront reads with dword j lies at 4 j + o, XOR-swizzled with the row, both done by the choice of the loads' addresses:
// fragment reads are free of bank conflicts (with the pieces in their own order a third of the LDS's cycles, 1 % of the time).
// Codes, scales and zeros of the next stage are on their way in registers, requested behind x, so that the wait for them covers
// it. Bound by issue: beside 64 matrix instructions of a wavefront and stage stand 300 vector instructions (widening, scaling),
// and a matrix instruction hides three.  4096 rows, 8 experts, 2048 x 8192, group 128, tiles of 64 rows: 511 to 531 us a
// pass by the card, 810 to 780 TFLOP/s (356 + 197 with an event pair around each product).  In a kernel trace, where all take a
// tenth longer, the two products on those tiles 380 + 215, of 128 rows 383 + 232, the matrix cores busy for 39 %.  Tried
// against the latter: tiles of 128 x 256 on eight wavefronts, one block a compute unit, 432 + 279 us; the vector instructions
// placed by hand between the matrix instructions 375 + 225; weights scaled before the product (no sums per group, rounded to
// fp16) on four wavefronts and 128 x 256 tiles 471 + 286, 256 x 256 480 + 252: one wavefront per SIMD waits for its loads and
// numbers with nobody to step in.
template <int G, bool ZEROS, int BM, int BN, int KS>
__global__ __launch_bounds__(2 * BN * KS, KS == 4 && BN == 128 ? 4 : 2) void q4_ready_kernel(Q4Args a)
{
    constexpr int NT = 2 * BN, WAVES = NT / kWave, WM = BM / 64 > 1 ? 2 : 1, WN = WAVES / WM, TM = BM / WM / 16, TN = BN / 16 / WN;
    constexpr int GS = 128 / G, PER = 4 / GS;                // groups of a stage, dwords of 128 k and one group
    constexpr int X_BUF = BM * 256, Q_AT = 2 * X_BUF, S_AT = Q_AT + BN * 64;
    constexpr int XV = BM / 4 / WAVES;                           // loads of x per wavefront and stage, four rows each
    static_assert(KS == 1 || ready_lds(BM, BN, G) >= BM * BN * 4, "the sums lie there, too");
    extern __shared__ __attribute__((aligned(16))) char all_shared[];
    const int part_of = __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
    char *const shared = all_shared + part_of * ready_lds(BM, BN, G);
    const int tid = threadIdx.x % NT, lane = tid & 63, fr = lane & 15, oct = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % WM, wn = wave / WM;
    const bool gated = a.kind == kOutGated;
    const int width = gated ? a.N / 2 : a.N, KG = a.K / G, KB = a.K / 2;
    int expert, row0, row1, col0;
    if (!block_tile<BM>(a.offsets, a.E, a.tiles, blockIdx.x, expert, row0, row1, col0)) return;
    expert = __builtin_amdgcn_readfirstlane(expert);
    row0 = __builtin_amdgcn_readfirstlane(row0);
    row1 = __builtin_amdgcn_readfirstlane(row1);
    col0 = __builtin_amdgcn_readfirstlane(col0) * (gated ? BN / 2 : BN);

    // (rows past the expert's end: zeros that no load fetches)
    const __amdgpu_buffer_rsrc_t rsx = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t *>(a.x) + static_cast<size_t>(row0) * a.K, 0, static_cast<unsigned>(row1 - row0) * a.K * 2u, 0x00020000);
    int x_src[XV], x_col[4];                                 // (a lane's piece repeats every four loads)
#pragma unroll
    for (int q = 0; q < XV; ++q) {
        const int row = wave * (BM / WAVES) + q * 4 + (lane >> 4), at = (lane & 15) ^ (row & 15), piece = k_of<G>(at >> 2, at & 3) >> 3;
        x_src[q] = (row * a.K + piece * 8) * 2;
        if (q < 4) x_col[q] = piece * 8;
    }
    const uint32_t x_dest = lds_address(shared) + wave * (X_BUF / WAVES);
    auto load_x = [&](int s, int place) {
#pragma unroll
        for (int q = 0; q < XV; ++q)
            load_to_lds(rsx, s * 128 + x_col[q % 4] < a.K ? x_src[q] : 0x7ffffff0, x_dest + place * X_BUF + q * 1024, s * 256);
    };
    const uint8_t *q_src[2];
#pragma unroll
    for (int q = 0; q < 2; ++q)
        q_src[q] = a.q + (static_cast<size_t>(expert) * a.N + tile_code_row<TN>(gated, (tid + NT * q) / 4, col0, width)) * KB;
    const size_t g_row = (static_cast<size_t>(expert) * a.N + tile_code_row<TN>(gated, tid % BN, col0, width)) * KG;
    u32x4 qr[2];
    Run<GS * 2> gr;                                          // threads < BN: scales, others: zeros
    auto load_codes = [&](int s) {
#pragma unroll
        for (int q = 0; q < 2; ++q)
            qr[q] = *reinterpret_cast<const u32x4 *>(q_src[q] + min(s * 64 + (tid + NT * q) % 4 * 16, KB - 16));
        if (tid < BN) {
            if (s * GS + GS <= KG) {
                gr.load(a.scale + g_row + s * GS);
            } else {
#pragma unroll
                for (int g = 0; g < GS; ++g) gr.set16(g, s * GS + g < KG ? a.scale[g_row + min(s * GS + g, KG - 1)] : 0u);
            }
        } else if (ZEROS) {
#pragma unroll
            for (int g = 0; g < GS; ++g) gr.set16(g, a.zero[g_row + min(s * GS + g, KG - 1)]);
        }
    };
    auto place = [&]() {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int p = tid + NT * q, row = p / 4;
            *reinterpret_cast<u32x4 *>(shared + Q_AT + row * 64 + ((p % 4) ^ (row >> 2 & 3)) * 16) = qr[q];
        }
        // [group][BN] pairs of scale and -1024 - zero (twice, in fp16)
#pragma unroll
        for (int g = 0; g < GS; ++g) {
            uint32_t *to = reinterpret_cast<uint32_t *>(shared + S_AT) + (g * BN + tid % BN) * 2;
            if (tid < BN) {
                to[0] = __float_as_uint(gr.half(g));
            } else {
                const _Float16 m = static_cast<_Float16>(-1024.0f - (ZEROS ? static_cast<float>((gr.w[g / 2] >> (g % 2 * 16)) & 0xffu) : 8.0f));
                to[1] = __builtin_bit_cast(uint32_t, (f16x2){m, m});
            }
        }
    };
    f32x4 total[TN][TM];
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int r = 0; r < TM; ++r) total[t][r] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t exponent = exponent_of<kXF16>();
    int x_off[4];                                            // the lane's four fragments of a row
#pragma unroll
    for (int j = 0; j < 4; ++j) x_off[j] = (wm * (BM / WM) + fr) * 256 + ((4 * j + oct) ^ fr) * 16;
    const char *const qb = shared + Q_AT + (wn * TN * 16 + fr) * 64 + ((oct ^ (fr >> 2 & 3)) << 4);
    const u32x2 *const sb = reinterpret_cast<const u32x2 *>(shared + S_AT) + wn * TN * 16 + fr;
    auto multiply_stage = [&](int at) {
        const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
        const f16x2 up = {static_cast<_Float16>(960.0f), static_cast<_Float16>(960.0f)};
        u32x4 code[TN];
#pragma unroll
        for (int t = 0; t < TN; ++t) {
            code[t] = *reinterpret_cast<const u32x4 *>(qb + t * 16 * 64);
            regroup<G>(code[t]);
        }
#pragma unroll
        for (int g = 0; g < GS; ++g) {
            f32x4 part[TN][TM];
            u32x2 sz[TN];
#pragma unroll
            for (int t = 0; t < TN; ++t) sz[t] = sb[g * BN + t * 16];
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                u32x4 xf[TM];
#pragma unroll
                for (int r = 0; r < TM; ++r) xf[r] = *reinterpret_cast<const u32x4 *>(shared + at + x_off[g * PER + j] + r * 4096);
#pragma unroll
                for (int t = 0; t < TN; ++t) {
                    // (a scalar first: a bit cast of a vector's element is compiled as one of its first)
                    const uint32_t bits = sz[t][1];
                    const f16x2 m1 = __builtin_bit_cast(f16x2, bits);       // (m1 + 960, -64 - zero, is exact)
                    const u32x4 w = widen<kXF16>(code[t][g * PER + j], exponent, m1, m1 + up);
#pragma unroll
                    for (int r = 0; r < TM; ++r) part[t][r] = multiply<kXF16>(xf[r], w, j == 0 ? none : part[t][r]);
                }
                __builtin_amdgcn_sched_barrier(0);           // (32 k's numbers at a time)
            }
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int r = 0; r < TM; ++r)
#pragma unroll
                    for (int c = 0; c < 4; ++c) total[t][r][c] = __builtin_fmaf(__uint_as_float(sz[t][0]), part[t][r][c], total[t][r][c]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const int stages = (a.K + 127) / 128, turns = (stages + KS - 1) / KS;
    load_x(part_of, 0);
    load_codes(part_of);
    for (int i = 0; i < turns; ++i) {
        place();
        MOE_VMCNT(0);                                        // (x of this stage is older than what place() has waited for)
        __syncthreads();
        if (i + 1 < turns) {
            load_x((i + 1) * KS + part_of, (i + 1) & 1);     // (past K: zeros)
            load_codes((i + 1) * KS + part_of);
        }
        __builtin_amdgcn_sched_barrier(0);
        multiply_stage((i & 1) * X_BUF);
        __syncthreads();
    }
    const bool joined = join<KS, NT>(total, all_shared, ready_lds(BM, BN, G), part_of, tid);

    // total[t][r][c]: row wm * BM / WM + 16 r + 4 oct + c of the tile, its code row (wn * TN + t) * 16 + fr.  Out through
    // LDS, as whole lines.
    const int rows = row1 - row0;
    _Float16 *const tile = reinterpret_cast<_Float16 *>(all_shared);
    const int cols = gated ? BN / 2 : BN, pitch = cols + 8;
    float by[TM][4];
#pragma unroll
    for (int r = 0; r < TM; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c)
            by[r][c] = a.row_scale != nullptr ? a.row_scale[row0 + min(wm * (BM / WM) + r * 16 + oct * 4 + c, rows - 1)] : 1.0f;
#pragma unroll
    for (int t = 0; t < TN; ++t) {
        if (!joined || (gated && t >= TN / 2)) break;
        int col = gated ? wn * (8 * TN) + t * 16 + fr : (wn * TN + t) * 16 + fr;
        if (a.reorder_out) col = widened_place(col);
#pragma unroll
        for (int r = 0; r < TM; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float v = total[t][r][c] * by[r][c];
                if (gated) v = gated_by(a.act, v, total[(t + TN / 2) % TN][r][c] * by[r][c]);
                tile[(wm * (BM / WM) + r * 16 + oct * 4 + c) * pitch + col] = static_cast<_Float16>(v);
            }
    }
    __syncthreads();
    // (width is a multiple of 32)
    for (int p = threadIdx.x; p < BM * cols / 8; p += NT * KS) {
        const int row = p / (cols / 8), col = p % (cols / 8) * 8;
        if (row < rows && col0 + col < width)
            *reinterpret_cast<u32x4 *>(static_cast<_Float16 *>(a.out) + static_cast<size_t>(row0 + row) * width + col0 + col) =
                *reinterpret_cast<const u32x4 *>(tile + row * pitch + col);
    }
}

// ---------------------------------------------------------------- host side
// f(group, zeros or not) as constants
template <typename F>
void with_codes(const Q4Args &a, int group, F f)
{
    using std::integral_constant;
    auto with_group = [&](auto zeros) {
        if (group == 32) f(integral_constant<int, 32>{}, zeros);
        else if (group == 64) f(integral_constant<int, 64>{}, zeros);
        else f(integral_constant<int, 128>{}, zeros);
    };
    if (a.zero != nullptr) with_group(std::true_type{});
    else with_group(std::false_type{});
}

// f(rows of a tile, its columns, parts that its depth is shared out in) as constants.  Measured on either side of the lines, us:
//  * Tiles of 32 rows leave the fewest compute units idle; widening the codes once for every 32 rows costs most where
//    there are enough of larger tiles, too.  Block of 8 experts, 2048 x 8192, 32 / 64 rows a tile: 48 rows per expert 98 / 100,
//    96 153 / 133; of 4, 1024 x 2048, where tiles are few: 300 46 / 48, 512 64 / 66.  Linear map 4096 x 4096 of 640 rows 48 / 51,
//    of 1000 63 / 55; 2048 x 12000 of 160 35 / 43, of 320 52 / 45.
//  * 64 / 128 rows, 8 experts, 2048 x 8192: 512 per expert 525 / 540, 1024 1017 / 985, 2048 2139 / 1958; 4096 x 4096 654 / 684,
//    1247 / 1227, 2557 / 2297; linear map 2048 x 12000: 1000 rows 115 / 123, 2000 241 / 218.
//  * Few blocks of 32 rows, depth in 1 / 2 / 4 parts: 192 blocks 25 / 20 / 19, 352 36 / 32 / 36, 470 35 / 32 / 37, 640 48 / 49 / 57.
//  * Columns in 32s, the depth in 4 or 8 parts, while tiles of 128 columns would leave most compute units without one.  Blocks
//    of 32 x 32 in 8 / 4 parts / the tiles above: 64 .. 128 blocks 10 / 11 / 18, 256 10.4 / 11.5 / 18 and 20 / 21 / 37, 375 19 / 13 / 18, 504 51 /
//    41 / 53, 512 20 / 15.5 / 18 and 36 / 29 / 37, 640 27 / 19.5 / 18 and 34 / 23 / 23, 750 27 / 16.5 / 19, 768 52 / 38 / 37, 1024 37 / 26 / 20.
template <typename F>
void with_tile(int R, int E, int N, F f)
{
    using std::integral_constant;
    const integral_constant<int, 32> c32;
    const integral_constant<int, 64> c64;
    const integral_constant<int, 128> c128;
    const integral_constant<int, 1> whole;
    const int64_t blocks = (R / 32 + (std::min(R, E) + 1) / 2) * static_cast<int64_t>(ceil_div(N, 128));   // of 32 x 128
    const int64_t narrow = (R + 16ll * std::min(R, E) + 15) / 32 * ceil_div(N, 32);                        // of 32 x 32
    if (narrow <= 256) f(c32, c32, integral_constant<int, 8>{});
    else if (narrow <= 600) f(c32, c32, integral_constant<int, 4>{});
    else if (R / 1024 >= E) f(c128, c128, whole);
    else if (R / 64 >= E && blocks > 900) f(c64, c128, whole);
    else if (blocks > 512) f(c32, c128, whole);
    else if (blocks > 256) f(c32, c128, integral_constant<int, 2>{});
    else f(c32, c128, integral_constant<int, 4>{});
}
// Whether rows go through the kernel for few of them, which takes sixteen of an expert at a time.  That kernel / tiles, us: 16 and 20
// rows of 4096 x 4096 7 / 10 and 12 / 10, of 8192 x 8192 12 / 18 and 21 / 18, of 2048 x 12000 12 / 13 and 21 / 13; 4 experts, 2048 x 2048, 8
// and 12 rows each 6 / 8 and 10 / 8.  The gated block, 8 experts of 2048 x 8192, 10 and 14 rows each 52 / 54 and 79 / 54, of 1024 x 4096 26 /
// 28 and 39 / 28; one expert of 2048 x 5632, 14 and 20 rows 20 / 25 and 34 / 25.  At most 96 in all, since an expert's sixteens
// come one after the other, and of many experts' rows a popular one may have many: block, rows spread evenly (by 1 / rank; all
// of one expert), 64 experts of 2048 x 1536, 96 and 128 rows 67 / 89 (57 / 64; 113 / 42) and 73 / 94 (58 / 65; 150 / 42), of 512 x 1376, 128, 256 and
// 640 rows 33 / 34 (33 / 30; 100 / 18), 36 / 34 (56 / 30; 195 / 22) and 43 / 34 (106 / 44; 481 / 25); 32 of 2048 x 2048, 96 and 128 rows
// 47 / 48 (47 / 43) and 52 / 48 (50 / 48); 16 of 1024 x 4096, 96 and 112 rows 34 / 36 (37 / 36) and 36 / 35 (44 / 35); 8 of 4096 x 14336, group 64
// with zeros, 64 and 80 rows 197 / 311 (214 / 315) and 204 / 310 (219 / 315), group 128 172 / 193 (186 / 198) and 181 / 195 (190 / 202).
bool few_rows(int64_t R, int E) { return R <= 16 || (R <= 10 * E && R <= 96); }

// rows that are ready
void launch_q4_ready(Q4Args a, int R, int E, int group, int stage, hipStream_t st)
{
    a.E = E;
    with_codes(a, group, [&](auto g, auto zeros) {
        auto launch = [&](auto bmc, auto bnc, auto ksc) {
            constexpr int BM = decltype(bmc)::value, BN = decltype(bnc)::value, KS = decltype(ksc)::value, G = decltype(g)::value;
            auto kern = q4_ready_kernel<G, decltype(zeros)::value, BM, BN, KS>;
            constexpr int lds = KS * ready_lds(BM, BN, G);
            static PerDeviceOnce once;
            once.raise_lds(reinterpret_cast<const void *>(kern), lds);
            a.tiles = ceil_div(a.N, BN);                         // (of a gated product: of gates and values together)
            hipEvent_t t0, t1;
            prof_kernel_events(stage, &t0, &t1);
            hipExtLaunchKernelGGL(kern, dim3(block_tile_grid(R, E, BM, a.tiles)), dim3(2 * BN * KS), lds, st, t0, t1, 0, a);
        };
        with_tile(R, E, a.N, launch);
    });
}

template <int XT>
void launch_q4_tiles(Q4Args a, int R, int E, int group, hipStream_t st)
{
    a.E = E;
    with_codes(a, group, [&](auto g, auto zeros) {
        auto launch = [&](auto bmc, auto bnc, auto ksc) {
            constexpr int BM = decltype(bmc)::value, BN = decltype(bnc)::value, KS = decltype(ksc)::value, G = decltype(g)::value;
            auto kern = q4_tile_kernel<XT, G, decltype(zeros)::value, BM, BN, KS>;
            constexpr int lds = KS * tile_lds(BM, BN, G);
            static PerDeviceOnce once;
            once.raise_lds(reinterpret_cast<const void *>(kern), lds);
            a.tiles = ceil_div(a.N, BN);
            hipLaunchKernelGGL(kern, dim3(block_tile_grid(R, E, BM, a.tiles)), dim3(2 * BN * KS), lds, st, a);
        };
        with_tile(R, E, a.N, launch);
    });
}

void launch_q4_stream(Q4Args a, int R, int E, int group, int x, int stage, hipStream_t st)
{
    const bool gated = a.kind == kOutGated;
    const int width = gated ? a.N / 2 : a.N, used = std::min(R, E), steps = ceil_div(a.K, 256);
    // One or two column groups per block, and the depth shared out over as many wavefronts as occupy the compute units.  1 / 2 / 4 / 8
    // wavefronts everywhere against the rule, us: gated block of 2 rows, 8 experts, 4096 x 14336 62 / 47 / 36 / 42, 37; of 64 rows 219 / 197 /
    // 201 / 308, 193; 8 rows, 8 experts, 2048 x 8192 51 / 45 / 39 / 67, 38; 1 row, 2048 x 5632 27 / 19 / 14 / 15, 15; linear map of one row, 4096 x
    // 4096 12.4 / 7.7 / 6.1 / 6.2, 6.2; 4096 x 16384 13.5 / 10.9 / 8.0 / 8.4, 7.8; of 4 rows, 8192 x 1024 33 / 18 / 11 / 10.5, 10.6.
    int nt = R > 2 || gated || used * ceil_div(width, 32) >= 256 ? 2 : 1;
    a.tiles = ceil_div(width, gated ? nt * 8 : nt * 16);
    a.E = E;
    int waves = 1;
    while (waves < 8 && 2 * waves <= steps && (used * a.tiles * waves < 1536 || (used * a.tiles * waves < 4096 && steps >= 24 * waves))) waves *= 2;
    auto launch = [&](auto xt, auto g, auto zeros, auto ntc, auto xrc, auto tail) {
        constexpr int NT = decltype(ntc)::value, XR = decltype(xrc)::value, OWN = XR * 528 + NT * 16 * 144;
        auto kern = q4_stream_kernel<decltype(xt)::value, decltype(g)::value, decltype(zeros)::value, NT, XR, decltype(tail)::value>;
        static PerDeviceOnce once;
        once.raise_lds(reinterpret_cast<const void *>(kern), 8 * OWN);
        hipEvent_t t0 = nullptr, t1 = nullptr;
        if (stage >= 0) prof_kernel_events(stage, &t0, &t1);
        hipExtLaunchKernelGGL(kern, dim3(E * a.tiles), dim3(64 * waves), static_cast<size_t>(waves) * OWN, st, t0, t1, 0, a);
    };
    using std::integral_constant;
    auto with_tail = [&](auto xt, auto g, auto zeros, auto ntc, auto xrc) {
        if (a.K % 256 == 0) launch(xt, g, zeros, ntc, xrc, std::false_type{});
        else launch(xt, g, zeros, ntc, xrc, std::true_type{});
    };
    auto with_nt = [&](auto xt, auto g, auto zeros) {
        if (R > 2) with_tail(xt, g, zeros, integral_constant<int, 2>{}, integral_constant<int, 16>{});
        else if (nt == 2) with_tail(xt, g, zeros, integral_constant<int, 2>{}, integral_constant<int, 2>{});
        else with_tail(xt, g, zeros, integral_constant<int, 1>{}, integral_constant<int, 2>{});
    };
    with_codes(a, group, [&](auto g, auto zeros) {
        if (x == kXBf16) with_nt(integral_constant<int, kXBf16>{}, g, zeros);
        else with_nt(integral_constant<int, kXF16>{}, g, zeros);
    });
}

bool known_group(int group) { return group == 32 || group == 64 || group == 128; }

moe_status check_q4_block(const moe_shape *s)
{
    const moe_status rc = check_layer_shape(s);
    if (rc != MOE_OK) return rc;
    if (s->dtype != MOE_BF16) {
        set_error("moe_gated_ffn_q4: bf16 layers only");
        return MOE_EUNSUPPORTED;
    }
    if (s->d_ff >= 1 << 20 || s->d_model >= 1 << 20 || moe_max_rows(s) >= (1ll << 31) - 256) {
        set_error("moe_gated_ffn_q4: d_model and d_ff below 2^20, rows below 2^31 - 256");
        return MOE_EUNSUPPORTED;
    }
    return MOE_OK;
}

// Whether a block's rows are made ready and its products run on tiles.
bool many_rows(const moe_shape &s) { return !few_rows(moe_max_rows(&s), s.E); }

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" {

moe_status moe_q4_linear(const moe_q4_shape *s, const void *x, const int32_t *offsets, const void *q, const void *scale,
                         const void *zero, float *y, void *stream)
{
    if (s == nullptr) {
        set_error("moe_q4_linear: shape is NULL");
        return MOE_EINVAL;
    }
    if (s->R < 1 || s->E < 1 || s->N < 1 || s->K < 1 || (s->x != kXBf16 && s->x != kXF16)) {
        set_error("moe_q4_linear: R, E, N, K must be >= 1 and x 1 (bf16) or 2 (fp16)");
        return MOE_EINVAL;
    }
    if (s->E > kMaxExperts || s->N >= 1 << 24 || s->K >= 1 << 24 || s->R >= (1 << 30)) {
        set_error("moe_q4_linear: at most %d experts, N and K below 2^24, R below 2^30", kMaxExperts);
        return MOE_EUNSUPPORTED;
    }
    if (!known_group(s->group) || s->K % s->group != 0) {
        set_error("moe_q4_linear: group %d must be 32, 64 or 128 and divide K = %d", s->group, s->K);
        return MOE_EUNSUPPORTED;
    }
    MOE_REQUIRE_PTR(x);
    MOE_REQUIRE_PTR(offsets);
    MOE_REQUIRE_PTR(q);
    MOE_REQUIRE_PTR(scale);
    MOE_OPTIONAL_PTR(zero);
    MOE_REQUIRE_PTR(y);
    Q4Args a = {};
    a.x = static_cast<const uint16_t *>(x);
    a.offsets = offsets;
    a.q = static_cast<const uint8_t *>(q);
    a.scale = static_cast<const uint16_t *>(scale);
    a.zero = static_cast<const uint8_t *>(zero);
    a.out = y;
    a.N = s->N;
    a.K = s->K;
    a.kind = kOutF32;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (few_rows(s->R, s->E)) launch_q4_stream(a, s->R, s->E, s->group, s->x, -1, st);
    else if (s->x == kXBf16) launch_q4_tiles<kXBf16>(a, s->R, s->E, s->group, st);
    else launch_q4_tiles<kXF16>(a, s->R, s->E, s->group, st);
    MOE_TRY_HIP(hipGetLastError());
    return MOE_OK;
}

size_t moe_gated_q4_workspace_bytes(const moe_shape *s)
{
    if (check_q4_block(s) != MOE_OK) return 0;
    const size_t R = static_cast<size_t>(moe_max_rows(s));
    size_t bytes = align_up(R * s->d_ff * 2, 256);
    if (many_rows(*s)) bytes += align_up(R * s->d_model * 2, 256) + align_up(R * 4, 256);
    return bytes;
}

moe_status moe_gated_ffn_q4(const moe_shape *s, int32_t group, const void *xe, const int32_t *offsets, const void *q13,
                            const void *scale13, const void *zero13, const void *q2, const void *scale2, const void *zero2,
                            void *ye, void *workspace, void *stream)
{
    const moe_status rc = check_q4_block(s);
    if (rc != MOE_OK) return rc;
    if (!known_group(group) || s->d_model % group != 0 || s->d_ff % group != 0) {
        set_error("moe_gated_ffn_q4: group %d must be 32, 64 or 128 and divide d_model = %d and d_ff = %d", group, s->d_model, s->d_ff);
        return MOE_EUNSUPPORTED;
    }
    MOE_REQUIRE_PTR(xe);
    MOE_REQUIRE_PTR(offsets);
    MOE_REQUIRE_PTR(q13);
    MOE_REQUIRE_PTR(scale13);
    MOE_OPTIONAL_PTR(zero13);
    MOE_REQUIRE_PTR(q2);
    MOE_REQUIRE_PTR(scale2);
    MOE_OPTIONAL_PTR(zero2);
    MOE_REQUIRE_PTR(ye);
    MOE_REQUIRE_PTR(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int R = static_cast<int>(moe_max_rows(s));
    Q4Args a = {};
    a.x = static_cast<const uint16_t *>(xe);
    a.offsets = offsets;
    a.q = static_cast<const uint8_t *>(q13);
    a.scale = static_cast<const uint16_t *>(scale13);
    a.zero = static_cast<const uint8_t *>(zero13);
    a.out = workspace;
    a.N = 2 * s->d_ff;
    a.K = s->d_model;
    a.kind = kOutGated;
    a.act = s->act;
    const bool many = many_rows(*s);
    if (many) {
        char *at = static_cast<char *>(workspace) + align_up(static_cast<size_t>(R) * s->d_ff * 2, 256);
        float *row_scale = reinterpret_cast<float *>(at + align_up(static_cast<size_t>(R) * s->d_model * 2, 256));
        hipLaunchKernelGGL(q4_rows_kernel, dim3(std::min(parts_of(R, 4), 1 << 20)), dim3(256), 0, st, a.x, offsets, s->E, reinterpret_cast<_Float16 *>(at),
                           row_scale, s->d_model);
        a.x = reinterpret_cast<const uint16_t *>(at);
        a.row_scale = row_scale;
        a.reorder_out = true;
        launch_q4_ready(a, R, s->E, group, kStageGemm1, st);
    } else {
        launch_q4_stream(a, R, s->E, group, kXBf16, kStageGemm1, st);
    }
    a.row_scale = nullptr;
    a.reorder_out = false;
    a.x = static_cast<const uint16_t *>(workspace);
    a.q = static_cast<const uint8_t *>(q2);
    a.scale = static_cast<const uint16_t *>(scale2);
    a.zero = static_cast<const uint8_t *>(zero2);
    a.out = ye;
    a.N = s->d_model;
    a.K = s->d_ff;
    a.kind = kOutF16;
    if (many) launch_q4_ready(a, R, s->E, group, kStageGemm2, st);
    else launch_q4_stream(a, R, s->E, group, kXF16, kStageGemm2, st);
    MOE_TRY_HIP(hipGetLastError());
    return MOE_OK;
}

}  // extern "C"
