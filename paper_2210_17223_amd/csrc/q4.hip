// Products with weights held as 4-bit codes with group scales and zeros (include/moe_gated.h): one linear map, and the
// gated feed-forward block on them.
//
// The codes go from memory into registers and from there into the matrix instruction: eight codes of a lane become eight
// 16-bit numbers in place, by masks and an exponent: in bf16 128 + q, in fp16 1024 + q.  Products and sums over a group are
// then exact but for fp32's roundings, and a group's sum is scaled in fp32:
//   bf16   sum (q - z) x = sum (128 + q) x - (128 + z) sum x, with sum x from one more matrix instruction against ones
//          (shared by all of a wavefront's columns)
//   fp16   q - z by one packed subtraction (exact), no correction
#include "activation.h"
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

// Eight codes of a dword, c0 lowest, as eight 16-bit numbers in the order c0 c4 c1 c5 c2 c6 c3 c7.
template <int XT>
__device__ __forceinline__ u32x4 widen(uint32_t w, f16x2 minus, f16x2 minus16)
{
    if constexpr (XT == kXBf16) {
        auto part = [](uint32_t v) { return (v & 0x000f000fu) | 0x43004300u; };
        return (u32x4){part(w), part(w >> 4), part(w >> 8), part(w >> 12)};
    } else {
        // low four bits of a byte: 1024 + q; high: 1024 + 16 q, a sixteenth of which is 64 + q
        const f16x2 sixteenth = {static_cast<_Float16>(0.0625f), static_cast<_Float16>(0.0625f)};
        auto low = [&](uint32_t v) {
            return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, (v & 0x000f000fu) | 0x64006400u) + minus);
        };
        auto high = [&](uint32_t v) {
            return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (v & 0x00f000f0u) | 0x64006400u),
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
// depth in steps of 256 (a 128-byte line of every column's codes), two of them on their way, and add up through LDS in a fixed
// order; rows are taken 16 at a time, of which those past the expert's last one are zeros that no load fetches.  x comes
// straight from memory, too, half a step ahead, and feeds NT column groups: with one its reads, not the codes', would fill
// the address unit (1 KiB of x for 256 bytes of codes).
// KTAIL: K is not a multiple of 256.
template <int XT, int G, bool ZEROS, int NT, bool KTAIL>
__global__ __launch_bounds__(512) void q4_stream_kernel(Q4Args a)
{
    constexpr int PD = 2, GROUPS = 256 / G, PER = 4 / (128 / G);      // groups of a step; dwords of 128 k and one group
    const int expert = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles;
    const int r0 = a.offsets[expert], r1 = a.offsets[expert + 1];
    if (r0 >= r1) return;
    const int lane = lane_id(), fr = lane & 15, oct = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
    extern __shared__ __attribute__((aligned(16))) float sums[];      // [waves][NT][4][64]
    const bool gated = a.kind == kOutGated;
    const int half = gated ? NT / 2 : NT, width = gated ? a.N / 2 : a.N, col0 = tile * half * 16;
    const int KG = a.K / G, KB = a.K / 2;
    // group t's first row of codes, and the rows it has (past the last column: one, again)
    auto first_row = [&](int t) {
        return static_cast<size_t>(expert) * a.N + min(col0 + t % half * 16, width - 1) + (t >= half ? width : 0);
    };
    auto rows_of = [&](int t) { return min(max(width - col0 - t % half * 16, 1), 16); };
    const int q_at = fr * KB + oct * 16;
    unsigned g_at[NT];                                   // the lane's row of groups
#pragma unroll
    for (int t = 0; t < NT; ++t) g_at[t] = static_cast<unsigned>(min(fr, rows_of(t) - 1)) * KG;
    const int steps = a.K / 256;
    const int s0 = steps * wave / waves, s1 = steps * (wave + 1) / waves;

    for (int row0 = r0; row0 < r1; row0 += 16) {
        const __amdgpu_buffer_rsrc_t rsx = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint16_t *>(a.x) + static_cast<size_t>(row0) * a.K, 0, static_cast<unsigned>(min(r1 - row0, 16)) * a.K * 2u, 0x00020000);
        f32x4 total[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) total[t] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
        u32x4 code[PD][NT][2], xr[2][4];
        Run<GROUPS * 2> sc[PD][NT];
        Run<GROUPS> zr[PD][NT];
        auto load = [&](auto uc, int s) {
            constexpr int u = decltype(uc)::value;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
                    const_cast<uint8_t *>(a.q) + first_row(t) * KB + s * 128, 0, static_cast<unsigned>(max(rows_of(t) * KB - s * 128, 0)), 0x00020000);
#pragma unroll
                for (int b = 0; b < 2; ++b)
                    code[u][t][b] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, q_at + b * 64, 0, 0));
                const uint16_t *sp = a.scale + first_row(t) * KG;
                const uint8_t *zp = a.zero + first_row(t) * KG;
                sc[u][t].load(reinterpret_cast<const char *>(sp + s * GROUPS) + g_at[t] * 2u);
                if constexpr (ZEROS) zr[u][t].load(zp + s * GROUPS + g_at[t]);
            }
        };
        // (what lies past K reads as zeros: x alone decides there)
        auto load_x = [&](auto bc, auto tail, int s) {
            constexpr int b = decltype(bc)::value;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = s * 256 + b * 128 + k_of<G>(j, oct);
                int at = (fr * a.K + k) * 2;
                if constexpr (decltype(tail)::value) at = k < a.K ? at : 0x7ffffff0;
                xr[b][j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsx, at, 0, 0));
            }
        };
        auto use = [&](auto uc, auto bc) {
            constexpr int u = decltype(uc)::value, b = decltype(bc)::value;
            const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
            const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
            f32x4 xsum[GROUPS / 2];
#pragma unroll
            for (int j = 0; j < 4; ++j) xr[b][j] = reorder(xr[b][j]);
            if constexpr (XT == kXBf16) {
#pragma unroll
                for (int g = 0; g < GROUPS / 2; ++g) {
                    xsum[g] = none;
#pragma unroll
                    for (int j = 0; j < PER; ++j) xsum[g] = multiply<XT>(xr[b][g * PER + j], ones, xsum[g]);
                }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                regroup<G>(code[u][t][b]);
#pragma unroll
                for (int g = 0; g < GROUPS / 2; ++g) {
                    const float sv = sc[u][t].half(b * (GROUPS / 2) + g);
                    const float z = ZEROS ? static_cast<float>(zr[u][t].byte(b * (GROUPS / 2) + g)) : 8.0f;
                    const _Float16 m1 = static_cast<_Float16>(-1024.0f - z), m16 = static_cast<_Float16>(-64.0f - z);
                    f32x4 part = none;
#pragma unroll
                    for (int j = 0; j < PER; ++j)
                        part = multiply<XT>(xr[b][g * PER + j],
                                            widen<XT>(code[u][t][b][g * PER + j], (f16x2){m1, m1}, (f16x2){m16, m16}), part);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float v = part[c];
                        if constexpr (XT == kXBf16) v = __builtin_fmaf(-128.0f - z, xsum[g][c], v);
                        total[t][c] = __builtin_fmaf(sv, v, total[t][c]);
                    }
                }
                if (t % 2 == 1) __builtin_amdgcn_sched_barrier(0);   // (two column groups' numbers at a time)
            }
        };
        using B0 = std::integral_constant<int, 0>;
        using B1 = std::integral_constant<int, 1>;
        if (s0 < s1) {
            // (past the last step: the last one again, never used)
            unrolled<PD>([&](auto u) { load(u, min(s0 + decltype(u)::value, s1 - 1)); });
            using Whole = std::false_type;
            load_x(B0{}, Whole{}, s0);
            auto one = [&](auto u, int s) {
                load_x(B1{}, Whole{}, s);
                use(u, B0{});
                load_x(B0{}, Whole{}, min(s + 1, s1 - 1));
                use(u, B1{});
                load(u, min(s + PD, s1 - 1));
                __builtin_amdgcn_sched_barrier(0);
            };
            int s = s0;
            for (; s + PD <= s1; s += PD) unrolled<PD>([&](auto u) { one(u, s + decltype(u)::value); });
            if (s < s1) one(B0{}, s);
        }
        if constexpr (KTAIL) {
            // what is left of K, in the last wavefront: groups past it have no scale, codes and x past it read as zeros
            // or the next row's codes against zeros
            if (wave == waves - 1) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
                        const_cast<uint8_t *>(a.q) + first_row(t) * KB + steps * 128, 0, static_cast<unsigned>(rows_of(t) * KB - steps * 128), 0x00020000);
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        code[0][t][b] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, q_at + b * 64, 0, 0));
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) {
                        const bool there = steps * GROUPS + g < KG;
                        const unsigned at = g_at[t] + min(steps * GROUPS + g, KG - 1);
                        sc[0][t].set16(g, there ? (a.scale + first_row(t) * KG)[at] : 0u);
                        if constexpr (ZEROS) zr[0][t].set8(g, (a.zero + first_row(t) * KG)[at]);
                    }
                }
                load_x(B0{}, std::true_type{}, steps);
                load_x(B1{}, std::true_type{}, steps);
                use(B0{}, B0{});
                use(B0{}, B1{});
            }
        }

        // total[t][c]: row row0 + 4 oct + c, column fr of group t
        float *own = sums + wave * (NT * 256);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c) own[(t * 4 + c) * 64 + lane] = total[t][c];
        __syncthreads();
        const int rows = min(r1 - row0, 16), cols = half * 16;
        auto add_up = [&](int row, int t, int n) {
            const int at = (t * 4 + row % 4) * 64 + row / 4 * 16 + n;
            float v = 0.0f;
            for (int w = 0; w < waves; ++w) v += sums[w * (NT * 256) + at];
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

// ---------------------------------------------------------------- host side
void launch_q4(Q4Args a, int R, int E, int group, int x, int stage, hipStream_t st)
{
    const bool gated = a.kind == kOutGated;
    const int width = gated ? a.N / 2 : a.N, used = std::min(R, E), steps = ceil_div(a.K, 256);
    // Column groups per block: the more of them the fewer reads of x, as long as the blocks occupy the compute units.
    int nt = a.K % 256 == 0 ? 4 : 2;              // (with a part of a step left, four take more than 256 registers)
    while (nt > (gated ? 2 : 1) && used * ceil_div(width, gated ? nt * 8 : nt * 16) < 256) nt /= 2;
    a.tiles = ceil_div(width, gated ? nt * 8 : nt * 16);
    a.E = E;
    int waves = 1;
    while (waves < 8 && 2 * waves <= steps && used * a.tiles * waves < 4096) waves *= 2;
    auto launch = [&](auto xt, auto g, auto zeros, auto ntc, auto tail) {
        constexpr int NT = decltype(ntc)::value;
        auto kern = q4_stream_kernel<decltype(xt)::value, decltype(g)::value, decltype(zeros)::value, NT, decltype(tail)::value>;
        hipEvent_t t0 = nullptr, t1 = nullptr;
        if (stage >= 0) prof_kernel_events(stage, &t0, &t1);
        hipExtLaunchKernelGGL(kern, dim3(E * a.tiles), dim3(64 * waves), static_cast<size_t>(waves) * NT * 1024, st, t0, t1, 0, a);
    };
    using std::integral_constant;
    auto with_tail = [&](auto xt, auto g, auto zeros, auto ntc) {
        if (a.K % 256 == 0) launch(xt, g, zeros, ntc, std::false_type{});
        else launch(xt, g, zeros, ntc, std::true_type{});
    };
    auto with_nt = [&](auto xt, auto g, auto zeros) {
        if (nt == 4) launch(xt, g, zeros, integral_constant<int, 4>{}, std::false_type{});
        else if (nt == 2) with_tail(xt, g, zeros, integral_constant<int, 2>{});
        else with_tail(xt, g, zeros, integral_constant<int, 1>{});
    };
    auto with_zeros = [&](auto xt, auto g) {
        if (a.zero != nullptr) with_nt(xt, g, std::true_type{});
        else with_nt(xt, g, std::false_type{});
    };
    auto with_group = [&](auto xt) {
        if (group == 32) with_zeros(xt, integral_constant<int, 32>{});
        else if (group == 64) with_zeros(xt, integral_constant<int, 64>{});
        else with_zeros(xt, integral_constant<int, 128>{});
    };
    if (x == kXBf16) with_group(integral_constant<int, kXBf16>{});
    else with_group(integral_constant<int, kXF16>{});
}

bool bad_pointer(const void *p, const char *name, bool optional)
{
    if ((p == nullptr && !optional) || (reinterpret_cast<uintptr_t>(p) & 15u) != 0) {
        set_error(optional ? "%s is not 16-byte aligned" : "%s is NULL or not 16-byte aligned", name);
        return true;
    }
    return false;
}
#define MOE_Q4_PTR(p) \
    if (bad_pointer(p, #p, false)) return MOE_EINVAL
#define MOE_Q4_OPTIONAL(p) \
    if (bad_pointer(p, #p, true)) return MOE_EINVAL

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
    MOE_Q4_PTR(x);
    MOE_Q4_PTR(offsets);
    MOE_Q4_PTR(q);
    MOE_Q4_PTR(scale);
    MOE_Q4_OPTIONAL(zero);
    MOE_Q4_PTR(y);
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
    launch_q4(a, s->R, s->E, s->group, s->x, -1, static_cast<hipStream_t>(stream));
    MOE_TRY_HIP(hipGetLastError());
    return MOE_OK;
}

size_t moe_gated_q4_workspace_bytes(const moe_shape *s)
{
    if (check_q4_block(s) != MOE_OK) return 0;
    return align_up(static_cast<size_t>(moe_max_rows(s)) * s->d_ff * 2, 256);
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
    MOE_Q4_PTR(xe);
    MOE_Q4_PTR(offsets);
    MOE_Q4_PTR(q13);
    MOE_Q4_PTR(scale13);
    MOE_Q4_OPTIONAL(zero13);
    MOE_Q4_PTR(q2);
    MOE_Q4_PTR(scale2);
    MOE_Q4_OPTIONAL(zero2);
    MOE_Q4_PTR(ye);
    MOE_Q4_PTR(workspace);
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
    launch_q4(a, R, s->E, group, kXBf16, kStageGemm1, st);
    a.x = static_cast<const uint16_t *>(workspace);
    a.q = static_cast<const uint8_t *>(q2);
    a.scale = static_cast<const uint16_t *>(scale2);
    a.zero = static_cast<const uint8_t *>(zero2);
    a.out = ye;
    a.N = s->d_model;
    a.K = s->d_ff;
    a.kind = kOutF16;
    launch_q4(a, R, s->E, group, kXF16, kStageGemm2, st);
    MOE_TRY_HIP(hipGetLastError());
    return MOE_OK;
}

}  // extern "C"
