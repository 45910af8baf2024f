// What the kernels of 8-bit products share.  Included inside the translation unit's own namespace.
#pragma once

typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
typedef __attribute__((ext_vector_type(4))) int i32x4;

#include "gemm_w4.h"

enum { kF32 = 0, kB16 = 1, kF16 = 2 };       // element types as in moe_q8_shape

// one of the two fp16 (bf16) values of a dword.  (By value: a bit cast of a vector's element casts its first one.)
__device__ __forceinline__ float f16_of(uint32_t w, int i) { return static_cast<float>(__builtin_bit_cast(f16x2, w)[i]); }
__device__ __forceinline__ float b16_of(uint32_t w, int i) { return __uint_as_float(i ? w & 0xffff0000u : w << 16); }

// v as it is in fp32, rounded to fp16: the compiler may not fold the product or sum before it into one instruction that rounds once, in
// some kernels and not in others.
__device__ __forceinline__ _Float16 to_f16(float v)
{
    asm("" : "+v"(v));
    return static_cast<_Float16>(v);
}
__device__ __forceinline__ uint32_t pack_16(int type, float lo, float hi)
{
    if (type == kF16) {
        f16x2 h;
        h[0] = to_f16(lo);
        h[1] = to_f16(hi);
        return __builtin_bit_cast(uint32_t, h);
    }
    bf16x2 b;
    b[0] = static_cast<__bf16>(lo);
    b[1] = static_cast<__bf16>(hi);
    return __builtin_bit_cast(uint32_t, b);
}

// The tile of block entry b: a panel of kPanel tiles' rows of an expert column by column, then the next; an eighth of all tiles for
// each XCD.  A wavefront holds the experts' row tiles and their running sum, a lane each.
constexpr int kPanel = 8;
template <int BM, int BN>
struct Tiles {
    int first, end, row_tiles, sum, per_xcd, total, tiles;
    __device__ __forceinline__ Tiles(const int32_t *__restrict__ offsets, int E, int column_tiles) : tiles(column_tiles)
    {
        const int lane = lane_id(), e = min(lane, E - 1);
        first = offsets[e];
        end = lane < E ? offsets[e + 1] : first;
        row_tiles = end > first ? (end - first + BM - 1) / BM : 0;
        sum = row_tiles * tiles;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int v = __shfl_up(sum, d);
            if (lane >= d) sum += v;
        }
        total = __builtin_amdgcn_readlane(sum, kWave - 1);
        per_xcd = (total + 7) / 8;
    }
    __device__ __forceinline__ WorkItem operator[](int b) const
    {
        const int slot = b / 8, index = b % 8 * per_xcd + slot;
        if (slot >= per_xcd || index >= total) return WorkItem{-1, 0, 0, 0};
        const int e = __builtin_amdgcn_readfirstlane(__popcll(__ballot(sum <= index)));
        const int mt = __builtin_amdgcn_readlane(row_tiles, e);
        const int within = index - (__builtin_amdgcn_readlane(sum, e) - mt * tiles);
        const int panel = within / (kPanel * tiles), rest = within - panel * (kPanel * tiles), high = min(kPanel, mt - panel * kPanel);
        const int column = rest / high, row0 = __builtin_amdgcn_readlane(first, e) + (panel * kPanel + rest - column * high) * BM;
        return WorkItem{e, row0, min(row0 + BM, __builtin_amdgcn_readlane(end, e)), column * BN};
    }
};
inline int64_t tile_entries(int64_t rows, int E, int bm, int tiles)
{
    return static_cast<int64_t>(align_up((static_cast<size_t>(rows) / bm + std::min<int64_t>(rows, E)) * tiles, 8));
}

// All activations but the erf form of the GeLU as factor * max(v, lowest) / (1 + 2^-(v (a + b v^2))): silu; its tanh form; and relu and
// identity, 2 max(v, lowest) / 2, of which nothing is rounded.  An epilogue that holds accumulators takes no branch, and a
// kernel for each activation is five times the code.  (v^2 is bounded so that 0 v^2 is 0.)
struct ActForm {
    float a, b, factor, lowest;
    __device__ __forceinline__ explicit ActForm(int act)
    {
        a = act == MOE_ACT_SILU ? 1.44269504088896341f : act == MOE_ACT_GELU_TANH ? 2.3022082f : 0.0f;
        b = act == MOE_ACT_GELU_TANH ? 0.10294324f : 0.0f;
        factor = act == MOE_ACT_IDENTITY || act == MOE_ACT_RELU ? 2.0f : 1.0f;
        // (of -infinity silu's and the tanh form's limit is 0)
        lowest = act == MOE_ACT_IDENTITY ? -__builtin_inff() : act == MOE_ACT_RELU ? 0.0f : -3.4e38f;
    }
    __device__ __forceinline__ float operator()(float v) const
    {
#pragma clang fp contract(off)
        // (the last product is rounded before a residual is added to it, in every kernel)
        const float in = __builtin_elementwise_minimum(__builtin_elementwise_maximum(v, -1e30f), 1e30f);
        const float slope = __builtin_fmaf(b, __builtin_elementwise_minimum(in * in, 1e30f), a);
        return __builtin_elementwise_maximum(v, lowest) * (factor * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-(in * slope))));
    }
};
// The erf form of the GeLU, max(v, 0) - a Phi(-a) with a = |v|, as good as what follows rounds: fp32 outputs by gelu_erf_32, 16-bit ones and the
// block's hidden rows by gelu_erf_16, of one transcendental and seven instructions fewer (8192 rows, 1024 to 4096 columns, bias, bf16: 58.5 us,
// by the former 64; first products of 8192 rows, 768 to 2 x 2048, and back 95 and 100; fp32 y 63.5, by the latter 59).
//
// Phi(-a) = exp(-a^2 / 2) R(t), t = 1 / (1 + 0.345 a), R a polynomial without constant (minimax of its relative error, 2^-25.5 on
// [0, 14]).  Within (14 + 1.5 v^2) 2^-24 of the result's size: three half steps of t, taken to a power of 2.3, seven roundings of R, the
// exponential and the products, and three of an exponent of 0.72 a^2; 0 where exp(-a^2 / 2) is below 2^-126.
__device__ __forceinline__ float gelu_erf_32(float v)
{
#pragma clang fp contract(off)
    const float a = __builtin_elementwise_minimum(__builtin_fabsf(v), 20.0f);      // (infinity stays off the product; NaN stays NaN)
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.345f, a, 1.0f));
    float r = -2.838195488e-02f;
    r = __builtin_fmaf(r, t, 1.452819407e-01f);
    r = __builtin_fmaf(r, t, -2.711730301e-01f);
    r = __builtin_fmaf(r, t, 1.871966124e-01f);
    r = __builtin_fmaf(r, t, -3.760161251e-02f);
    r = __builtin_fmaf(r, t, 1.117995679e-01f);
    r = __builtin_fmaf(r, t, 1.172382906e-01f);
    r = __builtin_fmaf(r, t, 1.380208880e-01f);
    r = __builtin_fmaf(r, t, 1.376192868e-01f);
    return __builtin_fmaf(-a, r * t * __builtin_amdgcn_exp2f(a * a * -0.72134752f), __builtin_elementwise_maximum(v, 0.0f));
}
// Phi(-a) = 2^P(a), P a polynomial of degree 7 with P(0) = -1, minimax of the error over the smaller of 2^-14 of a Phi(-a) and 2e-7 on [0, 8], and
// falling on from there: 2^-17.8 of the result's size for |v| <= 2, 2^-13.5 down to -8 (a third of fp16's half step at most), and below
// that, where the result is under 5e-15, within 1e-16.
__device__ __forceinline__ float gelu_erf_16(float v)
{
    const float a = __builtin_elementwise_minimum(__builtin_fabsf(v), 14.0f);
    float p = -1.512625886e-06f;
    p = __builtin_fmaf(p, a, 5.506610978e-05f);
    p = __builtin_fmaf(p, a, -8.806571714e-04f);
    p = __builtin_fmaf(p, a, 8.329684846e-03f);
    p = __builtin_fmaf(p, a, -5.365595222e-02f);
    p = __builtin_fmaf(p, a, -4.586960375e-01f);
    p = __builtin_fmaf(p, a, -1.151185513e+00f);
    p = __builtin_fmaf(p, a, -1.0f);
    return __builtin_fmaf(-a, __builtin_amdgcn_exp2f(p), __builtin_elementwise_maximum(v, 0.0f));
}
// The activation in every kernel (kForm: by its form), so that all give the same bits.
enum { kForm = 9 };
template <int ACT>
__device__ __forceinline__ float activate(const ActForm &form, float v)
{
#pragma clang fp contract(off)
    if constexpr (ACT == kForm) return form(v);
    // (the form's steps without those that change nothing)
    else if constexpr (ACT == MOE_ACT_SILU)
        return __builtin_elementwise_maximum(v, -3.4e38f) * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * v));
    else if constexpr (ACT == kGeluErf32) return gelu_erf_32(v);
    else if constexpr (ACT == MOE_ACT_GELU_ERF) return gelu_erf_16(v);
    else {
        static_assert(ACT == MOE_ACT_IDENTITY, "the others go by their form");
        return v;
    }
}
// f(integral_constant of one of `kinds`, or of kForm)
template <int... KINDS, typename F>
__host__ __device__ __forceinline__ void with_activation(int act, F f)
{
    if (((act == KINDS ? (f(std::integral_constant<int, KINDS>{}), true) : false) || ...)) return;
    f(std::integral_constant<int, kForm>{});
}
__device__ __forceinline__ float sum_of(float bits) { return static_cast<float>(__builtin_bit_cast(int, bits)); }

// The way of a wavefront's sums to y: rows row0 .. row1 - 1, of each a lane's columns n .. n + PER - 1 (four where N is a multiple of four,
// else one).  No branch on types: each of r's and y's two sizes has a buffer resource of its own, the one that is not theirs is empty,
// and what is asked of it or left to it takes no way to memory; so do a row past the last and a column past N.
template <int PER>
struct WayOut {
    static_assert(PER == 1 || PER == 4, "one column, or four");
    struct Residual {
        uint32_t wide[PER], half[(PER + 1) / 2];
    };
    __amdgpu_buffer_rsrc_t y32, y16, r32, r16;
    int pitch, column;
    uint32_t none;                         // without a residual -0 is added, which leaves every value as it is, -0 too
    bool r_wide, r_f16, y_f16;
    __device__ __forceinline__ WayOut(const Q8Args &a, int row0, int row1, int n) : pitch(a.N), column(n < a.N ? n : 0x1ff00000)
    {
        const size_t first = static_cast<size_t>(row0) * a.N;
        const unsigned values = static_cast<unsigned>(max(row1 - row0, 0)) * static_cast<unsigned>(a.N);
        auto resource = [&](const void *p, unsigned size, bool used) {
            return __builtin_amdgcn_make_buffer_rsrc(static_cast<char *>(const_cast<void *>(p)) + first * size, 0, used ? values * size : 0u, 0x00020000);
        };
        none = a.r != nullptr ? 0u : 0x80000000u;
        r_wide = a.r == nullptr || a.res == kF32;
        r_f16 = a.res == kF16;
        y_f16 = a.type == kF16;
        y32 = resource(a.y, 4, a.type == kF32);
        y16 = resource(a.y, 2, a.type != kF32);
        r32 = resource(a.r, 4, a.r != nullptr && r_wide);
        r16 = resource(a.r, 2, a.r != nullptr && !r_wide);
    }
    __device__ __forceinline__ int at(int row) const { return column == 0x1ff00000 ? column : row * pitch + column; }
    __device__ __forceinline__ void ask(int row, Residual &r) const
    {
        if constexpr (PER == 4) {
            const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(r32, at(row) * 4, 0, 0);
            const u32x2 h = __builtin_amdgcn_raw_buffer_load_b64(r16, at(row) * 2, 0, 0);
#pragma unroll
            for (int c = 0; c < 4; ++c) r.wide[c] = w[c];
            r.half[0] = h[0], r.half[1] = h[1];
        } else {
            r.wide[0] = __builtin_amdgcn_raw_buffer_load_b32(r32, at(row) * 4, 0, 0);
            r.half[0] = __builtin_amdgcn_raw_buffer_load_b16(r16, at(row) * 2, 0, 0);
        }
    }
    __device__ __forceinline__ float value(const Residual &r, int c) const
    {
        const float half = r_f16 ? f16_of(r.half[c / 2], c % 2) : b16_of(r.half[c / 2], c % 2);
        return r_wide ? __uint_as_float(r.wide[c] | none) : half;
    }
    __device__ __forceinline__ void leave(int row, const float (&v)[PER]) const
    {
        if constexpr (PER == 4) {
            const u32x4 w = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
            const u32x2 h = {pack_16(kF16, v[0], v[1]), pack_16(kF16, v[2], v[3])}, b = {pack_16(kB16, v[0], v[1]), pack_16(kB16, v[2], v[3])};
            __builtin_amdgcn_raw_buffer_store_b128(w, y32, at(row) * 4, 0, 0);
            __builtin_amdgcn_raw_buffer_store_b64(y_f16 ? h : b, y16, at(row) * 2, 0, 0);
        } else {
            const uint16_t h = static_cast<uint16_t>(y_f16 ? pack_16(kF16, v[0], 0.0f) : pack_16(kB16, v[0], 0.0f));
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[0]), y32, at(row) * 4, 0, 0);
            __builtin_amdgcn_raw_buffer_store_b16(h, y16, at(row) * 2, 0, 0);
        }
    }
};
__device__ __forceinline__ void store_hidden(const Q8Args &a, size_t row, int n, const float (&v)[4])
{
    f16x4 o;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] = to_f16(v[c]);
    *reinterpret_cast<f16x4 *>(static_cast<_Float16 *>(a.y) + row * a.h + n) = o;
}
__device__ __forceinline__ float row_scale(const Q8Args &a, int row)
{
    return a.xs[a.row_src != nullptr ? a.row_src[row] / a.row_div : row];
}
// scales of columns n .. n + 3, of the last column past it
__device__ __forceinline__ void column_scales(const float *__restrict__ p, int n, int N, float (&s)[4])
{
#pragma unroll
    for (int c = 0; c < 4; ++c) s[c] = p[min(n + c, N - 1)];
}

// a kernel of 256 threads that needs more LDS than a launch gets unasked
template <auto KERNEL>
void launch_product_kernel(const Q8Args &a, int64_t blocks, size_t lds, int stage, hipStream_t st)
{
    static PerDeviceOnce once;
    once.raise_lds(reinterpret_cast<const void *>(KERNEL), static_cast<int>(lds));
    hipEvent_t t0 = nullptr, t1 = nullptr;
    if (stage >= 0) prof_kernel_events(stage, &t0, &t1);
    hipExtLaunchKernelGGL(KERNEL, dim3(static_cast<unsigned>(blocks)), dim3(256), lds, st, t0, t1, 0, a);
}
