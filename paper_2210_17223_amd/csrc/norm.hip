// The step between two blocks: r = x + scale gate norm(z), next = norm(r), or next = norm(x) in front of the first one,
// forward and backward (include/moe_norm.h).
//
// A row is read once, stays in registers through both norms, and is written once, so that rows of up to 8192 forward and 4096
// backward are bound by HBM.  TPR threads
// (a wavefront, or a block) own a row, EPT of its columns each; a run of consecutive rows is one group of TPR threads' work,
// which keeps the vectors (weights, biases, gates) in registers; the forward pass has the next row's loads on their way
// while it reduces this one's.  Statistics are fp32: the mean first, then the sum of squares around it, from the registers.
// Backward: the vector gradients of a run are summed in registers and leave as one row of partial sums per run, which a
// second kernel adds up in a fixed order (no atomics: the same bits every time).
// Measured: forward, 32768 x 2048, fp32 x and z, bf16 next (0.94 GB) 188 us, 5.0 TB/s; 16384 x 4096, bf16 throughout, layer
// (0.54 GB) 106 us, 5.1 TB/s, its backward pass (0.81 GB, and 42 MB of partial sums both ways) 195 + 9 us, 4.3 TB/s.  A plain
// copy reaches 4.5 to 4.6 TB/s on these cards.
// Past these widths a block of 1024 threads, which has 128 registers a thread, does not hold a row and its vectors, and what
// it spills goes through the caches once a row: forward with z past 8192 34 to 97 registers, backward behind a block up to 8192 up to 60 and
// past it 185 to 385 (up to 4096 at most 18: with biases on eight bf16 columns a thread).  TB/s of the bytes that a row needs, forward /
// backward / the norm in front of the first block alone, 64 M values, bf16 layer with gates (fp32 x and z, RMS): d = 4096 4.6 / 4.2 / 6.1
// (5.0 / 4.8 / 5.0), 5120 4.5 / 2.2 / 5.4 (5.0 / 3.0 / 5.1), 8192 4.9 / 3.7 / 6.0 (5.1 / 4.3 / 5.1), 12288 2.8 / 0.6 / 5.6 (3.0 / 1.1 / 5.2),
// 16384 3.1 / 0.7 / 6.1 (3.3 / 1.2 / 5.3).  (At 5120 and 12288 three of eight and a quarter of the threads have no columns, too.)
#include "common.h"
#include "moe_norm.h"

#include <algorithm>
#include <type_traits>

namespace moe {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;

enum { kF32 = 0, kB16 = 1, kF16 = 2 };       // element types as in moe_norm_shape; -1: no z
constexpr int kMaxNormRow = 16384;

// VEC elements of a row as they lie in memory
template <int TY, int VEC>
struct Piece {
    static constexpr int W = TY == kF32 ? VEC : VEC / 2;
    uint32_t w[W];
    __device__ __forceinline__ void load(const void *row, int col)
    {
        const char *p = static_cast<const char *>(row) + static_cast<size_t>(col) * (TY == kF32 ? 4 : 2);
        if constexpr (W == 2) {
            const u32x2 v = *reinterpret_cast<const u32x2 *>(p);
            w[0] = v[0], w[1] = v[1];
        } else {
#pragma unroll
            for (int q = 0; q < W / 4; ++q) {
                const u32x4 v = *reinterpret_cast<const u32x4 *>(p + 16 * q);
#pragma unroll
                for (int c = 0; c < 4; ++c) w[4 * q + c] = v[c];
            }
        }
    }
    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (TY == kF32) {
            return __uint_as_float(w[i]);
        } else if constexpr (TY == kB16) {
            return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        } else {
            typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
            return static_cast<float>(__builtin_bit_cast(f16x2, w[i / 2])[i & 1]);
        }
    }
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    bf16x2 b;
    b[0] = static_cast<__bf16>(lo);
    b[1] = static_cast<__bf16>(hi);
    return __builtin_bit_cast(uint32_t, b);
}

// v to columns col .. col + VEC - 1 of a row, fp32 or rounded to bf16
template <int VEC>
__device__ __forceinline__ void store_row(void *row, bool f32, int col, const float (&v)[VEC])
{
    if (f32) {
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q)
            *reinterpret_cast<f32x4 *>(static_cast<float *>(row) + col + 4 * q) =
                (f32x4){v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    } else {
        uint32_t w[VEC / 2];
#pragma unroll
        for (int c = 0; c < VEC / 2; ++c) w[c] = pack_bf16(v[2 * c], v[2 * c + 1]);
        uint16_t *p = static_cast<uint16_t *>(row) + col;
        if constexpr (VEC == 8)
            *reinterpret_cast<u32x4 *>(p) = (u32x4){w[0], w[1], w[2], w[3]};
        else
            *reinterpret_cast<u32x2 *>(p) = (u32x2){w[0], w[1]};
    }
}

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v)
{
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// the sum over the wavefront, in every lane: rows of 16 lanes by data-parallel moves, the four rows through scalars
__device__ __forceinline__ float wave_sum(float v)
{
    v = dpp_add<0xb1>(v);          // lanes 1 0 3 2
    v = dpp_add<0x4e>(v);          // 2 3 0 1
    v = dpp_add<0x141>(v);         // halves of a row mirrored
    v = dpp_add<0x140>(v);         // rows mirrored
    auto lane = [&](int l) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)); };
    return (lane(0) + lane(16)) + (lane(32) + lane(48));
}

// Sums of N values over the TPR threads of a row.  Two places in turn: a wavefront that writes the one has seen all
// others read it behind the barrier of the other.
template <int TPR>
struct RowSum {
    static constexpr int WAVES = TPR / kWave;
    float (*part)[2][WAVES];       // [2] places of [2] values
    int turn = 0;
    template <int N>
    __device__ __forceinline__ void operator()(float (&v)[N])
    {
        static_assert(N <= 2, "two values at most");
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = wave_sum(v[n]);
        if constexpr (WAVES > 1) {
            if (lane_id() == 0) {
#pragma unroll
                for (int n = 0; n < N; ++n) part[turn][n][threadIdx.x / kWave] = v[n];
            }
            __syncthreads();
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) s += part[turn][n][w];
                v[n] = s;
            }
            turn ^= 1;
        }
    }
};

struct NormArgs {
    const void *x, *z, *r, *dr, *dnext;            // (backward: r is the residual that next came from)
    const float *w, *b, *gate, *w_next, *b_next;
    void *r_out, *next, *dx, *dz;
    float *dgate, *part;                           // part [runs][slots][d]
    int T, d, gate_tokens, per_run;
    bool layer, next_f32;
    float eps, scale;
};

constexpr int row_vec(int res, int z) { return res == kB16 && z != kF32 ? 8 : 4; }

// Forward.  Columns of thread t: (v TPR + t) VEC .. + VEC - 1.
template <int RES, int Z, int TPR, int EPT>
__global__ __launch_bounds__(TPR == kWave ? 256 : TPR) void norm_forward_kernel(NormArgs a)
{
    constexpr bool AFTER = Z >= 0;
    constexpr int ZT = AFTER ? Z : kF32, VEC = row_vec(RES, Z), NV = EPT / VEC;
    constexpr size_t RB = RES == kF32 ? 4 : 2, ZB = ZT == kF32 ? 4 : 2;
    __shared__ float part[2][2][TPR / kWave];
    RowSum<TPR> sum{part};
    const int d = a.d, t = TPR == kWave ? lane_id() : static_cast<int>(threadIdx.x);
    const int run = TPR == kWave ? static_cast<int>(blockIdx.x * 4 + threadIdx.x / kWave) : static_cast<int>(blockIdx.x);
    const int64_t first = static_cast<int64_t>(run) * a.per_run;
    const int i0 = static_cast<int>(min(first, static_cast<int64_t>(a.T))), i1 = min(a.T - i0, a.per_run) + i0;
    if (i0 >= i1) return;
    const float per = 1.0f / static_cast<float>(d);
    int col[NV];
    bool in[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        col[v] = (v * TPR + t) * VEC;
        in[v] = col[v] < d;
        col[v] = min(col[v], d - VEC);
    }
    Piece<RES, VEC> xr[NV];
    Piece<ZT, VEC> zr[NV];
    auto fetch = [&](int i) {
        const char *x = static_cast<const char *>(a.x) + static_cast<size_t>(i) * d * RB;
#pragma unroll
        for (int v = 0; v < NV; ++v) xr[v].load(x, col[v]);
        if constexpr (AFTER) {
            const char *z = static_cast<const char *>(a.z) + static_cast<size_t>(i) * d * ZB;
#pragma unroll
            for (int v = 0; v < NV; ++v) zr[v].load(z, col[v]);
        }
    };
    fetch(i0);
    // next = hat wn + bn;  r = x + zhat g + c
    float wn[NV][VEC], bn[NV][VEC], g[NV][VEC], c[NV][VEC];
    auto vector = [&](const float *p, float other, float (&out)[NV][VEC]) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            Piece<kF32, VEC> q;
            if (p != nullptr) q.load(p, col[v]);
#pragma unroll
            for (int e = 0; e < VEC; ++e) out[v][e] = p != nullptr ? q.at(e) : other;
        }
    };
    vector(a.w_next, 1.0f, wn);
    vector(a.b_next, 0.0f, bn);
    auto norm = [&](float (&v)[NV][VEC]) {         // v: the row, then (row - mean) factor
        if (a.layer) {
            float s[1] = {0.0f};
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < VEC; ++e) s[0] += v[q][e];
            sum(s);
            const float m = s[0] * per;
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[q][e] = in[q] ? v[q][e] - m : 0.0f;
        }
        float s[1] = {0.0f};
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < VEC; ++e) s[0] = __builtin_fmaf(v[q][e], v[q][e], s[0]);
        sum(s);
        const float f = rsqrtf(__builtin_fmaf(s[0], per, a.eps));
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[q][e] *= f;
    };
    int group_end = i0;
    for (int i = i0; i < i1; ++i) {
        float x[NV][VEC], z[NV][VEC];
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                x[v][e] = in[v] ? xr[v].at(e) : 0.0f;
                if constexpr (AFTER) z[v][e] = in[v] ? zr[v].at(e) : 0.0f;
            }
        if (i + 1 < i1) fetch(i + 1);
        if constexpr (AFTER) {
            if (i >= group_end) {                  // the row's gates
                const int group = a.gate_tokens != 0 ? i / a.gate_tokens : 0;
                group_end = a.gate_tokens != 0 ? min(a.T - group * a.gate_tokens, a.gate_tokens) + group * a.gate_tokens : a.T;
                vector(a.gate != nullptr ? a.gate + static_cast<size_t>(group) * d : nullptr, 1.0f, c);
                vector(a.w, 1.0f, g);
                float b[NV][VEC];
                vector(a.b, 0.0f, b);
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float s = a.scale * c[v][e];
                        g[v][e] *= s;
                        c[v][e] = b[v][e] * s;
                    }
            }
            norm(z);
            char *r = static_cast<char *>(a.r_out) + static_cast<size_t>(i) * d * RB;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    x[v][e] += __builtin_fmaf(z[v][e], g[v][e], c[v][e]);
                    // (what follows reads r as it is stored)
                    if constexpr (RES == kB16) x[v][e] = __uint_as_float(pack_bf16(0.0f, x[v][e]));
                    x[v][e] = in[v] ? x[v][e] : 0.0f;
                }
                if (in[v]) store_row<VEC>(r, RES == kF32, col[v], x[v]);
            }
        }
        norm(x);
        char *next = static_cast<char *>(a.next) + static_cast<size_t>(i) * d * (a.next_f32 ? 4 : 2);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[v][e] = __builtin_fmaf(x[v][e], wn[v][e], bn[v][e]);
            if (in[v]) store_row<VEC>(next, a.next_f32, col[v], x[v]);
        }
    }
}

// Rows of a run's partial sums: dw_next, db_next; behind a block also dw, db and what the run adds to the gradient
// of a gate whose rows begin in an earlier run, and of one whose rows begin here and go on in the next.
enum { kDwNext = 0, kDbNext, kDw, kDb, kGateFrom, kGateOn, kAfterSlots, kBeforeSlots = 2 };

// BIAS: the sums of dnext and D themselves are wanted (a norm has a bias, or its gradient was asked for).
template <int RES, int Z, int TPR, int EPT, bool BIAS>
__global__ __launch_bounds__(TPR == kWave ? 256 : TPR, TPR == kWave ? 3 : TPR <= 512 ? 4 : 1) void norm_backward_kernel(NormArgs a)
{
    constexpr bool AFTER = Z >= 0;
    constexpr int ZT = AFTER ? Z : kF32, VEC = row_vec(RES, Z), NV = EPT / VEC;
    constexpr size_t RB = RES == kF32 ? 4 : 2, ZB = ZT == kF32 ? 4 : 2;
    constexpr int slots = AFTER ? kAfterSlots : kBeforeSlots;
    __shared__ float part[2][2][TPR / kWave];
    RowSum<TPR> sum{part};
    const int d = a.d, t = TPR == kWave ? lane_id() : static_cast<int>(threadIdx.x);
    const int run = TPR == kWave ? static_cast<int>(blockIdx.x * 4 + threadIdx.x / kWave) : static_cast<int>(blockIdx.x);
    const int64_t first = static_cast<int64_t>(run) * a.per_run;
    const int i0 = static_cast<int>(min(first, static_cast<int64_t>(a.T))), i1 = min(a.T - i0, a.per_run) + i0;
    if (i0 >= i1) return;
    const float per = 1.0f / static_cast<float>(d);
    int col[NV];
    bool in[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        col[v] = (v * TPR + t) * VEC;
        in[v] = col[v] < d;
        col[v] = min(col[v], d - VEC);
    }
    Piece<RES, VEC> rr[NV], drr[NV];
    Piece<ZT, VEC> zr[NV];
    Piece<kF32, VEC> dnr[NV];                      // (of bf16: the first half)
    auto fetch = [&](int i) {
        const size_t at = static_cast<size_t>(i) * d;
        const char *r = static_cast<const char *>(a.r) + at * RB, *dr = static_cast<const char *>(a.dr) + at * RB;
#pragma unroll
        for (int v = 0; v < NV; ++v) rr[v].load(r, col[v]);
        if constexpr (AFTER) {
            const char *z = static_cast<const char *>(a.z) + at * ZB;
#pragma unroll
            for (int v = 0; v < NV; ++v) zr[v].load(z, col[v]);
        }
        const char *dn = static_cast<const char *>(a.dnext) + at * (a.next_f32 ? 4 : 2);
        if (a.next_f32) {
#pragma unroll
            for (int v = 0; v < NV; ++v) dnr[v].load(dn, col[v]);
        } else {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                Piece<kB16, VEC> p;
                p.load(dn, col[v]);
#pragma unroll
                for (int c = 0; c < VEC / 2; ++c) dnr[v].w[c] = p.w[c];
            }
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) drr[v].load(dr, col[v]);
    };
    auto vector = [&](const float *p, float other, float (&out)[NV][VEC]) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            Piece<kF32, VEC> q;
            if (p != nullptr) q.load(p, col[v]);
#pragma unroll
            for (int e = 0; e < VEC; ++e) out[v][e] = p != nullptr ? q.at(e) : other;
        }
    };
    float wn[NV][VEC], wa[NV][VEC];                // wa = scale gate w
    vector(a.w_next, 1.0f, wn);
    float dwn[NV][VEC], dbn[NV][VEC];              // sums of dnext rhat, dnext; of D zhat, D over the gate's rows so far
    float dz_sum[NV][VEC], d_sum[NV][VEC];
    auto clear = [&](float (&v)[NV][VEC]) {
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[q][e] = 0.0f;
    };
    clear(dwn);
    clear(dbn);
    clear(dz_sum);
    clear(d_sum);
    // the two rows' (value - mean) factor, in place, and the factors
    auto hats = [&](float (&u)[NV][VEC], float (&v)[NV][VEC], float (&f)[2]) {
        if (a.layer) {
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < VEC; ++e) s[0] += u[q][e], s[1] += AFTER ? v[q][e] : 0.0f;
            sum(s);
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    u[q][e] = in[q] ? u[q][e] - s[0] * per : 0.0f;
                    if constexpr (AFTER) v[q][e] = in[q] ? v[q][e] - s[1] * per : 0.0f;
                }
        }
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                s[0] = __builtin_fmaf(u[q][e], u[q][e], s[0]);
                if constexpr (AFTER) s[1] = __builtin_fmaf(v[q][e], v[q][e], s[1]);
            }
        sum(s);
        f[0] = rsqrtf(__builtin_fmaf(s[0], per, a.eps));
        f[1] = rsqrtf(__builtin_fmaf(s[1], per, a.eps));
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                u[q][e] *= f[0];
                if constexpr (AFTER) v[q][e] *= f[1];
            }
    };
    // g (of a norm's output without its weight's factor taken off) -> f (g - mean(g) - hat mean(g hat))
    auto through = [&](float (&g)[NV][VEC], const float (&hat)[NV][VEC], float f) {
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                s[0] = __builtin_fmaf(g[q][e], hat[q][e], s[0]);
                s[1] += g[q][e];
            }
        sum(s);
        const float m = s[0] * per, m1 = a.layer ? s[1] * per : 0.0f;
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < VEC; ++e) g[q][e] = f * (g[q][e] - m1 - hat[q][e] * m);
    };
    float *const own = a.part + static_cast<size_t>(run) * slots * d;
    auto leave = [&](float *row, const float (&v)[NV][VEC], bool add) {
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            if (!in[q]) continue;
            float s[VEC];
            Piece<kF32, VEC> before;
            if (add) before.load(row, col[q]);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s[e] = add ? v[q][e] + before.at(e) : v[q][e];
            store_row<VEC>(row, true, col[q], s);
        }
    };
    int group = 0, group_begin = 0, group_end = i0;
    bool left = false;                             // dw and db hold something already
    for (int i = i0; i < i1; ++i) {
        float r[NV][VEC], z[NV][VEC], D[NV][VEC], u[NV][VEC], f[2];
        fetch(i);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                r[v][e] = in[v] ? rr[v].at(e) : 0.0f;
                if constexpr (AFTER) z[v][e] = in[v] ? zr[v].at(e) : 0.0f;
                u[v][e] = in[v] ? (a.next_f32 ? dnr[v].at(e) : __uint_as_float(e & 1 ? dnr[v].w[e / 2] & 0xffff0000u : dnr[v].w[e / 2] << 16)) : 0.0f;
                D[v][e] = in[v] ? drr[v].at(e) : 0.0f;
            }
        if constexpr (AFTER) {
            if (i >= group_end) {
                group = a.gate_tokens != 0 ? i / a.gate_tokens : 0;
                group_begin = group * a.gate_tokens;
                group_end = a.gate_tokens != 0 ? min(a.T - group_begin, a.gate_tokens) + group_begin : a.T;
                float g[NV][VEC];
                vector(a.gate != nullptr ? a.gate + static_cast<size_t>(group) * d : nullptr, 1.0f, g);
                vector(a.w, 1.0f, wa);
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) wa[v][e] *= a.scale * g[v][e];
            }
        }
        hats(r, z, f);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                dwn[v][e] = __builtin_fmaf(u[v][e], r[v][e], dwn[v][e]);
                if constexpr (BIAS) dbn[v][e] += u[v][e];
                u[v][e] *= wn[v][e];
            }
        through(u, r, f[0]);
        char *dx = static_cast<char *>(a.dx) + static_cast<size_t>(i) * d * RB;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) D[v][e] = in[v] ? D[v][e] + u[v][e] : 0.0f;
            if (in[v]) store_row<VEC>(dx, RES == kF32, col[v], D[v]);
        }
        if constexpr (AFTER) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    dz_sum[v][e] = __builtin_fmaf(D[v][e], z[v][e], dz_sum[v][e]);
                    if constexpr (BIAS) d_sum[v][e] += D[v][e];
                    D[v][e] *= wa[v][e];
                }
            through(D, z, f[1]);
            char *dz = static_cast<char *>(a.dz) + static_cast<size_t>(i) * d * (ZT == kF32 ? 4 : 2);
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (in[v]) store_row<VEC>(dz, ZT == kF32, col[v], D[v]);
            if (i + 1 == group_end || i + 1 == i1) {
                // what the gate's rows of this run give: dw = scale gate S1, db = scale gate S0, dgate = scale (w S1 + b S0)
                float g[NV][VEC], w[NV][VEC], b[NV][VEC];
                vector(a.gate != nullptr ? a.gate + static_cast<size_t>(group) * d : nullptr, 1.0f, g);
                vector(a.w, 1.0f, w);
                vector(a.b, 0.0f, b);
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float s1 = a.scale * dz_sum[v][e], s0 = a.scale * d_sum[v][e];
                        w[v][e] = __builtin_fmaf(w[v][e], s1, b[v][e] * s0);
                        dz_sum[v][e] = g[v][e] * s1;
                        d_sum[v][e] = g[v][e] * s0;
                    }
                leave(own + kDw * d, dz_sum, left);
                if constexpr (BIAS) leave(own + kDb * d, d_sum, left);
                left = true;
                if (a.dgate != nullptr) {
                    if (group_begin < i0) leave(own + kGateFrom * d, w, false);
                    else if (group_end > i1) leave(own + kGateOn * d, w, false);
                    else leave(a.dgate + static_cast<size_t>(group) * d, w, false);
                }
                clear(dz_sum);
                clear(d_sum);
            }
        }
    }
    leave(own + kDwNext * d, dwn, false);
    if constexpr (BIAS) leave(own + kDbNext * d, dbn, false);
}

// Sums over the runs, 64 columns a block, 16 runs at a time: blockIdx.y < 4 the vectors, behind them the gates whose
// rows lie in more than one run, one row of blocks for each gate, or, if there are fewer of them, for each run (whose
// last gate it is).
struct NormReduceArgs {
    const float *part;
    float *out[4], *dgate;
    int T, d, gate_tokens, per_run, runs, slots, vectors;
    bool by_run;
};
__global__ __launch_bounds__(256) void norm_reduce_kernel(NormReduceArgs a)
{
    __shared__ f32x4 sums[16][16];
    int slot = blockIdx.y, run0 = 0, run1 = a.runs;
    float *out = nullptr;
    if (slot < a.vectors) {
        out = a.out[slot];
        if (out == nullptr) return;
    } else {
        const int which = slot - a.vectors, per = a.gate_tokens != 0 ? a.gate_tokens : a.T;
        int group = which;
        if (a.by_run) {
            const int end = min(a.T - which * a.per_run, a.per_run) + which * a.per_run;
            group = (end - 1) / per;
            if (group * per < which * a.per_run) return;       // (an earlier run's)
        }
        const int begin = group * per, end = min(a.T - begin, per) + begin;
        run0 = begin / a.per_run;
        run1 = (end - 1) / a.per_run + 1;
        if (run1 == run0 + 1) return;                          // (written where its rows are)
        slot = kGateFrom;
        out = a.dgate + static_cast<size_t>(group) * a.d;
    }
    const int lane = threadIdx.x % 16, part = threadIdx.x / 16, col = blockIdx.x * 64 + lane * 4;
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (col < a.d) {
#pragma unroll 4
        for (int r = run0 + part; r < run1; r += 16) {
            const int from = slot == kGateFrom && r == run0 ? kGateOn : slot;
            s += *reinterpret_cast<const f32x4 *>(a.part + (static_cast<size_t>(r) * a.slots + from) * a.d + col);
        }
    }
    sums[part][lane] = s;
    __syncthreads();
    if (part == 0 && col < a.d) {
#pragma unroll
        for (int p = 1; p < 16; ++p) s += sums[p][lane];
        *reinterpret_cast<f32x4 *>(out + col) = s;
    }
}

// ---------------------------------------------------------------- host side
int norm_gates(const moe_norm_shape &n) { return n.gate_tokens != 0 ? parts_of(n.T, n.gate_tokens) : 1; }

// Runs of the backward pass: as many as stay resident (their partial sums are 1 / per_run of a row's traffic).
int backward_runs(const moe_norm_shape &n, int *per_run)
{
    const int most = std::min(std::max(256, (1 << 21) / n.d), 2048);
    *per_run = parts_of(n.T, std::min(n.T, most));
    return parts_of(n.T, *per_run);
}

moe_status check_norm(const moe_norm_shape *n)
{
    if (n == nullptr) {
        set_error("norm shape is NULL");
        return MOE_EINVAL;
    }
    if (n->kind != MOE_NORM_RMS && n->kind != MOE_NORM_LAYER) {
        set_error("norm kind %d is neither MOE_NORM_RMS nor MOE_NORM_LAYER", n->kind);
        return MOE_EINVAL;
    }
    if (n->dtype < 0 || n->dtype > 1 || n->res < 0 || n->res > 1 || n->z < 0 || n->z > 2) {
        set_error("norm element types: dtype and res 0 or 1, z 0, 1 or 2 (got %d, %d, %d)", n->dtype, n->res, n->z);
        return MOE_EINVAL;
    }
    if (n->T < 1 || n->d < 1 || n->gate_tokens < 0 || !(n->eps >= 0.0f)) {
        set_error("norm shape: T, d >= 1, gate_tokens >= 0, eps >= 0");
        return MOE_EINVAL;
    }
    if (n->d % 8 != 0 || n->d > kMaxNormRow) {
        set_error("norm rows must be multiples of 8 up to %d (d = %d)", kMaxNormRow, n->d);
        return MOE_EUNSUPPORTED;
    }
    return MOE_OK;
}

// f(residual type, z's type or -1)
template <typename F>
void with_types(const moe_norm_shape &n, bool after, F f)
{
    auto with_z = [&](auto res) {
        if (!after) f(res, std::integral_constant<int, -1>{});
        else if (n.z == kF32) f(res, std::integral_constant<int, kF32>{});
        else if (n.z == kB16) f(res, std::integral_constant<int, kB16>{});
        else f(res, std::integral_constant<int, kF16>{});
    };
    if (n.res == kF32) with_z(std::integral_constant<int, kF32>{});
    else with_z(std::integral_constant<int, kB16>{});
}

NormArgs norm_args(const moe_norm_shape &n)
{
    NormArgs a = {};
    a.T = n.T;
    a.d = n.d;
    a.gate_tokens = n.gate_tokens;
    a.layer = n.kind == MOE_NORM_LAYER;
    a.next_f32 = n.dtype == kF32;
    a.eps = n.eps;
    a.scale = n.scale;
    return a;
}

moe_status launch_norm_forward(const moe_norm_shape &n, NormArgs a, bool after, hipStream_t st)
{
    with_types(n, after, [&](auto res, auto z) {
        auto launch = [&](auto tpr, auto ept, int most) {
            constexpr int TPR = decltype(tpr)::value;
            a.per_run = parts_of(n.T, std::min(n.T, most));
            const int runs = parts_of(n.T, a.per_run);
            hipLaunchKernelGGL((norm_forward_kernel<decltype(res)::value, decltype(z)::value, TPR, decltype(ept)::value>),
                               dim3(TPR == kWave ? ceil_div(runs, 4) : runs), dim3(TPR == kWave ? 256 : TPR), 0, st, a);
        };
        using std::integral_constant;
        if (n.d <= 512) launch(integral_constant<int, 64>{}, integral_constant<int, 8>{}, 256 * 16);
        else if (n.d <= 2048) launch(integral_constant<int, 256>{}, integral_constant<int, 8>{}, 256 * 6);
        else if (n.d <= 4096) launch(integral_constant<int, 256>{}, integral_constant<int, 16>{}, 256 * 4);
        else if (n.d <= 8192) launch(integral_constant<int, 512>{}, integral_constant<int, 16>{}, 256 * 2);
        else launch(integral_constant<int, 1024>{}, integral_constant<int, 16>{}, 256);
    });
    MOE_TRY_HIP(hipGetLastError());
    return MOE_OK;
}

moe_status launch_norm_backward(const moe_norm_shape &n, NormArgs a, bool after, float *const (&out)[4], hipStream_t st)
{
    const int runs = backward_runs(n, &a.per_run);
    with_types(n, after, [&](auto res, auto z) {
        auto launch = [&](auto tpr, auto ept) {
            constexpr int TPR = decltype(tpr)::value;
            auto run = [&](auto bias) {
                hipLaunchKernelGGL((norm_backward_kernel<decltype(res)::value, decltype(z)::value, TPR, decltype(ept)::value, decltype(bias)::value>),
                                   dim3(TPR == kWave ? ceil_div(runs, 4) : runs), dim3(TPR == kWave ? 256 : TPR), 0, st, a);
            };
            if (a.b != nullptr || out[kDbNext] != nullptr || out[kDb] != nullptr) run(std::true_type{});
            else run(std::false_type{});
        };
        using std::integral_constant;
        // As few columns per thread as a block of 1024 allows: without the next row's loads on their way in registers
        // and with 128 of these, other wavefronts' rows cover a row's latency, also where that spills some (16384 rows of 4096, bf16 throughout,
        // layer, with sixteen columns per thread and a row ahead 296 us, with eight 313, without the row ahead 195; fp32
        // throughout with eight columns 425, with four 358).
        if constexpr (row_vec(decltype(res)::value, decltype(z)::value) == 4) {
            if (n.d <= 256) return launch(integral_constant<int, 64>{}, integral_constant<int, 4>{});
            if (n.d <= 1024) return launch(integral_constant<int, 256>{}, integral_constant<int, 4>{});
            if (n.d <= 2048) return launch(integral_constant<int, 512>{}, integral_constant<int, 4>{});
            if (n.d <= 4096) return launch(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
        } else {
            if (n.d <= 512) return launch(integral_constant<int, 64>{}, integral_constant<int, 8>{});
            if (n.d <= 2048) return launch(integral_constant<int, 256>{}, integral_constant<int, 8>{});
            if (n.d <= 4096) return launch(integral_constant<int, 512>{}, integral_constant<int, 8>{});
        }
        if (n.d <= 8192) launch(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
        else launch(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
    });
    NormReduceArgs q = {};
    q.part = a.part;
    for (int i = 0; i < 4; ++i) q.out[i] = out[i];
    q.dgate = a.dgate;
    q.T = n.T;
    q.d = n.d;
    q.gate_tokens = n.gate_tokens;
    q.per_run = a.per_run;
    q.runs = runs;
    q.slots = after ? kAfterSlots : kBeforeSlots;
    q.vectors = after ? 4 : 2;
    const int gates = norm_gates(n);
    q.by_run = gates > runs;
    const int gate_rows = a.dgate != nullptr ? std::min(gates, runs) : 0;
    hipLaunchKernelGGL(norm_reduce_kernel, dim3(ceil_div(n.d, 64), q.vectors + gate_rows), dim3(256), 0, st, q);
    MOE_TRY_HIP(hipGetLastError());
    return MOE_OK;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" {

size_t moe_norm_workspace_bytes(const moe_norm_shape *n)
{
    if (check_norm(n) != MOE_OK) return 0;
    int per_run;
    return static_cast<size_t>(backward_runs(*n, &per_run)) * kAfterSlots * n->d * sizeof(float);
}

moe_status moe_norm_before(const moe_norm_shape *n, const void *x, const float *w_next,
                           const float *b_next, void *next, void *stream)
{
    const moe_status rc = check_norm(n);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE_PTR(x);
    MOE_REQUIRE_PTR(w_next);
    MOE_OPTIONAL_PTR(b_next);
    MOE_REQUIRE_PTR(next);
    NormArgs a = norm_args(*n);
    a.x = x;
    a.w_next = w_next;
    a.b_next = b_next;
    a.next = next;
    return launch_norm_forward(*n, a, false, static_cast<hipStream_t>(stream));
}

moe_status moe_norm_before_backward(const moe_norm_shape *n, const void *x, const float *w_next,
                                    const void *dnext, const void *dr, void *dx, float *dw_next,
                                    float *db_next, void *workspace, void *stream)
{
    const moe_status rc = check_norm(n);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE_PTR(x);
    MOE_REQUIRE_PTR(w_next);
    MOE_REQUIRE_PTR(dnext);
    MOE_REQUIRE_PTR(dr);
    MOE_REQUIRE_PTR(dx);
    MOE_REQUIRE_PTR(dw_next);
    MOE_OPTIONAL_PTR(db_next);
    MOE_REQUIRE_PTR(workspace);
    NormArgs a = norm_args(*n);
    a.r = x;
    a.w_next = w_next;
    a.dnext = dnext;
    a.dr = dr;
    a.dx = dx;
    a.part = static_cast<float *>(workspace);
    float *const out[4] = {dw_next, db_next, nullptr, nullptr};
    return launch_norm_backward(*n, a, false, out, static_cast<hipStream_t>(stream));
}

moe_status moe_norm_after(const moe_norm_shape *n, const void *x, const void *z, const float *w,
                          const float *b, const float *gate, void *r, const float *w_next,
                          const float *b_next, void *next, void *stream)
{
    const moe_status rc = check_norm(n);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE_PTR(x);
    MOE_REQUIRE_PTR(z);
    MOE_REQUIRE_PTR(w);
    MOE_OPTIONAL_PTR(b);
    MOE_OPTIONAL_PTR(gate);
    MOE_REQUIRE_PTR(r);
    MOE_REQUIRE_PTR(w_next);
    MOE_OPTIONAL_PTR(b_next);
    MOE_REQUIRE_PTR(next);
    NormArgs a = norm_args(*n);
    a.x = x;
    a.z = z;
    a.w = w;
    a.b = b;
    a.gate = gate;
    a.r_out = r;
    a.w_next = w_next;
    a.b_next = b_next;
    a.next = next;
    return launch_norm_forward(*n, a, true, static_cast<hipStream_t>(stream));
}

moe_status moe_norm_after_backward(const moe_norm_shape *n, const void *z, const void *r,
                                   const float *w, const float *b, const float *gate,
                                   const float *w_next, const void *dr, const void *dnext, void *dx,
                                   void *dz, float *dw, float *db, float *dgate, float *dw_next,
                                   float *db_next, void *workspace, void *stream)
{
    const moe_status rc = check_norm(n);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE_PTR(z);
    MOE_REQUIRE_PTR(r);
    MOE_REQUIRE_PTR(w);
    MOE_OPTIONAL_PTR(b);
    MOE_OPTIONAL_PTR(gate);
    MOE_REQUIRE_PTR(w_next);
    MOE_REQUIRE_PTR(dr);
    MOE_REQUIRE_PTR(dnext);
    MOE_REQUIRE_PTR(dx);
    MOE_REQUIRE_PTR(dz);
    MOE_REQUIRE_PTR(dw);
    MOE_OPTIONAL_PTR(db);
    MOE_OPTIONAL_PTR(dgate);
    MOE_REQUIRE_PTR(dw_next);
    MOE_OPTIONAL_PTR(db_next);
    MOE_REQUIRE_PTR(workspace);
    NormArgs a = norm_args(*n);
    a.z = z;
    a.r = r;
    a.w = w;
    a.b = b;
    a.gate = gate;
    a.w_next = w_next;
    a.dr = dr;
    a.dnext = dnext;
    a.dx = dx;
    a.dz = dz;
    a.dgate = dgate;
    a.part = static_cast<float *>(workspace);
    float *const out[4] = {dw_next, db_next, dw, db};
    return launch_norm_backward(*n, a, true, out, static_cast<hipStream_t>(stream));
}

}  // extern "C"
