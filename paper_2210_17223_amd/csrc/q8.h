// Rows held in 8 bits (include/moe_q8.h): the codes of a row whose largest magnitude is known, for the kernels that write such rows.
#pragma once

#include "common.h"

namespace moe {

// A code is the rounded quotient itself, for a dozen instructions a value where no value of a wavefront's lies near a border: they hide behind
// the memory (32768 fp16 rows of 2048 to codes in 38 us, 5.3 TB/s).  Scale and what codes come from.  bits: of the largest magnitude, as a whole number (a NaN's lie above infinity's).
struct Q8Row {
    float most, inverse, up;               // most and values are taken `up` times, a power of two
    float scale;
    __device__ __forceinline__ explicit Q8Row(uint32_t bits)
    {
        const float m = __uint_as_float(bits);
        // (127 v and 127 / most have to be ordinary numbers)
        up = bits >= 0x5f800000u ? 0x1p-40f : bits < 0x20000000u ? 0x1p80f : 1.0f;
        most = m * up;
        inverse = 127.0f / most;
        scale = m / 127.0f;
        if (bits == 0u) up = most = inverse = 0.0f;
        if (bits >= 0x7f800000u) {
            up = most = inverse = 0.0f;
            scale = __uint_as_float(0x7fc00000u);
        }
    }
    // Codes of N values.  127 v / most is approximated by v (127 / most), less than 2^-15 off (half a last digit of 127 / most and of
    // the product, each below 2^-24 of up to 127).  Only where that is as near to the border of two codes, and of 16-bit values many
    // lie on one, 127 v is compared with the border c most in exact terms: with p the rounded c most, c most - p and, so near,
    // 127 v - p are numbers of 24 digits, which fused multiply-adds give.
    template <int N>
    __device__ __forceinline__ void codes(const float (&v)[N], int (&code)[N]) const
    {
        float t[N], k[N], far = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            // (of zeros, and of a row that is not finite, 0 whatever v is)
            t[i] = up == 0.0f ? 0.0f : v[i] * up * inverse;
            k[i] = __builtin_rintf(t[i]);
            far = fmaxf(far, __builtin_fabsf(t[i] - k[i]));
        }
        if (far > 0.5f - 0x1p-14f) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float side = t[i] < k[i] ? -1.0f : 1.0f, c = __builtin_fmaf(0.5f, side, k[i]), p = c * most;
                const float d = side * (__builtin_fmaf(127.0f, v[i] * up, -p) - __builtin_fmaf(c, most, -p));
                if (d > 0.0f || (d == 0.0f && (static_cast<int>(k[i]) & 1))) k[i] += side;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) code[i] = static_cast<int>(k[i]);
    }
};

// four codes in a dword
__device__ __forceinline__ uint32_t pack_codes(const int *c)
{
    return (static_cast<uint32_t>(c[0]) & 0xffu) | (static_cast<uint32_t>(c[1]) & 0xffu) << 8 |
           (static_cast<uint32_t>(c[2]) & 0xffu) << 16 | static_cast<uint32_t>(c[3]) << 24;
}

// magnitude of v as a whole number that orders as the magnitudes do
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_most(uint32_t v)
{
    return max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xf, 0xf, true)));
}
// the largest over the wavefront, in every lane
__device__ __forceinline__ uint32_t wave_most(uint32_t v)
{
    v = dpp_most<0xb1>(v);          // lanes 1 0 3 2
    v = dpp_most<0x4e>(v);          // 2 3 0 1
    v = dpp_most<0x141>(v);         // halves of a row mirrored
    v = dpp_most<0x140>(v);         // rows mirrored
    auto lane = [&](int l) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), l)); };
    return max(max(lane(0), lane(16)), max(lane(32), lane(48)));
}

}  // namespace moe
