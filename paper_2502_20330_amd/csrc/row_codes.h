// How a row of bf16 values becomes 8-bit integers with one scale (quant_rows.hip, lm_head_quant.hip).
//
//     code[c] = 127 x[c] / m to the nearest whole number, ties to even;   scale = m / 127;   m = max |x[c]|
//
// 127 x is exact in 32 bits (7 bits more than bf16's 8), and 127 x / m is a ratio of a 15-bit and an 8-bit number: it lies on the border between two
// codes, as x = m / 2 does, or at least 2^-9 of itself over 127 away from it, so that a quotient of 32 bits falls on the same side as the exact one if
// it is exact on the borders.  (A multiplication by 127 / m alone is not.)
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

namespace {

constexpr uint32_t kNotFinite = 0x7f80;

// The largest magnitude of eight values and what there is, as bf16 bits, two at a time: the order of magnitudes is that of their bits.
__device__ __forceinline__ uint32_t largest_two(const u32x4& v, uint32_t m)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu)));
    return m;
}
// The larger of the two, over the lanes of a wave.
__device__ __forceinline__ uint32_t wave_max(uint32_t two)
{
    int m = max((int)(two >> 16), (int)(two & 0xffffu));
    auto with = [&](int other) { m = max(m, other); };
    with(__builtin_amdgcn_update_dpp(0, m, 0x128, 0xf, 0xf, false));       // rotations by 8, 4, 2, 1 in rows of 16 lanes
    with(__builtin_amdgcn_update_dpp(0, m, 0x124, 0xf, 0xf, false));
    with(__builtin_amdgcn_update_dpp(0, m, 0x122, 0xf, 0xf, false));
    with(__builtin_amdgcn_update_dpp(0, m, 0x121, 0xf, 0xf, false));
    with(__builtin_amdgcn_update_dpp(0, m, 0x142, 0xa, 0xf, false));       // lane 15 of a row into the next: rows 1 and 3
    with(__builtin_amdgcn_update_dpp(0, m, 0x143, 0xc, 0xf, false));       // lane 31 into the upper half
    return (uint32_t)__builtin_amdgcn_readlane(m, 63);
}

// What a row is divided by, and the quotient: the product with the reciprocal, put right by its remainder.  The remainder is exact (a product of 24 and
// 8 bits less a number near it), so that a quotient that 32 bits hold, as those on a border do, comes out as it is, and any other within 2^-23 of
// itself, which is 2^-7 of its distance from a border.  (A division of 32 bits by its ten instructions: 128256 rows of 4096 293 us.)
// m and x are 2^64 or 2^-64 of themselves where 127 m would overflow, or 1 / m; what x loses by that has a code of 0 anyhow.
struct Divisor {
    float m, inv, factor;                                    // factor: 127, with what brings m into range
    bool some;
    __device__ __forceinline__ explicit Divisor(uint32_t bits)
    {
        some = bits != 0 && bits < kNotFinite;               // else nothing, or nothing finite: codes of 0
        m = __uint_as_float(some ? bits << 16 : 0x3f800000u);
        const float pre = m > 0x1p60f ? 0x1p-64f : m < 0x1p-60f ? 0x1p64f : 1.0f;
        m *= pre;
        factor = 127.0f * pre;
        inv = 1.0f / m;
    }
    __device__ __forceinline__ uint32_t code(uint32_t x_bits) const        // x as a number of 32 bits; the code is the last byte
    {
        const float t = __uint_as_float(x_bits) * factor, r = t * inv;
        const float q = fmaf(fmaf(-r, m, t), inv, r);
        return __float_as_uint(q + 0x1.8p23f);
    }
    __device__ __forceinline__ u32x2 codes(const u32x4& v) const
    {
        u32x2 r = {0, 0};
        if (some) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t a = __builtin_amdgcn_perm(code(v[2 * i] & 0xffff0000u), code(v[2 * i] << 16), 0x0c0c0400u);
                const uint32_t b = __builtin_amdgcn_perm(code(v[2 * i + 1] & 0xffff0000u), code(v[2 * i + 1] << 16), 0x04000c0cu);
                r[i] = a | b;
            }
        }
        return r;
    }
};
__device__ __forceinline__ float scale_of(uint32_t bits)
{
    return bits >= kNotFinite ? __uint_as_float(0x7fc00000u) : __uint_as_float(bits << 16) / 127.0f;
}

}  // namespace
