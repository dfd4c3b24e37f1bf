// How rows become e4m3 codes with a power-of-two scale (kv_quant.hip, kv_rope.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rapid_internal.h"

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

namespace {

constexpr int kMinScale = -100, kMaxScale = 119;

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b)
{
    const u16x2 m = __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b));
    return __builtin_bit_cast(uint32_t, m);
}
// |x| of two bf16 values as bit patterns, 0 for what is not finite
__device__ __forceinline__ uint32_t finite_magnitudes(uint32_t two)
{
    const uint32_t m = two & 0x7fff7fffu;
    const uint32_t lo = (m & 0xffffu) >= 0x7f80u ? 0u : m & 0xffffu;
    const uint32_t hi = m >= 0x7f800000u ? 0u : m & 0xffff0000u;
    return lo | hi;
}
// The scale exponent of a row whose largest magnitude has these bf16 bits.  (1 + f/128) 2^(E-127) <= 1.75 * 2^8 * 2^k
__device__ __forceinline__ int scale_exponent(uint32_t bits)
{
    const int k = (int)(bits >> 7) - 135 + ((bits & 127u) > 96u);
    return min(max(k, kMinScale), kMaxScale);
}
__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// The largest of a row's magnitudes, two at a time, over its LPR = 16, 8 or 4 lanes (moves between lanes in registers).
template <int LPR>
__device__ __forceinline__ uint32_t row_max(uint32_t m)
{
    auto with = [&](uint32_t other) { m = max_u16x2(m, other); };
    if (LPR == 16) {
        with(__builtin_amdgcn_update_dpp(0, m, 0x128, 0xf, 0xf, false));          // rotations by 8, 4, 2, 1 in rows of 16 lanes
        with(__builtin_amdgcn_update_dpp(0, m, 0x124, 0xf, 0xf, false));
        with(__builtin_amdgcn_update_dpp(0, m, 0x122, 0xf, 0xf, false));
        with(__builtin_amdgcn_update_dpp(0, m, 0x121, 0xf, 0xf, false));
    } else {
        if (LPR == 8) with(__builtin_amdgcn_update_dpp(0, m, 0x141, 0xf, 0xf, false));          // the mirror image in eight lanes, then inside four
        with(__builtin_amdgcn_update_dpp(0, m, 0x4e, 0xf, 0xf, false));
        with(__builtin_amdgcn_update_dpp(0, m, 0xb1, 0xf, 0xf, false));
    }
    return max(m >> 16, m & 0xffffu);
}
// From here on the scale's upper bound may bind, or a value is not finite.
constexpr uint32_t kLargeBits = 0x7e00;

// Four bf16 values (two words) times `inv`, as e4m3; all finite, and within 448 by the scale's rule.
__device__ __forceinline__ uint32_t plain_codes_of(uint32_t w0, uint32_t w1, float inv)
{
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(w0 << 16) * inv, __uint_as_float(w0 & 0xffff0000u) * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(w1 << 16) * inv, __uint_as_float(w1 & 0xffff0000u) * inv, c, true);
}
// Any four.
__device__ __forceinline__ uint32_t codes_of(uint32_t w0, uint32_t w1, float inv)
{
    const uint32_t w[2] = {w0, w1};
    float y[4];
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t bits = i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16;
        y[i] = fminf(fmaxf(__uint_as_float(bits) * inv, -448.f), 448.f);
        if ((bits & 0x7f800000u) == 0x7f800000u) bad |= 0xffu << (8 * i);
    }
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
    return ((uint32_t)c & ~bad) | (bad & 0x7f7f7f7fu);
}

// Where the rows of token `tok` of sequence b begin: codes (of a bf16 cache: its bytes) and scales of head h.
struct RowPlace { int64_t codes, scales; };
__device__ __forceinline__ RowPlace place(const KvQuantLaunch& a, int b, int tok, int h)
{
    if (a.page_shift >= 0) {
        const int64_t pg = min(max(a.page_table[(int64_t)b * a.max_pages + (tok >> a.page_shift)], 0), a.page_hi);
        const int t = tok & a.page_mask;
        return {pg * a.pstride + t * a.tstride + h * a.hstride, pg * a.spstride + h * a.shstride + t};
    }
    return {b * a.bstride + tok * a.tstride + h * a.hstride, b * a.sbstride + h * a.shstride + tok};
}

}  // namespace
