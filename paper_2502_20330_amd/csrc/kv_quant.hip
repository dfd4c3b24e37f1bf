// A KV cache in 8 bits: rows are quantised as they are appended, and read back (gfx950).
//
// A row is the d values of one (token, kv head) of K or of V.  With a = max |x| over its finite values, the scale is the smallest
// power of two s with a <= 448 s (448: the largest e4m3 number), between 2^-100 and 2^119, and the codes are x / s rounded to
// e4m3.  A power of two makes x / s exact, so that there is one rounding and nothing to agree on between a division and a multiplication by a reciprocal, and code * s is a bf16 number.
//
// Both kernels only move bytes: 2 d + d + 1 per row.  Eight values, 16 bytes, a lane; d / 8 lanes hold a row and find its maximum by
// rotations inside them.  The maximum is taken on the bits: for values of one sign the order of bf16 numbers is that of their
// bit patterns, two of which are compared by one packed instruction.
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

// The largest of a row's magnitudes, two at a time, over its LPR = 16 or 8 lanes (moves between lanes in registers).
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
        with(__builtin_amdgcn_update_dpp(0, m, 0x141, 0xf, 0xf, false));          // the mirror image in eight lanes, then inside four
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

// Where the rows of token `tok` of sequence b begin: codes and scales of head h.
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

// Grid: (blocks of tokens, kv heads, sequence and side).  d / 8 lanes a row, U rows a thread, whose loads are all under way before the first is
// worked on: a prompt of 64K tokens (8 heads of 128) takes 84 us with one, 72 with four, 32K tokens are read in 42 and 37; a round's few rows are spread over more
// workgroups with one.
template <int D, int U>
__global__ void __launch_bounds__(256) kv_append_quant(KvQuantLaunch a)
{
    constexpr int LPR = D / 8, RPB = 256 / LPR;
    const int b = blockIdx.z >> 1, h = blockIdx.y;
    const KvQuantSide s = a.side[blockIdx.z & 1];
    const int Q = min(max(a.gammas ? a.gammas[b] : a.gamma, 0), a.Qmax - 1) + 1;
    const int i0 = blockIdx.x * RPB * U + threadIdx.x / LPR, c = threadIdx.x % LPR;
    const int first = max(min(a.ctx_lens[b], a.max_ctx), 0) - Q;           // token of row 0; negative: rows without a token
    u32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = i0 + u * RPB;
        const int64_t src = (((int64_t)b * a.Qmax + min(i, Q - 1)) * a.Hkv + h) * D + c * 8;
        x[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(s.rows + src));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = i0 + u * RPB, tok = first + i;
        if (i >= Q || tok < 0) continue;                   // (all lanes of a row alike)
        const u32x4 v = x[u];
        uint32_t m = row_max<LPR>(max_u16x2(max_u16x2(v[0] & 0x7fff7fffu, v[1] & 0x7fff7fffu), max_u16x2(v[2] & 0x7fff7fffu, v[3] & 0x7fff7fffu)));
        const bool large = __any(m >= kLargeBits);
        if (large)
            m = row_max<LPR>(max_u16x2(max_u16x2(finite_magnitudes(v[0]), finite_magnitudes(v[1])),
                                       max_u16x2(finite_magnitudes(v[2]), finite_magnitudes(v[3]))));
        const int k = scale_exponent(m);
        const float inv = power_of_two(-k);
        u32x2 codes = {plain_codes_of(v[0], v[1], inv), plain_codes_of(v[2], v[3], inv)};
        if (large) codes = u32x2{codes_of(v[0], v[1], inv), codes_of(v[2], v[3], inv)};
        const RowPlace at = place(a, b, tok, h);
        *reinterpret_cast<u32x2*>(s.codes + at.codes + c * 8) = codes;
        if (c == 0) s.scales[at.scales] = (uint8_t)(k + 127);
    }
}

template <int D, int U>
__global__ void __launch_bounds__(256) kv_read_quant(KvQuantLaunch a)
{
    constexpr int LPR = D / 8, RPB = 256 / LPR;
    const int b = blockIdx.z >> 1, h = blockIdx.y;
    const KvQuantSide s = a.side[blockIdx.z & 1];
    const int Q = min(max(a.gammas ? a.gammas[b] : a.gamma, 0), a.Qmax - 1) + 1;
    const int i0 = blockIdx.x * RPB * U + threadIdx.x / LPR, c = threadIdx.x % LPR;
    const int first = max(min(a.ctx_lens[b], a.max_ctx), 0) - Q;
    u32x2 x[U];
    uint32_t scale[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = i0 + u * RPB, tok = first + i;
        x[u] = u32x2{0, 0};
        scale[u] = 127;
        if (i < Q && tok >= 0) {
            const RowPlace at = place(a, b, tok, h);
            x[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(s.codes + at.codes + c * 8));
            scale[u] = s.scales[at.scales];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = i0 + u * RPB;
        if (i >= a.Qmax) return;
        const float f = __uint_as_float(scale[u] << 23);
        u32x4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bf16x2 two = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[u][j >> 1], f, true)
                                     : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[u][j >> 1], f, false);
            y[j] = __builtin_bit_cast(uint32_t, two);
        }
        *reinterpret_cast<u32x4*>(s.rows + (((int64_t)b * a.Qmax + i) * a.Hkv + h) * D + c * 8) = y;
    }
}

// Four rows a thread where that still leaves eight workgroups a compute unit.
constexpr int kRowsAThread = 4;
bool many_rows(const KvQuantLaunch& a)
{
    const int64_t rows = (int64_t)a.B * a.Qmax * a.Hkv * 2;
    return rows * (a.D / 8) >= (int64_t)256 * kRowsAThread * 2048 && a.Qmax >= 256 / (a.D / 8) * kRowsAThread;
}
dim3 row_grid(const KvQuantLaunch& a, int per_thread)
{
    const int rows = 256 / (a.D / 8) * per_thread;
    return dim3((a.Qmax + rows - 1) / rows, a.Hkv, 2 * a.B);
}

}  // namespace

hipError_t launch_kv_append_quant(const KvQuantLaunch& a, hipStream_t stream)
{
    const bool many = many_rows(a);
    auto fn = a.D == 128 ? (many ? kv_append_quant<128, kRowsAThread> : kv_append_quant<128, 1>)
                         : (many ? kv_append_quant<64, kRowsAThread> : kv_append_quant<64, 1>);
    hipLaunchKernelGGL(fn, row_grid(a, many ? kRowsAThread : 1), dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_kv_read_quant(const KvQuantLaunch& a, hipStream_t stream)
{
    const bool many = many_rows(a);
    auto fn = a.D == 128 ? (many ? kv_read_quant<128, kRowsAThread> : kv_read_quant<128, 1>)
                         : (many ? kv_read_quant<64, kRowsAThread> : kv_read_quant<64, 1>);
    hipLaunchKernelGGL(fn, row_grid(a, many ? kRowsAThread : 1), dim3(256), 0, stream, a);
    return hipGetLastError();
}
