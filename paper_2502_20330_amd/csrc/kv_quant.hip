// A KV cache in 8 bits: rows are quantised as they are appended, and read back (gfx950).
//
// A row is the d values of one (token, kv head) of K or of V.  With a = max |x| over its finite values, the scale is the smallest
// power of two s with a <= 448 s (448: the largest e4m3 number), between 2^-100 and 2^119, and the codes are x / s rounded to
// e4m3.  A power of two makes x / s exact, so that there is one rounding and nothing to agree on between a division and a multiplication by a reciprocal, and code * s is a bf16 number.
//
// Both kernels only move bytes: 2 d + d + 1 per row.  Eight values, 16 bytes, a lane; d / 8 lanes hold a row and find its maximum by
// rotations inside them.  The maximum is taken on the bits: for values of one sign the order of bf16 numbers is that of their
// bit patterns, two of which are compared by one packed instruction.
#include "kv_codes.h"
#include "rapid_internal.h"

namespace {

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
