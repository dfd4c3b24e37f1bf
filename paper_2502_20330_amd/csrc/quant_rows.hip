// Rows of bf16 values as 8-bit integers with a scale for each row (gfx950).
//
//     code[c] = 127 x[c] / m to the nearest whole number, ties to even;   scale = m / 127;   m = max |x[c]|
//
// 127 x is exact in 32 bits (7 bits more than bf16's 8), and 127 x / m is a ratio of a 15-bit and an 8-bit number: it lies on the border between two
// codes or at least 2^-17 of a code's step away from it, so that the correctly rounded quotient of 32 bits falls on the same side as the exact one.  (A
// multiplication by 127 / m does not: x = m / 2 is a border, and comes out on either side of it.)
// Rows of 2 cols bytes are read once, held in registers between the maximum and the codes, and written as pitch bytes: bound by memory.
#include "rapid_internal.h"

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

namespace {

constexpr uint32_t kNotFinite = 0x7f80;

// The largest magnitude of eight values, as bf16 bits (two at a time: the order of magnitudes is that of their bits).
__device__ __forceinline__ uint32_t largest_bits(const u32x4& v, uint32_t m)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m = max(m, v[i] & 0x7fffu);
        m = max(m, v[i] >> 16 & 0x7fffu);
    }
    return m;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t m)
{
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, x));
    return m;
}

// What a row is divided by.  Where 127 m might overflow, both sides are 2^-64 of themselves: what of x that loses has a code of 0 anyhow.
struct Divisor {
    float m, pre;
    __device__ __forceinline__ explicit Divisor(uint32_t bits)
    {
        m = __uint_as_float(bits << 16);
        pre = m > 0x1p100f ? 0x1p-64f : 1.0f;
        m = bits == 0 || bits >= kNotFinite ? INFINITY : m * pre;          // nothing, or nothing finite: codes of 0
    }
    __device__ __forceinline__ uint32_t code(uint32_t x_bits) const        // x as a number of 32 bits
    {
        const float x = __uint_as_float(x_bits) * pre;
        return (uint32_t)(int)rintf(127.0f * x / m) & 0xffu;
    }
    __device__ __forceinline__ u32x2 codes(const u32x4& v) const
    {
        if (m == INFINITY) return u32x2{0, 0};
        u32x2 r;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            r[i] = code(v[2 * i] << 16) | code(v[2 * i] & 0xffff0000u) << 8 | code(v[2 * i + 1] << 16) << 16 | code(v[2 * i + 1] & 0xffff0000u) << 24;
        return r;
    }
};
__device__ __forceinline__ float scale_of(uint32_t bits)
{
    return bits >= kNotFinite ? __uint_as_float(0x7fc00000u) : __uint_as_float(bits << 16) / 127.0f;
}

// LANES lanes a row, which hold it in NV vectors of eight values each; NV = 0: rows of any length, read twice.
template <int LANES, int NV>
__global__ void __launch_bounds__(256) quant_rows(QuantRowsLaunch a)
{
    const int tid = threadIdx.x, lane = tid % LANES;
    const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + tid / LANES;
    if (row >= a.rows) return;                               // (whole waves; a workgroup of one row has it)
    const u32x4* src = reinterpret_cast<const u32x4*>(a.x + row * a.stride);
    u32x2* dst = reinterpret_cast<u32x2*>(a.codes + row * a.pitch);
    const int n = a.cols / 8, all = a.pitch / 8;
    uint32_t m = 0;
    u32x4 v[NV ? NV : 1];
    if (NV) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = lane + i * LANES;
            v[i] = at < n ? __builtin_nontemporal_load(src + at) : u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) m = largest_bits(v[i], m);
    } else {
        for (int at = lane; at < n; at += LANES) m = largest_bits(src[at], m);
    }
    m = wave_max(m);
    if (LANES > 64) {
        __shared__ uint32_t part[4];
        if (tid % 64 == 0) part[tid / 64] = m;
        __syncthreads();
        m = max(max(part[0], part[1]), max(part[2], part[3]));
    }
    if (lane == 0) a.scales[row] = scale_of(m);
    const Divisor by(m);
    if (NV) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = lane + i * LANES;
            if (at < all) dst[at] = by.codes(v[i]);          // (zeros where there are no values)
        }
    } else {
        for (int at = lane; at < all; at += LANES) dst[at] = at < n ? by.codes(src[at]) : u32x2{0, 0};
    }
}

}  // namespace

hipError_t launch_quant_rows(const QuantRowsLaunch& a, hipStream_t stream)
{
    const int vectors = (a.pitch / 8 + 255) / 256;           // a thread's, of a workgroup a row
    auto fn = vectors <= 1 ? quant_rows<256, 1> : vectors <= 2 ? quant_rows<256, 2> : vectors <= 4 ? quant_rows<256, 4> : quant_rows<256, 0>;
    hipLaunchKernelGGL(fn, dim3((unsigned)a.rows), dim3(256), 0, stream, a);
    return hipGetLastError();
}
