// Rows of bf16 values as 8-bit integers with a scale for each row (gfx950): row_codes.h has the mathematics.
// Rows of 2 cols bytes are read once, held in registers between the maximum and the codes, and written as pitch bytes: bound by memory.
#include "rapid_internal.h"
#include "row_codes.h"

namespace {

// A row to a workgroup, whose threads hold it in NV vectors of eight values each; NV = 0: rows of any length, read twice.
template <int NV>
__global__ void __launch_bounds__(256) quant_rows(QuantRowsLaunch a)
{
    __shared__ uint32_t part[4];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const u32x4* src = reinterpret_cast<const u32x4*>(a.x + row * a.stride);
    u32x2* dst = reinterpret_cast<u32x2*>(a.codes + row * a.pitch);
    const int n = a.cols / 8, all = a.pitch / 8;
    uint32_t m = 0;
    u32x4 v[NV ? NV : 1];
    if (NV) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = tid + i * 256;
            v[i] = at < n ? __builtin_nontemporal_load(src + at) : u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) m = largest_two(v[i], m);
    } else {
        for (int at = tid; at < n; at += 256) m = largest_two(src[at], m);
    }
    m = wave_max(m);
    if (tid % 64 == 0) part[tid / 64] = m;
    __syncthreads();
    m = max(max(part[0], part[1]), max(part[2], part[3]));
    if (tid == 0) a.scales[row] = scale_of(m);
    const Divisor by(m);
    if (NV) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = tid + i * 256;
            if (at < all) dst[at] = by.codes(v[i]);          // (zeros where there are no values)
        }
    } else {
        for (int at = tid; at < all; at += 256) dst[at] = at < n ? by.codes(src[at]) : u32x2{0, 0};
    }
}

}  // namespace

// (A wave to a row: 128256 rows of 4096 268 us, 77 rows of 8192 5.4; a workgroup to a row 251 and 4.1.)
hipError_t launch_quant_rows(const QuantRowsLaunch& a, hipStream_t stream)
{
    const int vectors = (a.pitch / 8 + 255) / 256;
    auto fn = vectors <= 1 ? quant_rows<1> : vectors <= 2 ? quant_rows<2> : vectors <= 4 ? quant_rows<4> : vectors <= 8 ? quant_rows<8> : quant_rows<0>;
    hipLaunchKernelGGL(fn, dim3((unsigned)a.rows), dim3(256), 0, stream, a);
    return hipGetLastError();
}
