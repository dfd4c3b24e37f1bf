// The output head on 8-bit integers (gfx950):  z[r][v] = s_h[r] s_w[v] sum_k c_h[r][k] c_w[v][k]
//
// Codes and scales are those of quant_rows.hip: a scale for each row of h and for each vocabulary entry.  The sums are exact in 32 bits (127^2 times
// up to 2^17 terms stays below 2^31).  Half of the bytes of bf16 weights, which are what bounds the head; the matrix instruction takes 64 codes of a row
// where that of bf16 takes 32 numbers, from the same 16 bytes a lane, so that tiles, rings and swizzle are those of lm_head.hip
// (lm_head_stream.h).
#include "lm_head_stream.h"

namespace {

enum Kind { kNarrow, kWide };                            // slabs of 256 bytes, of 512
template <int NR, class F>
hipError_t for_build(Kind kind, F f)
{
    if (kind == kNarrow) return f(lm_head_stream<Int8Elements, 256, NR, false>, lds_bytes());
    if constexpr (NR >= 4) return f(lm_head_shared<Int8Elements, NR, false>, Shared<NR>::LDS);
    else return f(lm_head_stream<Int8Elements, 512, NR, false>, lds_bytes());
}
template <class F>
hipError_t for_build(int nr, Kind kind, F f)
{
    switch (nr) {
        case 1: return for_build<1>(kind, f);
        case 2: return for_build<2>(kind, f);
        case 3: return for_build<3>(kind, f);
        case 4: return for_build<4>(kind, f);
        case 5: return for_build<5>(kind, f);
        case 6: return for_build<6>(kind, f);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t configure_lm_head_quant()
{
    for (int nr = 1; nr <= 6; ++nr)
        for (Kind kind : {kNarrow, kWide}) {
            const hipError_t e = for_build(nr, kind, [](auto kernel, int lds) {
                return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
            });
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

hipError_t launch_lm_head_quant(const LmHeadLaunch& a, hipStream_t stream)
{
    if (a.row_bytes % 256 != 0 || a.nb < 1 || a.nb > kNB) return hipErrorInvalidValue;
    const int nwg = (a.vocab + a.nb * 16 - 1) / (a.nb * 16);
    return for_build((a.n_rows + 15) / 16, a.row_bytes % 512 ? kNarrow : kWide, [&](auto kernel, int lds) {
        hipLaunchKernelGGL(kernel, dim3(nwg), dim3(kWaves * 64), lds, stream, a);
        return hipGetLastError();
    });
}
