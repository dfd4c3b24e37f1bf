// Attention over a cache in 8 bits, and behind a shared prefix: the plain kernel (gfx950).
//
// One workgroup per query row.  Its four waves take every fourth token each; a lane holds d / 64 elements of the row, the scores are
// summed over the wave, and the running maximum and sum of the softmax are kept per wave and joined at the end.
#include "rapid_internal.h"

namespace {

constexpr int kWaves = 4;

__device__ __forceinline__ float bf16_value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float e4m3_value(uint8_t x) { return __builtin_amdgcn_cvt_f32_fp8((int)x, 0); }

template <int EPL>
struct RowState { float m = -INFINITY, l = 0.f, acc[EPL] = {}; };

// Tokens [0, n) of a source: keys of kv head h, row of page table or sequence b.
template <int EPL, bool QUANT>
__device__ __forceinline__ void fold_tokens(const AttnSource& s, int b, int h, int n, const float (&q)[EPL], float c, int wave, int lane,
                                            RowState<EPL>& st)
{
    for (int j = wave; j < n; j += kWaves) {
        int64_t at = h * s.hstride, sat = h * s.shstride;
        if (s.page_table) {
            const int64_t pg = min(max(s.page_table[(int64_t)b * s.max_pages + (j >> s.page_shift)], 0), s.page_hi);
            at += pg * s.pstride + (j & s.page_mask) * s.tstride;
            sat += pg * s.spstride + (j & s.page_mask);
        } else {
            at += b * s.bstride + j * s.tstride;
            sat += b * s.sbstride + j;
        }
        at += lane * EPL;
        float kx[EPL], vx[EPL], dot = 0.f;
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
            if (QUANT) {
                kx[e] = e4m3_value(static_cast<const uint8_t*>(s.k)[at + e]) * __uint_as_float((uint32_t)s.ks[sat] << 23);
                vx[e] = e4m3_value(static_cast<const uint8_t*>(s.v)[at + e]) * __uint_as_float((uint32_t)s.vs[sat] << 23);
            } else {
                kx[e] = bf16_value(static_cast<const uint16_t*>(s.k)[at + e]);
                vx[e] = bf16_value(static_cast<const uint16_t*>(s.v)[at + e]);
            }
            dot = fmaf(q[e], kx[e], dot);
        }
#pragma unroll
        for (int o = 32; o > 0; o /= 2) dot += __shfl_xor(dot, o, 64);
        const float score = dot * c;
        const float m = fmaxf(st.m, score), mu = m == -INFINITY ? 0.f : m;
        const float old = exp2f(st.m - mu), p = exp2f(score - mu);
        st.m = m;
        st.l = st.l * old + p;
#pragma unroll
        for (int e = 0; e < EPL; ++e) st.acc[e] = fmaf(p, vx[e], st.acc[e] * old);
    }
}

// Grid: (query row of the sequence, sequence); row = i * Hq + h.
template <int D, bool QUANT>
__global__ void __launch_bounds__(kWaves * 64) attn_rows(AttnRowsLaunch a)
{
    constexpr int EPL = D / 64;
    __shared__ float ml[kWaves][2];
    __shared__ float part[kWaves][D];
    const int b = blockIdx.y, i = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int Q = min(max(a.gammas ? a.gammas[b] : a.gamma, 0), a.Qmax - 1) + 1;
    const int L = max(min(a.ctx_lens[b], a.max_ctx), 0);
    const int64_t at = (((int64_t)b * a.Qmax + i) * a.Hq + h) * D;
    float q[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) q[e] = bf16_value(a.q[at + lane * EPL + e]);
    RowState<EPL> st;
    if (i < Q && L > 0) {
        if (a.prefix_len)
            fold_tokens<EPL, QUANT>(a.prefix, 0, h / a.G, min(max(a.prefix_len[0], 0), a.max_prefix), q, a.scale_log2e, wave, lane, st);
        fold_tokens<EPL, QUANT>(a.own, b, h / a.G, L - Q + i + 1, q, a.scale_log2e, wave, lane, st);
    }
    if (lane == 0) { ml[wave][0] = st.m; ml[wave][1] = st.l; }
#pragma unroll
    for (int e = 0; e < EPL; ++e) part[wave][lane * EPL + e] = st.acc[e];
    __syncthreads();
    float m = -INFINITY, l = 0.f, o = 0.f;
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, ml[w][0]);
    const float mu = m == -INFINITY ? 0.f : m;
    for (int w = 0; w < kWaves; ++w) l += ml[w][1] * exp2f(ml[w][0] - mu);
    if ((int)threadIdx.x < D) {
        for (int w = 0; w < kWaves; ++w) o += part[w][threadIdx.x] * exp2f(ml[w][0] - mu);
        const __bf16 r = (__bf16)(l == 0.f ? 0.f : o / l);
        a.out[at + threadIdx.x] = __builtin_bit_cast(uint16_t, r);
    }
    if (a.lse_out && threadIdx.x == 0)
        a.lse_out[((int64_t)b * a.Hq + h) * a.Qmax + i] = i < Q ? (m + log2f(l)) * 0.6931471805599453f : 0.f;
}

}  // namespace

hipError_t launch_attn_rows(const AttnRowsLaunch& a, hipStream_t stream)
{
    const dim3 grid(a.Qmax * a.Hq, a.B);
    const bool quant = a.own.ks != nullptr;
    auto fn = a.D == 128 ? (quant ? attn_rows<128, true> : attn_rows<128, false>) : (quant ? attn_rows<64, true> : attn_rows<64, false>);
    hipLaunchKernelGGL(fn, grid, dim3(kWaves * 64), 0, stream, a);
    return hipGetLastError();
}
