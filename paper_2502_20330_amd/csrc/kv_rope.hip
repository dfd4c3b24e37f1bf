// Rotary positions on the way into the cache: a round's queries, keys and values in one pass (gfx950).
//
// Pair c of a head's first `rot` elements is turned by the angle t = pos * inv_freq[c]:  (x, y) -> a (x cos t - y sin t, y cos t + x sin t).
// Queries go to a buffer of their own, keys into the cache, values are copied into it; a cache in 8 bits takes the codes of the row in bf16
// (kv_codes.h), so that a row is what rotating and appending it in turn would leave.
//
// It moves 4 d (Hq + 2 Hkv) bytes a row and computes next to nothing, so what counts is memory, and for a round's few rows the chain of dependent
// loads.  An angle is common to all heads of a row: a workgroup forms those of its rows once, in LDS, while its first loads are under way.  The
// angle is a product in 64 bits, of which whole turns are taken off before it is rounded to 32: at position 131071 an angle of 32 bits would be
// off by 4e-3 radians, this one is within 2^-25 turns up to position 2^28.
// A lane holds 16 elements of a head, in two pieces of 16 bytes that hold both sides of their pairs; d / 16 lanes hold a head.
#include "kv_codes.h"
#include "rapid_internal.h"

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

namespace {

// cos and sin of pos * freq, times a.
__device__ __forceinline__ float2 turn_of(int pos, float freq, float a)
{
    const double turns = (double)pos * (double)freq * 0.15915494309189533577;
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    return make_float2(a * c, a * s);
}

struct Sixteen { u32x4 lo, hi; };

__device__ __forceinline__ void turn(float& x, float& y, float2 t)
{
    const float x0 = x;
    x = fmaf(x0, t.x, -(y * t.y));
    y = fmaf(y, t.x, x0 * t.y);
}
// cs: the turns of this lane's eight pairs.
template <bool ADJACENT>
__device__ __forceinline__ Sixteen rotated(const Sixteen& x, const float2* cs)
{
    float f[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t w = i < 4 ? x.lo[i] : x.hi[i - 4];
        f[2 * i] = __uint_as_float(w << 16);
        f[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (ADJACENT) turn(f[2 * i], f[2 * i + 1], cs[i]);
        else turn(f[i], f[8 + i], cs[i]);
    }
    bf16x8 lo, hi;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo[i] = (__bf16)f[i];
        hi[i] = (__bf16)f[8 + i];
    }
    return {__builtin_bit_cast(u32x4, lo), __builtin_bit_cast(u32x4, hi)};
}

__device__ __forceinline__ uint32_t largest_of(const u32x4& v, bool finite)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max_u16x2(m, finite ? finite_magnitudes(v[i]) : v[i] & 0x7fff7fffu);
    return m;
}

constexpr int kMostThreads = 512;

// The 16 elements of a kv head that this lane holds; `codes` and `scale` are the head's.
template <bool QUANT, int LPH>
__device__ __forceinline__ void store_row(const Sixteen& y, uint8_t* codes, uint8_t* scale, int lo, int hi, int j)
{
    if constexpr (!QUANT) {
        *reinterpret_cast<u32x4*>(codes + lo * 2) = y.lo;
        *reinterpret_cast<u32x4*>(codes + hi * 2) = y.hi;
    } else {
        uint32_t m = row_max<LPH>(max_u16x2(largest_of(y.lo, false), largest_of(y.hi, false)));
        const bool large = m >= kLargeBits;
        if (large) m = row_max<LPH>(max_u16x2(largest_of(y.lo, true), largest_of(y.hi, true)));
        const int k = scale_exponent(m);
        const float inv = power_of_two(-k);
        u32x2 c_lo = {plain_codes_of(y.lo[0], y.lo[1], inv), plain_codes_of(y.lo[2], y.lo[3], inv)};
        u32x2 c_hi = {plain_codes_of(y.hi[0], y.hi[1], inv), plain_codes_of(y.hi[2], y.hi[3], inv)};
        if (large) {
            c_lo = u32x2{codes_of(y.lo[0], y.lo[1], inv), codes_of(y.lo[2], y.lo[3], inv)};
            c_hi = u32x2{codes_of(y.hi[0], y.hi[1], inv), codes_of(y.hi[2], y.hi[3], inv)};
        }
        *reinterpret_cast<u32x2*>(codes + lo) = c_lo;
        *reinterpret_cast<u32x2*>(codes + hi) = c_hi;
        if (j == 0) *scale = (uint8_t)(k + 127);
    }
}

// Grid: (rows, sequences).  A workgroup's units are the heads of a row, of q, k and v.
template <int D, bool QUANT, bool ADJACENT>
__global__ void __launch_bounds__(kMostThreads) kv_append_rope(KvRopeLaunch a)
{
    constexpr int LPH = D / 16;
    const int at_a_time = blockDim.x / LPH;
    __shared__ float2 turns[D / 2];
    const KvQuantLaunch& c = a.cache;
    const int b = blockIdx.y, i = blockIdx.x, tid = threadIdx.x;
    const int heads = a.Hq + 2 * c.Hkv, j = tid % LPH, half = a.rot / 2;
    const bool turned = j < a.rot / 16;
    const int lo = turned && !ADJACENT ? 8 * j : 16 * j, hi = turned && !ADJACENT ? half + 8 * j : 16 * j + 8;
    const int64_t row = (int64_t)b * c.Qmax + i;
    const uint16_t *q = a.q + row * a.q_stride, *k = a.k + row * a.k_stride, *v = a.v + row * a.v_stride;
    Sixteen x;
    auto load = [&](int h) {
        const uint16_t* src = h < a.Hq ? q + (int64_t)h * D : h < a.Hq + c.Hkv ? k + (int64_t)(h - a.Hq) * D : v + (int64_t)(h - a.Hq - c.Hkv) * D;
        x.lo = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + lo));
        x.hi = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + hi));
    };
    const float freq = tid < half ? a.inv_freq[tid] : 0.f;
    const int Q = min(max(c.gammas ? c.gammas[b] : c.gamma, 0), c.Qmax - 1) + 1;
    const int tok = max(min(c.ctx_lens[b], c.max_ctx), 0) - Q + i;        // negative: a row without a token
    if (i >= Q || tok < 0) return;
    const RowPlace at = place(c, b, tok, 0);
    load(min(tid / LPH, heads - 1));
    if (tid < half) turns[tid] = turn_of(a.positions ? a.positions[row] : tok, freq, a.amplitude);
    __syncthreads();
    for (int h = tid / LPH; h < heads; h += at_a_time) {                       // (all lanes of a head alike)
        const bool value = h >= a.Hq + c.Hkv;
        const Sixteen y = turned && !value ? rotated<ADJACENT>(x, &turns[8 * j]) : x;
        if (h + at_a_time < heads) load(h + at_a_time);
        if (h < a.Hq) {
            uint16_t* dst = a.q_out + (row * a.Hq + h) * D;
            *reinterpret_cast<u32x4*>(dst + lo) = y.lo;
            *reinterpret_cast<u32x4*>(dst + hi) = y.hi;
        } else {
            const int kv = h - a.Hq - (value ? c.Hkv : 0);
            const KvQuantSide& side = c.side[value];
            store_row<QUANT, LPH>(y, side.codes + at.codes + kv * c.hstride, side.scales + at.scales + kv * c.shstride, lo, hi, j);
        }
    }
}

// A row of q, k and v to a workgroup, with as many threads as its heads take, or the half, third .. of them that is at most 512.  The more workgroups a compute
// unit has, the more of their waits for lengths, pages and angles pass under others' loads, but a thread that has a second head to do waits twice.
// 64K rows of 32 / 8 / 8 heads of 128, which take 384 threads: 282 us with these, 292 with 256, 297 with 128, 307 with 64 (two rows to a workgroup: 20 us more, four
// 30, eight 47); into 8 bits 281, with 256 threads 272; 72 such rows 3.3, 4.9 with 64, in 8 bits 3.6 and 5.3; 2800 rows of 16 / 8 / 8 heads of 64 in 8 bits, which take 128: 8.5, 10.2 with 256, 13.7 with 384.
template <int D, bool QUANT, bool ADJACENT>
hipError_t launch(const KvRopeLaunch& a, hipStream_t stream)
{
    const int all = (a.Hq + 2 * a.cache.Hkv) * (D / 16), parts = (all + kMostThreads - 1) / kMostThreads;
    const int threads = ((all + parts - 1) / parts + 63) / 64 * 64;
    hipLaunchKernelGGL((kv_append_rope<D, QUANT, ADJACENT>), dim3(a.cache.Qmax, a.cache.B), dim3(threads), 0, stream, a);
    return hipGetLastError();
}
template <int D>
hipError_t launch(const KvRopeLaunch& a, hipStream_t stream)
{
    const bool quant = a.cache.side[0].scales != nullptr;
    if (a.adjacent) return quant ? launch<D, true, true>(a, stream) : launch<D, false, true>(a, stream);
    return quant ? launch<D, true, false>(a, stream) : launch<D, false, false>(a, stream);
}

}  // namespace

hipError_t launch_kv_append_rope(const KvRopeLaunch& a, hipStream_t stream)
{
    return a.cache.D == 128 ? launch<128>(a, stream) : launch<64>(a, stream);
}
