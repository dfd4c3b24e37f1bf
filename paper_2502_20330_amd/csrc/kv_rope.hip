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

// Grid: (blocks of T rows, sequences, parts of the heads).  Units of a workgroup: (row, head), U of them a thread at a time.
template <int D, bool QUANT, bool ADJACENT, int T, int U>
__global__ void __launch_bounds__(256) kv_append_rope(KvRopeLaunch a)
{
    constexpr int LPH = D / 16, UNITS = 256 / LPH;
    __shared__ float2 turns[T][D / 2];
    const KvQuantLaunch& c = a.cache;
    const int b = blockIdx.y, i0 = blockIdx.x * T, tid = threadIdx.x;
    const int Q = min(max(c.gammas ? c.gammas[b] : c.gamma, 0), c.Qmax - 1) + 1;
    if (i0 >= Q) return;
    const int first = max(min(c.ctx_lens[b], c.max_ctx), 0) - Q;          // token of row 0; negative: rows without a token
    if (first + min(i0 + T, Q) <= 0) return;
    const int h0 = blockIdx.z * a.heads_each, nh = min(a.Hq + 2 * c.Hkv - h0, a.heads_each);
    const int j = tid % LPH, half = a.rot / 2;
    const bool turned = j < a.rot / 16;
    const int lo = turned && !ADJACENT ? 8 * j : 16 * j, hi = turned && !ADJACENT ? half + 8 * j : 16 * j + 8;

    for (int u0 = tid / LPH, start = 0; start < T * nh; start += U * UNITS, u0 += U * UNITS) {
        Sixteen x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int unit = min(u0 + u * UNITS, T * nh - 1);
            const int r = T == 1 ? 0 : unit / nh, h = h0 + unit - r * nh;
            const int64_t row = (int64_t)b * c.Qmax + min(i0 + r, Q - 1);
            const uint16_t* src = h < a.Hq ? a.q + row * a.q_stride + (int64_t)h * D
                                  : h < a.Hq + c.Hkv ? a.k + row * a.k_stride + (int64_t)(h - a.Hq) * D
                                                     : a.v + row * a.v_stride + (int64_t)(h - a.Hq - c.Hkv) * D;
            x[u].lo = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + lo));
            x[u].hi = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + hi));
        }
        if (start == 0) {
            for (int t = tid; t < T * half; t += 256) {
                const int r = T == 1 ? 0 : t / half, p = t - r * half, i = min(i0 + r, Q - 1);
                const int pos = a.positions ? a.positions[(int64_t)b * c.Qmax + i] : first + i;
                turns[r][p] = turn_of(pos, a.inv_freq[p], a.amplitude);
            }
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int unit = u0 + u * UNITS;
            const int r = T == 1 ? 0 : unit / nh, h = h0 + unit - r * nh, i = i0 + r, tok = first + i;
            if (unit >= T * nh || i >= Q || tok < 0) continue;             // (all lanes of a head alike)
            const bool value = h >= a.Hq + c.Hkv;
            const Sixteen y = turned && !value ? rotated<ADJACENT>(x[u], &turns[r][8 * j]) : x[u];
            if (h < a.Hq) {
                uint16_t* dst = a.q_out + (((int64_t)b * c.Qmax + i) * a.Hq + h) * D;
                *reinterpret_cast<u32x4*>(dst + lo) = y.lo;
                *reinterpret_cast<u32x4*>(dst + hi) = y.hi;
                continue;
            }
            const int kv = h - a.Hq - (value ? c.Hkv : 0);
            const KvQuantSide& side = c.side[value];
            const RowPlace at = place(c, b, tok, kv);
            if constexpr (!QUANT) {
                *reinterpret_cast<u32x4*>(side.codes + at.codes + lo * 2) = y.lo;
                *reinterpret_cast<u32x4*>(side.codes + at.codes + hi * 2) = y.hi;
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
                *reinterpret_cast<u32x2*>(side.codes + at.codes + lo) = c_lo;
                *reinterpret_cast<u32x2*>(side.codes + at.codes + hi) = c_hi;
                if (j == 0) side.scales[at.scales] = (uint8_t)(k + 127);
            }
        }
    }
}

template <int D, bool QUANT, bool ADJACENT>
hipError_t launch(KvRopeLaunch a, hipStream_t stream)
{
    constexpr int UNITS = 256 / (D / 16);
    const int heads = a.Hq + 2 * a.cache.Hkv;
    if ((int64_t)a.cache.B * a.cache.Qmax >= 2048) {
        a.heads_each = heads;
        hipLaunchKernelGGL((kv_append_rope<D, QUANT, ADJACENT, 4, 4>), dim3((a.cache.Qmax + 3) / 4, a.cache.B, 1), dim3(256), 0, stream, a);
    } else {
        a.heads_each = heads < UNITS ? heads : UNITS;
        hipLaunchKernelGGL((kv_append_rope<D, QUANT, ADJACENT, 1, 1>), dim3(a.cache.Qmax, a.cache.B, (heads + a.heads_each - 1) / a.heads_each),
                           dim3(256), 0, stream, a);
    }
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
