// The output head on 8-bit integers (gfx950):  z[r][v] = s_h[r] s_w[v] sum_k c_h[r][k] c_w[v][k]
//
// Codes and scales are those of quant_rows.hip: a scale for each row of h and for each vocabulary entry.  The sums are exact in 32 bits (127^2 times
// up to 2^17 terms stays below 2^31).  Half of the bytes of bf16 weights, which are what bounds the head; the matrix instruction takes 64 codes of a row
// where that of bf16 takes 32 numbers, from the same 16 bytes a lane, so that tiles, rings and swizzle are those of lm_head.hip
// (lm_head_stream.h).  Measured, 4096 x 128256 (525 MB, 75.6 us at the rate of a pure read): one row 79.2 us; with the launch that brings h to codes, 72 rows 96 to 98, of
// which about 15 are the logits' stores; 11 rows of 3584 x 152064 90 (79.5).
#include "lm_head_stream.h"
#include "row_codes.h"

namespace {

// Vocabularies that leave half of a workgroup's waves without a block (up to 8192 entries on 256 compute units): the waves share the slabs instead of the
// blocks, each takes every fourth one for all blocks, and the sums meet in LDS.  (Whole numbers: the order does not matter.)  5120 x 4000, with the
// rows' codes: one row 12.6 -> 10.4 us, 20 rows 17.1 -> 12.3, 60 rows 22.1 -> 17.1; x 8000 13.2 -> 12.8, 17.7 -> 15.3, 23.8 -> 20.7; with three blocks of four (x 12000) one
// row loses, 15.3 -> 16.1, what 60 rows win.
constexpr int kSplitBlocks = 2;
template <int SB, int NR>
__global__ void __launch_bounds__(kWaves * 64) lm_head_split(LmHeadLaunch a)
{
    using T = Tile<SB>;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ln = lane & 15, lg = lane >> 4;
    const int nb = a.nb, v0 = blockIdx.x * nb * 16;
    const uint32_t row_bytes = (uint32_t)a.row_bytes;
    const int mine = (a.row_bytes / SB - wave + kWaves - 1) / kWaves;      // slabs wave, wave + 4, ..
    char* ring = smem + wave * kRing;
    const uint32_t ring_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + wave * kRing;
    uint32_t woff[T::NLD], coff[T::NLD];
    int rrow[T::NLD];
#pragma unroll
    for (int e = 0; e < T::NLD; ++e) {
        rrow[e] = T::RPI * e + lane / T::CPR;
        coff[e] = (uint32_t)((lane % T::CPR) ^ (rrow[e] & 15)) * 16u;
        woff[e] = (uint32_t)rrow[e] * row_bytes + coff[e];
    }
    // tile j of this wave's slab s: row blocks of h, then blocks of W
    auto issue = [&](int s, int j, int slot) {
        const int64_t kbyte = (int64_t)(wave + s * kWaves) * SB;
        const uint32_t dst = ring_lds + slot * T::BYTES;
        const char* base = j < NR ? static_cast<const char*>(a.h) + kbyte
                                  : static_cast<const char*>(a.w) + (int64_t)loaded_row0(a, v0 + (j - NR) * 16) * row_bytes + kbyte;
#pragma unroll
        for (int e = 0; e < T::NLD; ++e) {
            if (j < NR) dma16_keep(base, (uint32_t)min(j * 16 + rrow[e], a.n_rows - 1) * row_bytes + coff[e], dst + e * 1024);
            else dma16(base, woff[e], dst + e * 1024);
        }
    };
    intx4 acc[kSplitBlocks][NR];
#pragma unroll
    for (int j = 0; j < kSplitBlocks; ++j)
#pragma unroll
        for (int rb = 0; rb < NR; ++rb) acc[j][rb] = intx4{0, 0, 0, 0};
    if (mine > 0) {
        int ps = 0, pj = 0, pt = 0;                      // next tile to request: slab, index, linear number
        auto request_next = [&]() {
            issue(min(ps, mine - 1), ps < mine ? pj : 0, pt & (T::SLOTS - 1));             // (past the end any: the count stays uniform)
            ++pt;
            if (++pj >= NR + nb) { pj = 0; ++ps; }
        };
#pragma unroll
        for (int j = 0; j < T::AHEAD; ++j) request_next();
        intx4 hreg[NR][T::KS];
        int t = 0;
        for (int s = 0; s < mine; ++s) {
#pragma unroll
            for (int j = 0; j < NR + kSplitBlocks; ++j) {
                if (j < NR + nb) {
                    wait_loads<(T::AHEAD - 1) * T::NLD>();
                    request_next();
                    const char* tile = ring + (t & (T::SLOTS - 1)) * T::BYTES + ln * SB;
                    ++t;
#pragma unroll
                    for (int ks = 0; ks < T::KS; ++ks) {
                        const intx4 x = *reinterpret_cast<const intx4*>(tile + (((ks * 4 + lg) ^ ln) * 16));
                        if (j < NR) {
                            hreg[j < NR ? j : 0][ks] = x;
                        } else {
#pragma unroll
                            for (int rb = 0; rb < NR; ++rb) acc[j >= NR ? j - NR : 0][rb] = Int8Elements::mma(x, hreg[rb][ks], acc[j >= NR ? j - NR : 0][rb]);
                        }
                    }
                    lds_reads_done();
                }
            }
        }
        wait_loads<0>();
    }
    __syncthreads();                                     // the rings are dead from here on
    intx4* part = reinterpret_cast<intx4*>(smem);        // [kWaves][kSplitBlocks][NR][64]
#pragma unroll
    for (int j = 0; j < kSplitBlocks; ++j)
#pragma unroll
        for (int rb = 0; rb < NR; ++rb)
            if (j < nb) part[((wave * kSplitBlocks + j) * NR + rb) * 64 + lane] = acc[j][rb];
    __syncthreads();
    intx4 sum[kNBW][NR];                                 // block `wave`, if there is one
#pragma unroll
    for (int j = 0; j < kNBW; ++j)
#pragma unroll
        for (int rb = 0; rb < NR; ++rb) sum[j][rb] = intx4{0, 0, 0, 0};
    if (wave < nb)
#pragma unroll
        for (int rb = 0; rb < NR; ++rb)
#pragma unroll
            for (int w = 0; w < kWaves; ++w) sum[0][rb] += part[((w * kSplitBlocks + wave) * NR + rb) * 64 + lane];
    finish<Int8Elements, NR>(a, a.h_scales, sum, wave < nb ? 1 : 0, v0, reinterpret_cast<float*>(smem + kWaves * kRing));
}

// Few rows that are short: the workgroups bring them to codes by themselves, while their first tiles of W are on the way, which spares a launch and its end.
// The rows go HBM -> LDS into the slot of each wave's ring that is filled last, a wave takes every fourth piece of 512 values, and the codes stay in LDS: row r's
// chunk c of 16 codes at c ^ r, so that rows do not meet in a bank.  (One row of 4096 x 128256 80.6 -> 79.2 us, 2048 x 128256 43.7 -> 41.8, 1024 x 50000 12.9 -> 11.2,
// eight rows of that 13.5 -> 13.0, one of 8192 x 32000 43.7 -> 43.3; beyond, every workgroup doing all rows costs more: 16 rows of 1024 x 50000 13.9 and 15.3.)
constexpr int kOwnCodes = 8192;                          // n_rows * hidden at most
struct OwnCodes {
    static constexpr int CODES = lds_bytes(), SCALES = CODES + kOwnCodes, PART = SCALES + 16 * 4, LDS = PART + kOwnCodes / 512 * 4;
};
static_assert(kOwnCodes / kWaves * 2 <= Tile<512>::BYTES, "pieces of a wave, in a slot of its ring");
bool own_codes(const LmHeadLaunch& a) { return a.n_rows <= 16 && a.hidden % 512 == 0 && (int64_t)a.n_rows * a.hidden <= kOwnCodes && a.nb > kSplitBlocks; }
__global__ void __launch_bounds__(kWaves * 64) lm_head_own_codes(LmHeadLaunch a, const uint16_t* h)
{
    using T = Tile<512>;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ln = lane & 15, lg = lane >> 4;
    const int nb = a.nb, nbw = (nb + kWaves - 1 - wave) / kWaves, v0 = blockIdx.x * nb * 16;
    const uint32_t row_bytes = (uint32_t)a.row_bytes;    // (the hidden size: rows are whole slabs)
    const int nslab = a.row_bytes / 512, s0 = first_slab<Int8Elements>(nslab);
    char* ring = smem + wave * kRing;
    const uint32_t ring_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + wave * kRing;
    char* codes = smem + OwnCodes::CODES;
    float* scales = reinterpret_cast<float*>(smem + OwnCodes::SCALES);
    uint32_t* part = reinterpret_cast<uint32_t*>(smem + OwnCodes::PART);       // the largest magnitude of each piece

    const int mine = (a.n_rows * nslab + kWaves - 1 - wave) / kWaves;          // pieces wave, wave + 4, ..: at most 4
    for (int i = 0; i < mine; ++i)
        dma16_keep(reinterpret_cast<const char*>(h), (uint32_t)((wave + i * kWaves) * 1024 + lane * 16), ring_lds + T::AHEAD * T::BYTES + i * 1024);
    uint32_t woff[T::NLD];
#pragma unroll
    for (int e = 0; e < T::NLD; ++e) {
        const int row = T::RPI * e + lane / T::CPR;
        woff[e] = (uint32_t)row * row_bytes + (uint32_t)((lane % T::CPR) ^ (row & 15)) * 16u;
    }
    int ps = 0, pj = 0, pt = 0;                          // next tile to request: slab, block, linear number
    auto request_next = [&]() {
        const uint32_t dst = ring_lds + (pt & (T::SLOTS - 1)) * T::BYTES;
        if (ps < nslab) {
            const char* base = static_cast<const char*>(a.w) + (int64_t)loaded_row0(a, v0 + (pj * kWaves + wave) * 16) * row_bytes +
                               slab_of<Int8Elements>(ps, s0, nslab) * 512;
#pragma unroll
            for (int e = 0; e < T::NLD; ++e) dma16(base, woff[e], dst + e * 1024);
        } else {                                         // past the end: the first piece of h keeps the count uniform
#pragma unroll
            for (int e = 0; e < T::NLD; ++e) dma16_keep(reinterpret_cast<const char*>(h), (uint32_t)lane * 16u, dst + e * 1024);
        }
        ++pt;
        if (++pj >= nbw) { pj = 0; ++ps; }
    };
    if (nbw > 0) {
#pragma unroll
        for (int j = 0; j < T::AHEAD; ++j) request_next();
        wait_loads<T::AHEAD * T::NLD>();                 // this wave's pieces of h have landed
    } else {
        wait_loads<0>();
    }
    const char* raw = ring + T::AHEAD * T::BYTES + lane * 16;
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
        const uint32_t m = wave_max(largest_two(*reinterpret_cast<const u32x4*>(raw + i * 1024), 0));
        if (lane == 0) part[wave + i * kWaves] = m;
    }
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
        const int q = wave + i * kWaves, r = q / nslab, x = q - r * nslab;     // piece x of row r
        const uint32_t m = wave_max(lane < nslab ? part[r * nslab + lane] : 0);
        const int chunk = x * 32 + lane / 2;
        *reinterpret_cast<u32x2*>(codes + r * row_bytes + (chunk ^ r) * 16 + lane % 2 * 8) = Divisor(m).codes(*reinterpret_cast<const u32x4*>(raw + i * 1024));
        if (x == 0 && lane == 0) scales[r] = scale_of(m);
    }
    lds_reads_done();                                    // the last slot is free from here on
    __syncthreads();

    intx4 acc[kNBW][1];
#pragma unroll
    for (int j = 0; j < kNBW; ++j) acc[j][0] = intx4{0, 0, 0, 0};
    if (nbw > 0) {
        const int r = min(ln, a.n_rows - 1);
        const char* my_row = codes + r * row_bytes;
        const int rd_row = ln * 512;
        int t = 0;
        for (int s = 0; s < nslab; ++s) {
            const int first = slab_of<Int8Elements>(s, s0, nslab) * 32 + lg;
            intx4 hreg[T::KS];
#pragma unroll
            for (int ks = 0; ks < T::KS; ++ks) hreg[ks] = *reinterpret_cast<const intx4*>(my_row + ((first + ks * 4) ^ r) * 16);
#pragma unroll
            for (int j = 0; j < kNBW; ++j) {
                if (j < nbw) {
                    wait_loads<(T::AHEAD - 1) * T::NLD>();
                    request_next();
                    const char* tile = ring + (t & (T::SLOTS - 1)) * T::BYTES;
                    ++t;
#pragma unroll
                    for (int ks = 0; ks < T::KS; ++ks)
                        acc[j][0] = Int8Elements::mma(*reinterpret_cast<const intx4*>(tile + rd_row + (((ks * 4 + lg) ^ ln) * 16)), hreg[ks], acc[j][0]);
                    lds_reads_done();
                }
            }
        }
        wait_loads<0>();
    }
    finish<Int8Elements, 1>(a, scales, acc, nbw, v0, reinterpret_cast<float*>(smem + kWaves * kRing));
}

enum Kind { kNarrow, kWide, kSplitNarrow, kSplitWide };  // slabs of 256 bytes, of 512
template <int NR, class F>
hipError_t for_build(Kind kind, F f)
{
    if (kind == kSplitNarrow) return f(lm_head_split<256, NR>, lds_bytes());
    if (kind == kSplitWide) return f(lm_head_split<512, NR>, lds_bytes());
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
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(lm_head_own_codes), hipFuncAttributeMaxDynamicSharedMemorySize, OwnCodes::LDS);
    if (e != hipSuccess) return e;
    for (int nr = 1; nr <= 6; ++nr)
        for (Kind kind : {kNarrow, kWide, kSplitNarrow, kSplitWide}) {
            const hipError_t e = for_build(nr, kind, [](auto kernel, int lds) {
                return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
            });
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

hipError_t launch_lm_head_quant(const LmHeadLaunch& a, const QuantRowsLaunch& rows, hipStream_t stream)
{
    if (a.row_bytes % 256 != 0 || a.nb < 1 || a.nb > kNB) return hipErrorInvalidValue;
    const int nwg = (a.vocab + a.nb * 16 - 1) / (a.nb * 16);
    if (own_codes(a)) {
        static_assert(OwnCodes::LDS <= 160 * 1024, "LDS of a compute unit");
        hipLaunchKernelGGL(lm_head_own_codes, dim3(nwg), dim3(kWaves * 64), OwnCodes::LDS, stream, a, rows.x);
        return hipGetLastError();
    }
    const hipError_t e = launch_quant_rows(rows, stream);
    if (e != hipSuccess) return e;
    const bool narrow = a.row_bytes % 512 != 0, split = a.nb <= kSplitBlocks;
    return for_build((a.n_rows + 15) / 16, split ? (narrow ? kSplitNarrow : kSplitWide) : narrow ? kNarrow : kWide, [&](auto kernel, int lds) {
        hipLaunchKernelGGL(kernel, dim3(nwg), dim3(kWaves * 64), lds, stream, a);
        return hipGetLastError();
    });
}
