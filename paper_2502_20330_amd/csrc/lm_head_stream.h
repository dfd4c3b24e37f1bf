// Streaming product of a tall matrix with a few rows, used by lm_head.hip (bf16) and lm_head_quant.hip (8-bit integers): the two differ in the
// matrix instruction and in how a sum becomes a logit; a tile is the same bytes.
#pragma once
#include "rapid_internal.h"

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));

namespace {

constexpr int kWaves = 4;
constexpr int kNB = 32;                      // 16-row vocabulary blocks per workgroup
constexpr int kRing = 32768;                 // LDS ring per wave
// Tile geometry for slabs of SB bytes of a row (512, or 256 for rows that are a multiple of 256 bytes but not of 512).
template <int SB>
struct Tile {
    static constexpr int BYTES = 16 * SB;              // 8 KiB / 4 KiB
    static constexpr int NLD = BYTES / 1024;           // 1 KiB load instructions per tile
    static constexpr int RPI = 1024 / SB;              // rows moved by one instruction
    static constexpr int CPR = SB / 16;                // 16-byte chunks per row
    static constexpr int KS = SB / 64;                 // MFMA k-steps per tile
    static constexpr int SLOTS = kRing / BYTES;        // 4 / 8
    static constexpr int AHEAD = SLOTS - 1;            // tiles requested ahead of the math
};
constexpr float kLog2e = 1.4426950408889634f;

// The elements: a lane gives 16 bytes of a row to a matrix instruction, whatever they are.
struct Bf16Elements {
    typedef bf16x8 Op;
    typedef floatx4 Acc;
    static constexpr bool INT8 = false;
    static __device__ __forceinline__ Acc mma(Op w, Op h, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, h, c, 0, 0, 0); }
};
struct Int8Elements {
    typedef intx4 Op;
    typedef intx4 Acc;
    static constexpr bool INT8 = true;
    static __device__ __forceinline__ Acc mma(Op w, Op h, Acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, h, c, 0, 0, 0); }
};

// Where the slabs of a row lie.  Slabs of 256 bytes: one run.  Of 512: two, the second kHalf bytes behind the first: in
// rows that are a multiple of 4 KiB (TWO), the runs of eight slabs fill either half of 4 KiB in turn; else they adjoin (a pitch that is no
// multiple of 4 KiB spreads the rows of a tile by itself, and whole lines of 512 bytes are 1 % faster: 5 rows of
// 2304 x 100000 69.9 us against 71.1; for powers of two see lm_head.hip).  A template parameter: told apart
// at every load it made heads of a few thousand entries 3 to 10 % slower.
template <int SB, bool TWO>
struct Slabs {
    static_assert(SB == 512 || !TWO, "");
    static constexpr uint32_t kHalf = TWO ? 2048u : 256u;
    static __device__ __forceinline__ int64_t byte(int s) { return TWO ? (int64_t)(s >> 3) * 4096 + (s & 7) * 256 : (int64_t)s * SB; }
};

__device__ __forceinline__ void dma16(const char* base, uint32_t byte_off, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1 nt"
                 :
                 : "v"(byte_off), "s"(base), "s"(lds_addr)
                 : "memory", "m0");
}
// h is re-read by every workgroup: no streaming hint, it should stay in cache
__device__ __forceinline__ void dma16_keep(const char* base, uint32_t byte_off, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(byte_off), "s"(base), "s"(lds_addr)
                 : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void lds_reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

constexpr int kNBW = kNB / kWaves;                      // vocabulary blocks per wave at most
constexpr int lds_bytes() { return kWaves * kRing + kWaves * 96 * 2 * 4; }   // rings + (max, sum) of 96 rows per wave

// First vocabulary row of a block as loaded: a block that reaches past the vocabulary reads the last 16 rows instead (the
// epilogue drops the rows that belong to the block before).
__device__ __forceinline__ int loaded_row0(const LmHeadLaunch& a, int nominal) { return min(nominal, a.vocab - 16); }

// acc[jj][rb]: lane (ln, lg) holds, for row rb*16 + ln of h, the four vocabulary
// entries loaded_row0 + lg*4 .. +3 of block jj.  Logits go out from the registers; the chunk statistics
// are formed per wave (own maximum) and combined over the four waves by the first threads; red: [kWaves][NR * 16][2].
// A NaN among the logits: NAN_SUM makes the chunk's sum NaN, the maximum is that of the numbers; else the wave that holds it has no part in the sum.
template <int NR, bool NAN_SUM>
__device__ __forceinline__ void epilogue(const LmHeadLaunch& a, const floatx4 (&acc)[kNBW][NR], int nbw, int v0, float* red)
{
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ln = lane & 15, lg = lane >> 4;
    const float c = a.inv_T * kLog2e;
    const bool vec_ok = (a.ldz & 3) == 0 && (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0;
#pragma unroll
    for (int rb = 0; rb < NR; ++rb) {
        const int hrow = rb * 16 + ln;
        const bool row_ok = hrow < a.n_rows;
        float m = -INFINITY;
#pragma unroll
        for (int jj = 0; jj < kNBW; ++jj) {
            const int nominal = v0 + (jj * kWaves + wave) * 16;
            if (jj < nbw && nominal < a.vocab && row_ok) {
                const int vi = loaded_row0(a, nominal) + lg * 4;
                float* dst = a.logits + (int64_t)hrow * a.ldz + vi;
                if (vec_ok && vi >= nominal && (vi & 3) == 0) {
                    *reinterpret_cast<floatx4*>(dst) = acc[jj][rb];
#pragma unroll
                    for (int i = 0; i < 4; ++i) m = fmaxf(m, acc[jj][rb][i]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (vi + i >= nominal) { dst[i] = acc[jj][rb][i]; m = fmaxf(m, acc[jj][rb][i]); }
                }
            }
        }
        if (!a.stats) continue;                                // uniform
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        float sum = 0.f;
        const float base = NAN_SUM && !(m > -INFINITY) ? 0.f : m;           // (entries of -infinity alone: a sum of 0, and of NaN where there is one)
        if (NAN_SUM || m > -INFINITY) {
#pragma unroll
            for (int jj = 0; jj < kNBW; ++jj) {
                const int nominal = v0 + (jj * kWaves + wave) * 16;
                if (jj < nbw && nominal < a.vocab && row_ok) {
                    const int vi = loaded_row0(a, nominal) + lg * 4;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (vi + i >= nominal) sum += __builtin_amdgcn_exp2f((acc[jj][rb][i] - base) * c);
                }
            }
        }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (lg == 0) {
            red[((wave * NR * 16) + hrow) * 2 + 0] = m;
            red[((wave * NR * 16) + hrow) * 2 + 1] = sum;
        }
    }
    if (!a.stats) return;
    __syncthreads();
    if (tid < a.n_rows) {
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, red[((w * NR * 16) + tid) * 2]);
        float S = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float mw = red[((w * NR * 16) + tid) * 2], sw = red[((w * NR * 16) + tid) * 2 + 1];
            if (NAN_SUM ? sw != 0.f : sw > 0.f) S += sw * __builtin_amdgcn_exp2f((mw - M) * c);
        }
        a.stats[((int64_t)tid * gridDim.x + blockIdx.x) * 2 + 0] = M;
        a.stats[((int64_t)tid * gridDim.x + blockIdx.x) * 2 + 1] = S;
    }
}

// A sum of 8-bit products becomes a logit: times the row's scale, times the vocabulary entry's.  The sum itself is exact, and three roundings of
// half a step, 2^-24 of the value, follow: of a sum beyond 2^24, and of either product.
template <class E, int NR>
__device__ __forceinline__ void finish(const LmHeadLaunch& a, const float* h_scales, const typename E::Acc (&acc)[kNBW][NR], int nbw, int v0, float* red)
{
    if constexpr (!E::INT8) {
        epilogue<NR, false>(a, acc, nbw, v0, red);
    } else {
        const int lane = threadIdx.x & 63, ln = lane & 15, lg = lane >> 4;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        float hs[NR];
#pragma unroll
        for (int rb = 0; rb < NR; ++rb) hs[rb] = h_scales[min(rb * 16 + ln, a.n_rows - 1)];
        floatx4 z[kNBW][NR];
#pragma unroll
        for (int jj = 0; jj < kNBW; ++jj) {
            const int nominal = v0 + (jj * kWaves + wave) * 16;
            floatx4 ws = {0.f, 0.f, 0.f, 0.f};
            if (jj < nbw && nominal < a.vocab) {
#pragma unroll
                for (int i = 0; i < 4; ++i) ws[i] = a.w_scales[loaded_row0(a, nominal) + lg * 4 + i];
            }
#pragma unroll
            for (int rb = 0; rb < NR; ++rb)
#pragma unroll
                for (int i = 0; i < 4; ++i) z[jj][rb][i] = (float)acc[jj][rb][i] * hs[rb] * ws[i];
        }
        epilogue<NR, true>(a, z, nbw, v0, red);
    }
}

// The order of the slabs.  Sums of bf16 products depend on it and take them all from the first on; of integers they do not, and the workgroups begin at
// different ones, so that they ask different memory channels at a time: 4096 x 128256, one row 109 -> 81 us, 72 rows 121 -> 95, 16 rows of 4096 x 32000 32 -> 27; 2048
// to 8192 otherwise alike (6144 x 64000 64 -> 63, 8192 x 128256 156, 5120 x 64000 62, 3584 x 152064 91).
template <class E>
__device__ __forceinline__ int first_slab(int nslab)
{
    return E::INT8 ? (int)(blockIdx.x / 8 % (unsigned)nslab) : 0;
}
template <class E>
__device__ __forceinline__ int slab_of(int s, int s0, int nslab)
{
    if (!E::INT8) return s;
    return s + s0 >= nslab ? s + s0 - nslab : s + s0;
}

template <class E, int SB, int NR, bool TWO>
__global__ void __launch_bounds__(kWaves * 64) lm_head_stream(LmHeadLaunch a)
{
    using T = Tile<SB>;
    using At = Slabs<SB, TWO>;
    using Op = typename E::Op;
    using Acc = typename E::Acc;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ln = lane & 15, lg = lane >> 4;
    const int nb = a.nb;                                 // 16-row vocabulary blocks per workgroup (<= 32)
    const int nbw = (nb + kWaves - 1 - wave) / kWaves;   // blocks of this wave: wave, wave + 4, ...
    const int v0 = blockIdx.x * nb * 16;
    const uint32_t row_bytes = (uint32_t)a.row_bytes;
    const int nslab = a.row_bytes / SB;
    const int s0 = first_slab<E>(nslab);
    char* ring = smem + wave * kRing;
    const uint32_t ring_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + wave * kRing;

    // Per-lane byte offsets of the loads of a tile, relative to the tile's first row and the slab:
    // instruction e moves RPI consecutive rows; lane i writes LDS bytes [16 i, 16 i + 16) of that
    // 1 KiB and fetches the chunk the swizzle assigns there (chunks 16..31: the slab's second run).
    uint32_t woff[T::NLD], coff[T::NLD];
    int rrow[T::NLD];
#pragma unroll
    for (int e = 0; e < T::NLD; ++e) {
        rrow[e] = T::RPI * e + lane / T::CPR;
        coff[e] = (uint32_t)((lane % 16) ^ (rrow[e] & 15)) * 16u + (uint32_t)((lane % T::CPR) / 16) * At::kHalf;
        woff[e] = (uint32_t)rrow[e] * row_bytes + coff[e];
    }
    auto block_row0 = [&](int jj) { return loaded_row0(a, v0 + (jj * kWaves + wave) * 16); };

    // tile j of slab s: j = 0..NR-1 the row blocks of the h slab, j = NR.. the wave's W blocks
    auto issue = [&](int s, int j, int slot) {
        const int64_t kbyte = At::byte(slab_of<E>(s, s0, nslab));
        const uint32_t dst = ring_lds + slot * T::BYTES;
        if (j < NR) {
            const char* base = reinterpret_cast<const char*>(a.h) + kbyte;
#pragma unroll
            for (int e = 0; e < T::NLD; ++e)
                dma16_keep(base, (uint32_t)min(j * 16 + rrow[e], a.n_rows - 1) * row_bytes + coff[e], dst + e * 1024);
            return;
        }
        const char* base = reinterpret_cast<const char*>(a.w) + (int64_t)block_row0(j - NR) * row_bytes + kbyte;
#pragma unroll
        for (int e = 0; e < T::NLD; ++e) dma16(base, woff[e], dst + e * 1024);
    };

    Acc acc[kNBW][NR];
#pragma unroll
    for (int j = 0; j < kNBW; ++j)
#pragma unroll
        for (int rb = 0; rb < NR; ++rb) acc[j][rb] = Acc{0, 0, 0, 0};

    if (nbw > 0) {                                       // (a wave without blocks: ranges of fewer than four blocks)
        int ps = 0, pj = 0, pt = 0;                      // next tile to request: slab, index, linear number
        auto request_next = [&]() {
            const int sl = pt & (T::SLOTS - 1);
            if (ps < nslab) issue(ps, pj, sl);
            else issue(nslab - 1, 0, sl);                // past the end: a cached h tile keeps the count uniform
            ++pt;
            if (++pj >= NR + nbw) { pj = 0; ++ps; }
        };
#pragma unroll
        for (int j = 0; j < T::AHEAD; ++j) request_next();

        Op hreg[NR][T::KS];
        const int rd_row = ln * SB;
        const int rd_swz = ln & 15;
        int t = 0;
        for (int s = 0; s < nslab; ++s) {
#pragma unroll
            for (int j = 0; j < NR + kNBW; ++j) {
                if (j < NR + nbw) {
                    wait_loads<(T::AHEAD - 1) * T::NLD>();     // tile (s, j) has landed
                    request_next();
                    const char* tile = ring + (t & (T::SLOTS - 1)) * T::BYTES;
                    ++t;
                    if (j < NR) {
#pragma unroll
                        for (int ks = 0; ks < T::KS; ++ks)
                            hreg[j < NR ? j : 0][ks] = *reinterpret_cast<const Op*>(tile + rd_row + (((ks * 4 + lg) ^ rd_swz) * 16));
                    } else {
#pragma unroll
                        for (int ks = 0; ks < T::KS; ++ks) {
                            Op wa = *reinterpret_cast<const Op*>(tile + rd_row + (((ks * 4 + lg) ^ rd_swz) * 16));
#pragma unroll
                            for (int rb = 0; rb < NR; ++rb)
                                acc[j >= NR ? j - NR : 0][rb] =
                                    E::mma(wa, hreg[rb][ks], acc[j >= NR ? j - NR : 0][rb]);
                        }
                    }
                    lds_reads_done();
                }
            }
        }
        wait_loads<0>();
    }

    finish<E, NR>(a, a.h_scales, acc, nbw, v0, reinterpret_cast<float*>(smem + kWaves * kRing));
}

// ---------------------------------------------------------------- many rows: one copy of h per workgroup
// From four row blocks on.  The four waves load a slab of h together (256-wide, NR tiles) and all read it into their registers; two
// barriers a slab, eight tiles of W apart, and the loads of the next slab of h go out right behind them.  What the
// LDS has left is the rings of W, in units of half a tile (one of the slab's two runs: 16 rows x 256 bytes), five or six units
// ahead of the math.  Against h through every wave's own ring: 72 rows of 4096 x 128256 179 -> 171 us, 96 rows 190 -> 175, 72
// rows of 2048 x 128256 100 -> 95; 60 rows 171 -> 168; 40 rows 162 -> 164, so three row blocks stay there.  Two or four
// passes over the hidden dimension, so that the logits of the first leave under the loads of the second: 184 and 224 us.
template <int NR>
struct Shared {
    static constexpr int HBYTES = NR * 16 * 512;                              // a slab of h
    static constexpr int RED = kWaves * NR * 16 * 2 * 4;
    static constexpr int UNIT = 16 * 256;                                     // half a tile of W
    static constexpr int ULD = UNIT / 1024;                                   // loads per unit
    static constexpr int HLD = NR * 8 / kWaves;                               // loads of a wave per slab of h
    static constexpr int SLOTS = (160 * 1024 - HBYTES - RED) / kWaves / UNIT;
    static constexpr int AHEAD = SLOTS - 1;
    static constexpr int LDS = HBYTES + RED + kWaves * SLOTS * UNIT;
};

template <class E, int NR, bool TWO>
__global__ void __launch_bounds__(kWaves * 64) lm_head_shared(LmHeadLaunch a)
{
    using S = Shared<NR>;
    using At = Slabs<512, TWO>;
    using Op = typename E::Op;
    using Acc = typename E::Acc;
    constexpr int KH = 4;                                // k-steps of a unit
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ln = lane & 15, lg = lane >> 4;
    const int nb = a.nb;                                 // 16-row vocabulary blocks per workgroup (<= 32)
    const int nbw = (nb + kWaves - 1 - wave) / kWaves;   // blocks of this wave: wave, wave + 4, ...
    const int v0 = blockIdx.x * nb * 16;
    const uint32_t row_bytes = (uint32_t)a.row_bytes;
    const int nslab = a.row_bytes / 512;
    const int s0 = first_slab<E>(nslab);
    char* hbuf = smem;
    char* ring = smem + S::HBYTES + wave * (S::SLOTS * S::UNIT);
    const uint32_t h_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const uint32_t ring_lds = h_lds + S::HBYTES + wave * (S::SLOTS * S::UNIT);

    // Loads of a unit: instruction e moves rows 4 e .. 4 e + 3; the swizzle as above, within 16 chunks.
    uint32_t woff[S::ULD];
#pragma unroll
    for (int e = 0; e < S::ULD; ++e) {
        const int row = 4 * e + lane / 16;
        woff[e] = (uint32_t)row * row_bytes + (uint32_t)((lane & 15) ^ (row & 15)) * 16u;
    }
    // This wave's share of slab s of h: 1 KiB (two rows) of every 4.
    auto issue_h = [&](int s) {
        const char* base = reinterpret_cast<const char*>(a.h) + At::byte(slab_of<E>(s, s0, nslab));
#pragma unroll
        for (int i = 0; i < S::HLD; ++i) {
            const int e = i * kWaves + wave, row = 2 * e + lane / 32;
            const uint32_t c = (uint32_t)((lane & 15) ^ (row & 15)) * 16u + (uint32_t)((lane & 31) / 16) * At::kHalf;
            dma16_keep(base, (uint32_t)min(row, a.n_rows - 1) * row_bytes + c, h_lds + e * 1024);
        }
    };
    // The next unit to request: half pq of slab ps of block pj; past the end any valid one keeps the count uniform.
    int ps = 0, pj = 0, pq = 0, pslot = 0;
    auto request_next = [&]() {
        const char* base = reinterpret_cast<const char*>(a.w) +
                           (int64_t)loaded_row0(a, v0 + (pj * kWaves + wave) * 16) * row_bytes + At::byte(slab_of<E>(min(ps, nslab - 1), s0, nslab)) + (pq ? At::kHalf : 0u);
#pragma unroll
        for (int e = 0; e < S::ULD; ++e) dma16(base, woff[e], ring_lds + pslot * S::UNIT + e * 1024);
        if (++pslot == S::SLOTS) pslot = 0;
        pq ^= 1;
        if (pq == 0 && ++pj >= nbw) { pj = 0; ++ps; }
    };

    Acc acc[kNBW][NR];
#pragma unroll
    for (int j = 0; j < kNBW; ++j)
#pragma unroll
        for (int rb = 0; rb < NR; ++rb) acc[j][rb] = Acc{0, 0, 0, 0};

    // (a wave without blocks, in ranges of fewer than four, only loads its share of h and meets the barriers)
    issue_h(0);
    if (nbw > 0)
#pragma unroll
        for (int j = 0; j < S::AHEAD; ++j) request_next();
    int slot = 0;
    for (int s = 0; s < nslab; ++s) {
        // The own share of h has landed: AHEAD units at least were requested after it, unless the wave has too few blocks.
        if (s == 0 ? nbw > 0 : 2 * nbw >= S::AHEAD) wait_loads<S::AHEAD * S::ULD>();
        else wait_loads<0>();
        __syncthreads();                                 // everybody's has
        Op hreg[NR][2 * KH];
#pragma unroll
        for (int rb = 0; rb < NR; ++rb)
#pragma unroll
            for (int ks = 0; ks < 2 * KH; ++ks)
                hreg[rb][ks] = *reinterpret_cast<const Op*>(hbuf + rb * 8192 + ln * 512 + (((ks * 4 + lg) ^ ln) * 16));
        lds_reads_done();
        __syncthreads();                                 // everybody has read it
        issue_h(min(s + 1, nslab - 1));                  // (the last one again: the count stays uniform)
#pragma unroll
        for (int j = 0; j < kNBW; ++j)
            if (j < nbw) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    // the slab's first AHEAD units were requested before the loads of h just issued, so those are behind them too
                    if (2 * j + q < S::AHEAD) wait_loads<(S::AHEAD - 1) * S::ULD + S::HLD>();
                    else wait_loads<(S::AHEAD - 1) * S::ULD>();
                    request_next();
                    const char* unit = ring + slot * S::UNIT;
                    if (++slot == S::SLOTS) slot = 0;
#pragma unroll
                    for (int ks = 0; ks < KH; ++ks) {
                        const Op wa = *reinterpret_cast<const Op*>(unit + ln * 256 + (((ks * 4 + lg) ^ ln) * 16));
#pragma unroll
                        for (int rb = 0; rb < NR; ++rb)
                            acc[j][rb] = E::mma(wa, hreg[rb][q * KH + ks], acc[j][rb]);
                    }
                    lds_reads_done();
                }
            }
    }
    wait_loads<0>();
    finish<E, NR>(a, a.h_scales, acc, nbw, v0, reinterpret_cast<float*>(smem + S::HBYTES + kWaves * S::SLOTS * S::UNIT));
}

}  // namespace
