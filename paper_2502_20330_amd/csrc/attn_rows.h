// Tiles of tokens against many query rows (attn_prefix.hip, attn_window.hip): how a workgroup's eight waves hold rows and share tiles, and the products
// with their operands read ahead.
#pragma once
#include "attn_tile.h"

namespace {

// T: waves that share a stream; RB0, RB1: row blocks of the first and of the last four waves (equal where T = 4).
template <int D, int T_, int RB0_, int RB1_>
struct RowsGeo : TileGeo<D, false, D == 64 ? 4 : 2> {
    using Tile = TileGeo<D, false, D == 64 ? 4 : 2>;
    using Tile::SLOT, Tile::TT, Tile::NLD;
    static constexpr int T = T_, RB0 = RB0_, RB1 = RB1_;
    static constexpr int NW = 8, NP = NW / T;                     // waves, token streams
    static constexpr int H = NLD / T;                             // loads of a tile of K or V that a wave issues
    static constexpr int QUANTUM = NP * TT;
    static constexpr int S = 128 * 1024 / NP / (2 * SLOT);        // tiles of a ring
    static constexpr int RING = S * 2 * SLOT;
    static constexpr int NB = S / 4;                              // tiles from one meeting of the waves to the next
    static constexpr int RP = (T == 8 ? RB0 + RB1 : RB0) * 64;    // rows of a workgroup
    static constexpr int NH = NP * RP * (D + 4) * 4 > 140 * 1024 ? 2 : 1;   // passes of the last exchange, D / NH columns each
    static constexpr int OROW = D / NH + 4;
    static constexpr int MERGE = NP > 1 ? NP * RP * OROW * 4 : 0;
    static constexpr int ML = NP * RING > MERGE ? NP * RING : MERGE;
    static constexpr int TAKEN = ML + NP * RP * 8;                // a word for each stream
    static constexpr int LDS = TAKEN + NP * 4;
};

// Loads of tile part `team` of K and V.
template <class G, bool PAGED, bool KEEP = false>
__device__ __forceinline__ void load_both(const RowAddr& ra, const TilePages<G, PAGED>& pages, uint32_t kslot, uint32_t vslot, int t0, int last_tok,
                                          int lane, int team)
{
    load_tile<G, PAGED, false, G::H, KEEP>(ra, pages, kslot, t0, last_tok, lane, team * G::H);
    load_tile<G, PAGED, true, G::H, KEEP>(ra, pages, vslot, t0, last_tok, lane, team * G::H);
}

// The operands of a tile's two products, from LDS to registers: half `x` of V^T's blocks, and half `x` of K's.
template <class G>
constexpr int kHalfV = G::TB / 2 * G::DB / 2;
template <class G>
__device__ __forceinline__ void read_v(bf16x8 (&vf)[kHalfV<G>], char* vt, int x, int lane)
{
    const int ln = lane & 15, lg = lane >> 4;
#pragma unroll
    for (int i = 0; i < kHalfV<G>; ++i) {
        const int kk = (x * kHalfV<G> + i) / G::DB, db = (x * kHalfV<G> + i) % G::DB;
        s16x4 half[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = kk * 32 + h * 16 + lg * 4 + (ln >> 2);
            const int c = (db * 2) ^ v_swz<false, G::ROWB>(row);
            half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (s16x4 __attribute__((address_space(3)))*)(vt + row * G::ROWB + c * 16 + (ln & 3) * 8));
        }
        const s16x8 both = __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
        vf[i] = __builtin_bit_cast(bf16x8, both);
    }
}
template <class G>
__device__ __forceinline__ void read_k(bf16x8 (&kf)[G::TB / 2][G::KS], const char* kt, int x, int lane)
{
#pragma unroll
    for (int i = 0; i < G::TB / 2; ++i) {
        const int row = (x * (G::TB / 2) + i) * 16 + (lane & 15);
#pragma unroll
        for (int ks = 0; ks < G::KS; ++ks)
            kf[i][ks] = *reinterpret_cast<const bf16x8*>(kt + row * G::ROWB + ((ks * 4 + (lane >> 4)) ^ k_swz<G::ROWB>(row)) * 16);
    }
}
// Half `x` of V^T P^T, of K Q^T.
template <class G, int RB>
__device__ __forceinline__ void mma_v(WaveState<G, RB>& st, const bf16x8 (&vf)[kHalfV<G>], const bf16x8 (&pb)[G::TB / 2][RB], int x)
{
#pragma unroll
    for (int i = 0; i < kHalfV<G>; ++i) {
        const int kk = (x * kHalfV<G> + i) / G::DB, db = (x * kHalfV<G> + i) % G::DB;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
            st.acc[db][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i], pb[kk][rb], st.acc[db][rb], 0, 0, 0);
    }
}
template <class G, int RB>
__device__ __forceinline__ void mma_k(floatx4 (&s)[G::TB][RB], const bf16x8 (&kf)[G::TB / 2][G::KS], const bf16x8 (&qf)[RB][G::KS], int x)
{
#pragma unroll
    for (int i = 0; i < G::TB / 2; ++i) {
        const int tb = x * (G::TB / 2) + i;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) s[tb][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < G::KS; ++ks)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
                s[tb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[i][ks], qf[rb][ks], s[tb][rb], 0, 0, 0);
    }
}

// Calls f(RowsGeo) for the kernel of `rows` rows a workgroup.
constexpr int kRowTiles[] = {384, 320, 256, 192, 128};
template <int D, class F>
hipError_t with_rows(int rows, F f)
{
    switch (rows) {
        case 128: return f(RowsGeo<D, 4, 2, 2>());
        case 192: return f(RowsGeo<D, 4, 3, 3>());
        case 256: return f(RowsGeo<D, 8, 2, 2>());
        case 320: return f(RowsGeo<D, 8, 3, 2>());
        case 384: return f(RowsGeo<D, 8, 3, 3>());
    }
    return hipErrorInvalidValue;
}
template <class F>
hipError_t with_rows(int D, int rows, F f) { return D == 128 ? with_rows<128>(rows, f) : with_rows<64>(rows, f); }

}  // namespace
