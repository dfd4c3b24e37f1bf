// Attention of a whole batch's rows over one shared prefix (gfx950).
//
// All rows of the batch, R = B (gamma_max + 1) G per kv head, attend the same P tokens, without a mask: the prefix is one "sequence"
// with R rows.  Reading it costs 4 d bytes per token and kv head, computing 4 R d multiply-adds and R exponentials, so that from about a hundred rows on the
// matrix cores and the exponentials bound it and no longer the memory.  Up to 96 rows, and where all of it is little work, the streaming kernel (attn_stream.hip) does it; this one takes more.
// The rows are packed as q holds them: those past a sequence's drafts, and the last tile's padding, are computed like the others and read by nobody.
//  * A workgroup has eight waves, T of which share a stream of token tiles (8 / T streams) and hold one to three blocks of 16 rows each, 128 to 384 rows
//    together.  Tiles go HBM -> LDS once a workgroup; S of them lie in a ring, and the waves meet every S / 4 tiles: then the next ones have landed
//    and the slots of the ones before are free.
//  * Rows beyond that go to other workgroups, which read the same tokens at about the same time on the same die (blockIdx modulo 8), so that its L2
//    serves all but one of them.
// Measured (8 kv heads of 128): 131000 tokens, 320 rows 187 to 207 us (830 to 920 TFLOP/s of what is computed; 228 of the rows exist in that case: 590 to
// 650), 32K tokens, 288 rows 58.  By counters the matrix cores are busy in 43 % of the compute units' cycles there, 1284 of about 3000 a tile of 32 tokens; 304 vector
// instructions of a SIMD's two waves a tile, exponentials and conversions, run beside them in part only.
#include "attn_rows.h"

namespace {

// Tokens [c0, c1) for the rows of tile `rt`, of which this wave has RB blocks from team_row on; the partial goes to the rows from pbase on.
template <class G, int RB, bool PAGED>
__device__ __forceinline__ void prefix_piece(const StreamLaunch& a, char* smem, int h, int rt, int c0, int c1, int64_t pbase, int team_row)
{
    const int tid = opaque(threadIdx.x), lane = tid & 63, ln = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int part = wave / G::T, team = wave % G::T;
    const int rows = a.Qmax * a.G - rt * G::RP;          // of this tile, if there are so many

    const int ntile = (c1 - c0 + G::TT - 1) / G::TT;
    const int nt = (ntile + G::NP - 1) / G::NP;          // tiles of a stream; all run as many, those past the end are masked
    const int first = part * nt;
    const int last_tok = min(c1, c0 + (first + nt) * G::TT) - 1;
    auto tile_t0 = [&](int it) { return c0 + (first + it) * G::TT; };
    const RowAddr addr = make_row_addr<G, PAGED>(a.own, 0, h);
    char* kring = smem + part * G::RING;
    char* vring = kring + G::S * G::SLOT;
    const uint32_t kring_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + part * G::RING;
    const uint32_t vring_lds = kring_lds + G::S * G::SLOT;
    int* taken_word = reinterpret_cast<int*>(smem + G::TAKEN) + part;
    if (lane == 0) *taken_word = 0;

    // Q^T as the B operand, straight to registers: each wave has rows of its own
    bf16x8 qf[RB][G::KS];
    int lim[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = team_row + rb * 16 + ln, r = rt * G::RP + min(row, rows - 1);
        lim[rb] = c1 - 1;
        const u32x4* src = reinterpret_cast<const u32x4*>(a.q + ((int64_t)(r / a.G) * a.Hq + h * a.G + r % a.G) * G::D);
#pragma unroll
        for (int ks = 0; ks < G::KS; ++ks) {
            u32x4 raw = src[ks * 4 + lg];
            if (row >= rows) raw = u32x4{0, 0, 0, 0};
            qf[rb][ks] = __builtin_bit_cast(bf16x8, raw);
        }
    }
    TilePages<G, PAGED> pages;
#pragma unroll
    for (int it = 0; it < G::S - G::NB; ++it) {
        pages.find(addr, tile_t0(it), last_tok);
        load_both<G, PAGED>(addr, pages, kring_lds + it * G::SLOT, vring_lds + it * G::SLOT, tile_t0(it), last_tok, lane, team);
    }

    WaveState<G, RB> st;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        st.m[rb] = kNoMaximum;
        st.l[rb] = 0.f;
#pragma unroll
        for (int db = 0; db < G::DB; ++db) st.acc[db][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const float c = a.scale_log2e;
    auto hidden = [&](int tok, int rb) { return tok > lim[rb]; };
    const int first_masked_t0 = c1 - (G::TT - 1);        // tiles from here on reach past the end
    bool taken = false;
    const uint32_t no_scales[G::TB] = {};

    // The waves run freely between meetings, NB tiles apart, so that of the two waves of a SIMD one is at its matrix products while the other is at its
    // softmax.  (Meetings at every tile hold all waves to the same step: the products of the two then wait for one another, and so do
    // the softmaxes.  Handing the two halves of a step to and fro between them was no better: the halves are not equally long.)
    // Before the first K of a block of NB tiles every wave has its part of the block, and nobody needs the block before any more: its slots take the tiles
    // three blocks on.
    int fill = G::S - G::NB, fill_slot = G::S - G::NB;   // the tile that is loaded next, and its slot
    auto next_block = [&]() {
        wait_loads<(G::S - 2 * G::NB) * 2 * G::H>();
        lds_reads_done();
        meet();
#pragma unroll
        for (int x = 0; x < G::NB; ++x) {
            pages.find(addr, tile_t0(fill), last_tok);
            load_both<G, PAGED>(addr, pages, kring_lds + fill_slot * G::SLOT, vring_lds + fill_slot * G::SLOT, tile_t0(fill), last_tok, lane, team);
            ++fill;
            fill_slot = fill_slot + 1 == G::S ? 0 : fill_slot + 1;
        }
    };
    // Products of step `it`: V(it-1) and K(it); the last step's K is behind the end, and its scores are not used.  Their operands come from LDS ahead of them:
    // half of V's before the step, the rest and K's under the products with V.
    floatx4 s[G::TB][RB];
    bf16x8 pb[G::TB / 2][RB], v0[kHalfV<G>];             // weights of a tile, the first half of its V
    char *kt = kring, *vt = vring;
    next_block();
    {
        bf16x8 k0[G::TB / 2][G::KS], k1[G::TB / 2][G::KS];
        read_k<G>(k0, kt, 0, lane);
        read_k<G>(k1, kt, 1, lane);
        mma_k<G, RB>(s, k0, qf, 0);
        mma_k<G, RB>(s, k1, qf, 1);
    }
    for (int it = 0; it < nt; ++it) {
        const int t0 = tile_t0(it);
        softmax_tile<G, RB>(st, s, pb, no_scales, t0, t0 >= first_masked_t0, hidden, c1, c, lane);
        if (t0 >= first_masked_t0) taken |= take_not_finite<G>(vt, lane);      // (whoever comes second finds zeros)
        in_order();
        bf16x8 v1[kHalfV<G>], k0[G::TB / 2][G::KS], k1[G::TB / 2][G::KS];
        read_v<G>(v0, vt, 0, lane);
        read_v<G>(v1, vt, 1, lane);
        in_order();
        mma_v<G, RB>(st, v0, pb, 0);
        in_order();
        if ((it + 1) % G::NB == 0) next_block();
        const bool wrap = kt == kring + (G::S - 1) * G::SLOT;
        kt = wrap ? kring : kt + G::SLOT;
        read_k<G>(k0, kt, 0, lane);
        in_order();
        mma_v<G, RB>(st, v1, pb, 1);
        read_k<G>(k1, kt, 1, lane);
        in_order();
        mma_k<G, RB>(s, k0, qf, 0);
        mma_k<G, RB>(s, k1, qf, 1);
        in_order();
        vt = wrap ? vring : vt + G::SLOT;
    }
    wait_loads<0>();                                     // no load may land after the rings are used below
    if (taken && lane == 0) *taken_word = 1;
    __syncthreads();                                     // all rings are dead from here on
    if (*taken_word != 0) {
        const int it = max(0, (max(first_masked_t0 - c0, 0) + G::TT - 1) / G::TT - first);
        add_not_finite<G, RB, PAGED>(st, addr, tile_t0(it), min(c1, tile_t0(nt)), G::TT, lim, lane);
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) st.l[rb] = sum_over_groups(st.l[rb]);

    const int row0 = team_row + ln;
    if constexpr (G::NP == 1) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int row = row0 + rb * 16;
            if (row >= rows) continue;
            if (lg == 0) {
                a.part_ml[(pbase + row) * 2 + 0] = st.m[rb];
                a.part_ml[(pbase + row) * 2 + 1] = st.l[rb];
            }
#pragma unroll
            for (int db = 0; db < G::DB; ++db)
                *reinterpret_cast<floatx4*>(a.part_o + (pbase + row) * G::D + db * 16 + lg * 4) = st.acc[db][rb];
        }
        __syncthreads();                                 // everybody has read the words in LDS
        return;
    }
    // ---- join the streams, in a fixed order
    float* obuf = reinterpret_cast<float*>(smem);                              // [NP][RP][OROW]
    float* mlbuf = reinterpret_cast<float*>(smem + G::ML);                     // [NP][RP][2]
    if (lg == 0) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            mlbuf[(part * G::RP + row0 + rb * 16) * 2 + 0] = st.m[rb];
            mlbuf[(part * G::RP + row0 + rb * 16) * 2 + 1] = st.l[rb];
        }
    }
    __syncthreads();
    float own[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = row0 + rb * 16;
        float mw[G::NP], mm = kNoMaximum, ll = 0.f;
#pragma unroll
        for (int p = 0; p < G::NP; ++p) {
            mw[p] = mlbuf[(p * G::RP + row) * 2];
            mm = fmaxf(mm, mw[p]);
        }
#pragma unroll
        for (int p = 0; p < G::NP; ++p) ll += mlbuf[(p * G::RP + row) * 2 + 1] * fast_exp2(mw[p] - mm);
        own[rb] = fast_exp2(st.m[rb] - mm);
        if (part == 0 && lg == 0 && row < rows) {
            a.part_ml[(pbase + row) * 2 + 0] = mm;
            a.part_ml[(pbase + row) * 2 + 1] = ll;
        }
    }
    constexpr int DH = G::D / G::NH;
#pragma unroll
    for (int half = 0; half < G::NH; ++half) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int x = 0; x < G::DB / G::NH; ++x)
                *reinterpret_cast<floatx4*>(obuf + (part * G::RP + row0 + rb * 16) * G::OROW + x * 16 + lg * 4) =
                    st.acc[half * (G::DB / G::NH) + x][rb] * own[rb];
        __syncthreads();
        for (int f = tid; f < min(rows, G::RP) * (DH / 4); f += G::NW * 64) {
            const int row = f / (DH / 4), x = f % (DH / 4) * 4;
            floatx4 sum = *reinterpret_cast<const floatx4*>(obuf + row * G::OROW + x);
#pragma unroll
            for (int p = 1; p < G::NP; ++p) sum += *reinterpret_cast<const floatx4*>(obuf + (p * G::RP + row) * G::OROW + x);
            *reinterpret_cast<floatx4*>(a.part_o + (pbase + row) * G::D + half * DH + x) = sum;
        }
        __syncthreads();
    }
}

// One workgroup per (share, kv head, row tile); the row tiles of a (share, kv head) are eight apart, on one die.
template <class G, bool PAGED>
__global__ void __launch_bounds__(G::NW * 64) attn_prefix(StreamLaunch a)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int units = a.groups * a.Hkv, whole = units / 8 * 8, idx = blockIdx.x;
    int u, rt;
    if (idx < whole * a.tiles) {
        u = idx / (8 * a.tiles) * 8 + idx % 8;
        rt = idx / 8 % a.tiles;
    } else {
        u = whole + (idx - whole * a.tiles) % (units - whole);
        rt = (idx - whole * a.tiles) / (units - whole);
    }
    u = __builtin_amdgcn_readfirstlane(u);
    rt = __builtin_amdgcn_readfirstlane(rt);
    const int g = u / a.Hkv, h = __builtin_amdgcn_readfirstlane(u % a.Hkv);
    const int lane = threadIdx.x & 63;
    for_each_piece(a, __builtin_amdgcn_readfirstlane(g), lane, lane == 0 ? seq_len(a, 0) : 0, G::QUANTUM, [&](int, int, int c0, int c1) {
        const int64_t pbase = ((int64_t)(h * a.tiles + rt) * a.nslots + g) * G::RP;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        // (the two arms run the same barriers)
        if (G::RB0 == G::RB1 || wave < 4) prefix_piece<G, G::RB0, PAGED>(a, smem, h, rt, c0, c1, pbase, wave % G::T * G::RB0 * 16);
        else prefix_piece<G, G::RB1, PAGED>(a, smem, h, rt, c0, c1, pbase, G::RB0 * 64 + (wave - 4) * G::RB1 * 16);
        wait_loads<0>();
    });
}

}  // namespace

hipError_t configure_attn_prefix()
{
    for (int D = 64; D <= 128; D += 64)
        for (int rows : kRowTiles) {
            const hipError_t e = with_rows(D, rows, [](auto geo) {
                using G = decltype(geo);
                static_assert(G::LDS <= 160 * 1024, "LDS of a compute unit");
                const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(attn_prefix<G, false>),
                                                         hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
                if (e != hipSuccess) return e;
                return hipFuncSetAttribute(reinterpret_cast<const void*>(attn_prefix<G, true>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
            });
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

// Rows a workgroup: the choice that pads least, the larger of equals (fewer readers of the prefix).
void plan_attn_prefix(StreamLaunch& a, int n_cu)
{
    const int R = a.Qmax * a.G;
    int64_t least = -1;
    for (int rows : kRowTiles) {
        const int64_t padded = ((int64_t)R + rows - 1) / rows * rows;
        if (least >= 0 && padded >= least) continue;
        least = padded;
        a.RP = rows;
    }
    a.tiles = (R + a.RP - 1) / a.RP;
    (void)with_rows(a.D, a.RP, [&](auto geo) {
        a.quantum = decltype(geo)::QUANTUM;
        return hipSuccess;
    });
    const int64_t units = (int64_t)a.Hkv * a.tiles;
    a.groups = n_cu > units ? (int)(n_cu / units) : 1;
    const int64_t most = ((int64_t)a.max_ctx + a.quantum - 1) / a.quantum;
    if (a.groups > most) a.groups = (int)most;
    // A share more divides the tiles further, and is one more partial of every row to write and read: the sum of the two is least where
    // groups^2 is about 2 max_ctx / units (4 kv heads, 266 rows, 2000 tokens: 64 shares 35 us, 31 of them 31; more tokens want them all).
    while (a.groups > 1 && (int64_t)a.groups * a.groups * units > (int64_t)2 * a.max_ctx) --a.groups;
    a.nslots = a.groups;
    a.rot = 0;
}

hipError_t launch_attn_prefix(const StreamLaunch& a, hipStream_t stream)
{
    return with_rows(a.D, a.RP, [&](auto geo) {
        using G = decltype(geo);
        auto fn = a.own.page_table ? attn_prefix<G, true> : attn_prefix<G, false>;
        hipLaunchKernelGGL(fn, dim3(a.groups * a.Hkv * a.tiles), dim3(G::NW * 64), G::LDS, stream, a);
        return hipGetLastError();
    });
}
