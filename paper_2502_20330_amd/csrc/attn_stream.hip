// Verification attention over a cache in 8 bits (gfx950), over the sequences' own tokens behind a shared prefix, and over a sliding window (there the tokens
// of each sequence, or of each tile of its rows, are divided by themselves: attn_stream_window).
//
// The mathematics is that of verify_attn.hip: softmax(scale <q, k>) v with a running maximum m and sum l per query row; partial
// results (m, l, O) of disjoint token ranges are joined as O = sum 2^(m_i - M) O_i, l likewise.
//
// What bounds it is the cache: 2 d + 2 bytes per token and kv head are read once for all R = (gamma + 1) G packed rows, against 4 R d
// multiplications on the matrix cores and R exponentials.  Hence:
//  * The batch is divided by tokens, not by sequences: one workgroup per compute unit and kv head share, whatever the lengths are.  Every
//    workgroup finds its share from ctx_lens by a wave scan; no length is needed on the host.
//  * A workgroup has eight waves, two per SIMD, so that one wave's exponentials and conversions run under the other's matrix
//    instructions.  Up to three blocks of 16 rows every wave streams token tiles of its own; from four blocks on, two teams of
//    waves share the tiles of four streams and each takes half of the rows (four waves, one per SIMD, where the cache is bf16).
//  * Tiles travel HBM -> LDS directly, two or more ahead of the mathematics, with an XOR swizzle on the 16-byte chunks.
//  * Codes become bf16 on the way from LDS to the matrix core (one instruction for two values, exact).  A key's scale rides on that
//    conversion: in the S^T = K Q^T form a lane holds one token's row.  A value's scale cannot (there a lane holds one column of eight
//    tokens) and is multiplied into the token's weight instead, in 32 bits, before the weight's own rounding to bf16.
//  * ds_read_b64_tr_b8 delivers V^T, eight tokens of one column, straight from LDS.
// Measured, 8 kv heads of 128 and 128K tokens (271 MB, 39 us at the rate of a pure read): 4 rows 46 us, 36 rows 53 to 59, 72 rows 70 to 75; eight sequences
// of 16K to 128K, 16-token pages, 36 rows (1291 MB, 186 us): 216 to 220.  Of the 55 us, 5 pass until the first tiles are there, 4.5 in the epilogue and 6.5
// between the kernel's end and the merge's; from 36 rows on the matrix and softmax work is as long as the reads.
#include "attn_exchange.h"
#include "attn_stream.h"
#include "attn_tile.h"

namespace {

// RB0: row blocks of 16 that a wave has, or team 0; RB1: those of team 1, 0 = there are no teams.
template <int D, bool QUANT, int RB0_, int RB1_>
struct Geo : TileGeo<D, QUANT, QUANT && D == 64 ? 4 : 2> {
    using Tile = TileGeo<D, QUANT, QUANT && D == 64 ? 4 : 2>;
    using Tile::SLOT, Tile::SC, Tile::TT, Tile::QROWB;
    static constexpr int RB0 = RB0_, RB1 = RB1_, RB = RB0 + RB1;
    static constexpr bool TEAMS = RB1 > 0;
    static constexpr int NP = QUANT && !TEAMS ? 8 : 4;            // token streams of a workgroup
    static constexpr int NW = TEAMS ? 2 * NP : NP;                // waves
    static constexpr int QUANTUM = NP * TT;                       // tokens of a workgroup's step
    static constexpr int S = 128 * 1024 / NP / (2 * SLOT);        // tiles of a ring: the loads in flight fill 128 KiB
    static constexpr int RING = S * (2 * SLOT + SC * 256);        // S tiles of K, of V, of scales
    static constexpr int QCPR = QROWB / 16, QRPI = 64 / QCPR;
    static constexpr int RP = RB * 16;
    static constexpr int NH = NP * RP * (D + 4) * 4 > 140 * 1024 ? 2 : 1;   // passes of the last exchange, D / NH columns each
    static constexpr int OROW = D / NH + 4;                       // padded row of the exchange (floats)
    static constexpr int TILES = NP * RING + RP * QROWB;
    static constexpr int MERGE = NP * RP * OROW * 4;
    static constexpr int ML = TILES > MERGE ? TILES : MERGE;      // where the waves' (m, l) lie
    static constexpr int TAKEN = ML + NW * (TEAMS ? (RB0 > RB1 ? RB0 : RB1) : RB0) * 16 * 8 + RP * 4;   // behind the rows' sums: a word for each stream
    static constexpr int LDS = TAKEN + (TEAMS ? NP * 4 : 0);
};

// Where packed row `row` of (sequence b, kv head h) goes.
__device__ __forceinline__ int64_t lse_index(const StreamLaunch& a, int b, int h, int row)
{
    return ((int64_t)b * a.Hq + h * a.G + row % a.G) * a.Qmax + row / a.G;
}
template <int D>
__device__ __forceinline__ int64_t out_index(const StreamLaunch& a, int b, int h, int row)
{
    return (((int64_t)b * a.Qmax + row / a.G) * a.Hq + h * a.G + row % a.G) * D;
}

// ---- one piece: tokens [c0, c1) of one (sequence, kv head)
struct Piece {
    RowAddr addr;
    char *kring, *vring, *sring, *qlds;
    int* taken;                                   // teams: the stream's word for take_not_finite
    uint32_t kring_lds, vring_lds, sring_lds;
    int b, h;
    int L, Q, R, c0, c1, nt, last_tok;            // nt: this stream's tiles (positions c0 + (part + it NP) TT ..; these are tokens, but for a window)
    int joint, gap, r0;                           // a window: of the rows' span; the first of the packed rows
    int first, last;                              // and their positions
    int lane, wave, part, team;
};

// ---- a window: the span (attn_tile.h) of a tile of packed rows takes the tokens' place
constexpr int kWindowStep = 32;
// Packed rows r0 .. r0 + RP - 1 of sequence b, of which `rows` exist.
struct WindowRows {
    int L, Q, r0, rows;
    int first, last;                              // the positions of those that do
    __device__ __forceinline__ WindowRows(const StreamLaunch& a, int b, int r0_) : L(seq_len(a, b)), Q(seq_queries(a, b)), r0(r0_)
    {
        rows = min(Q * a.G - r0, a.RP);
        first = L - Q + r0 / a.G;
        last = L - Q + (r0 + rows - 1) / a.G;
    }
    __device__ __forceinline__ bool attend() const { return rows > 0 && L > 0 && last >= 0; }
    __device__ __forceinline__ WindowSpan span(const StreamLaunch& a) const { return WindowSpan(first, last, a.window, a.sinks, kWindowStep); }
};
// Into how many shares a span is cut: `groups`, of a quantum at least.
__device__ __forceinline__ int window_shares(const StreamLaunch& a, int len) { return min(a.groups, (len + a.quantum - 1) / a.quantum); }
// The partials of (sequence b, kv head h, packed row `row`), RP slots apart.
__device__ __forceinline__ int64_t window_slot(const StreamLaunch& a, int b, int h, int row)
{
    return (((int64_t)h * a.B + b) * a.tiles + row / a.RP) * a.groups * a.RP + row % a.RP;
}
template <bool WINDOW>
__device__ __forceinline__ int tile_token(const Piece& w, int x) { return WINDOW && x >= w.joint ? x + w.gap : x; }

// Row blocks row0 / 16 .. of the workgroup, over this wave's stream.
template <class G, int RB, bool PAGED, bool WINDOW>
__device__ __forceinline__ void run_piece(const StreamLaunch& a, const Piece& w, char* smem, int row0, int64_t pbase)
{
    constexpr int MLS = (G::TEAMS && G::RB1 > G::RB0 ? G::RB1 : G::RB0) * 16;
    const int lane = w.lane, ln = lane & 15, lg = lane >> 4;
    auto tile_t0 = [&](int it) { return tile_token<WINDOW>(w, w.c0 + (w.part + it * G::NP) * G::TT); };

    bf16x8 qf[RB][G::KS];
    int lim[RB];                                         // last token that a row attends in this piece
    [[maybe_unused]] int before[RB];                     // last token ahead of a row's window
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = row0 + rb * 16 + ln;
        const bool real = row < w.R;
        const int place = WINDOW ? w.r0 + row : row;
        lim[rb] = min(real && !a.shared ? w.L - w.Q + place / a.G : w.L - 1, WINDOW ? w.last_tok : w.c1 - 1);
        before[rb] = WINDOW && real ? w.L - w.Q + place / a.G - a.window : -1;
#pragma unroll
        for (int ks = 0; ks < G::KS; ++ks) {
            const int chunk = G::QUANT ? (ks >> 1) * 8 + 2 * lg + (ks & 1) : ks * 4 + lg;
            u32x4 raw = *reinterpret_cast<const u32x4*>(w.qlds + row * G::QROWB + (chunk ^ k_swz<G::QROWB>(row)) * 16);
            if (!real) raw = u32x4{0, 0, 0, 0};
            qf[rb][ks] = __builtin_bit_cast(bf16x8, raw);
        }
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
    auto hidden = [&](int tok, int rb) { return tok > lim[rb] || (WINDOW && tok <= before[rb] && tok >= a.sinks); };
    const int first_masked_t0 = min(a.shared ? w.L : w.L - w.Q, w.c1) - (G::TT - 1);     // tiles from here on hold tokens that some row does not attend
    auto masked = [&](int t0) {
        return WINDOW ? window_masks(t0, G::TT, w.first, w.last, w.last_tok, a.window, a.sinks) : t0 >= first_masked_t0;
    };
    TilePages<G, PAGED> pages;
    bool taken = false;
    [[maybe_unused]] const uint32_t no_scales[G::TB] = {};

    int slot = 0;                                        // ring slot of tile it
    auto next = [](int s) { return s + 1 == G::S ? 0 : s + 1; };
    if constexpr (G::QUANT) {
        // A tile's codes of V are in registers before the softmax, so that the products with V wait for nothing and the tile's slots are free early.
        // Streams of their own: S tiles are under way, and the slot is filled again by the wave that has read it.
        // Two waves a stream: each issues half of a tile's loads (both the scales); at the meeting tile `it` is complete and everybody has read
        // tile it - 1, whose slot takes tile it + S - 1.
        int before_slot = G::S - 1;
        for (int it = 0; it < w.nt; ++it, before_slot = slot, slot = next(slot)) {
            char* kt = w.kring + slot * G::SLOT;
            char* vt = w.vring + slot * G::SLOT;
            const int t0 = tile_t0(it), fill = G::TEAMS ? before_slot : slot, t_fill = tile_t0(it + G::S - (G::TEAMS ? 1 : 0));
            constexpr int H = G::TEAMS ? G::NLD / 2 : G::NLD;
            auto refill = [&]() {
                load_scales<G, PAGED>(w.addr, pages, w.sring_lds + fill * 256, t_fill, w.last_tok, lane);
                load_tile<G, PAGED, false, H>(w.addr, pages, w.kring_lds + fill * G::SLOT, t_fill, w.last_tok, lane, w.team * H);
                load_tile<G, PAGED, true, H>(w.addr, pages, w.vring_lds + fill * G::SLOT, t_fill, w.last_tok, lane, w.team * H);
            };
            pages.find(w.addr, t_fill, w.last_tok);
            wait_loads<(G::S - (G::TEAMS ? 2 : 1)) * (2 * H + G::SC)>();
            if (G::TEAMS) {
                meet();
                refill();
            }
            if (masked(t0)) taken |= take_not_finite<G>(vt, lane);      // (of a team, whoever comes second finds zeros)
            RawTile<G> x;
            x.read_k(kt, w.sring + slot * 256, lane);
            in_order();
            floatx4 s[G::TB][RB];
            bf16x8 pb[G::TB / 2][RB];
            x.scores(s, qf);
            x.read_v(vt, lane);
            lds_reads_done();
            if (!G::TEAMS) refill();
            softmax_tile<G, RB>(st, s, pb, x.vs, t0, masked(t0), hidden, w.c1, c, lane);
            x.add_values(st, pb);
        }
    } else if constexpr (!G::TEAMS) {
        // oldest load first: K(it) V(it) K(it+1) V(it+1) ..
        for (int it = 0; it < w.nt; ++it, slot = next(slot)) {
            char* kt = w.kring + slot * G::SLOT;
            char* vt = w.vring + slot * G::SLOT;
            const int t0 = tile_t0(it), t_next = tile_t0(it + G::S);
            floatx4 s[G::TB][RB];
            bf16x8 pb[G::TB / 2][RB];

            pages.find(w.addr, t_next, w.last_tok);
            wait_loads<(2 * G::S - 1) * G::NLD>();              // K(it)
            score_tile<G, RB>(s, qf, kt, lane);
            lds_reads_done();
            load_tile<G, PAGED, false, G::NLD>(w.addr, pages, w.kring_lds + slot * G::SLOT, t_next, w.last_tok, lane, 0);

            softmax_tile<G, RB>(st, s, pb, no_scales, t0, masked(t0), hidden, w.c1, c, lane);

            wait_loads<(2 * G::S - 1) * G::NLD>();              // V(it)
            if (masked(t0)) taken |= take_not_finite<G>(vt, lane);
            pv_tile<G, RB>(st, pb, vt, lane);
            lds_reads_done();
            load_tile<G, PAGED, true, G::NLD>(w.addr, pages, w.vring_lds + slot * G::SLOT, t_next, w.last_tok, lane, 0);
        }
    } else {
        // Two waves share a stream; each issues half of a tile's loads.
        // Barrier A: K(it) is complete, and everybody has done with V(it-1), whose slot V(it+S-1) takes.
        // Barrier B: V(it) is complete, and everybody has done with K(it), whose slot K(it+S) takes.
        constexpr int H = G::NLD / 2, BEHIND = 2 * (G::S - 1) * H;
        TilePages<G, PAGED> vpages;
        vpages.find(w.addr, tile_t0(G::S - 1), w.last_tok);
        int before_slot = G::S - 1;                             // the slot of tile it - 1
        for (int it = 0; it < w.nt; ++it, before_slot = slot, slot = next(slot)) {
            char* kt = w.kring + slot * G::SLOT;
            char* vt = w.vring + slot * G::SLOT;
            const int t0 = tile_t0(it), t_next = tile_t0(it + G::S);
            floatx4 s[G::TB][RB];
            bf16x8 pb[G::TB / 2][RB];

            pages.find(w.addr, t_next, w.last_tok);
            wait_loads<BEHIND>();                               // own half of K(it)
            __syncthreads();                                    // A
            load_tile<G, PAGED, true, H>(w.addr, vpages, w.vring_lds + before_slot * G::SLOT, tile_t0(it + G::S - 1), w.last_tok, lane, w.team * H);
            score_tile<G, RB>(s, qf, kt, lane);
            softmax_tile<G, RB>(st, s, pb, no_scales, t0, masked(t0), hidden, w.c1, c, lane);

            wait_loads<BEHIND>();                               // own half of V(it)
            lds_reads_done();
            __syncthreads();                                    // B
            load_tile<G, PAGED, false, H>(w.addr, pages, w.kring_lds + slot * G::SLOT, t_next, w.last_tok, lane, w.team * H);
            if (masked(t0)) taken |= take_not_finite<G>(vt, lane);      // (whoever comes second finds zeros)
            pv_tile<G, RB>(st, pb, vt, lane);
            lds_reads_done();
            vpages = pages;
        }
    }
    wait_loads<0>();                                     // no load may land after the rings are used below
    if constexpr (G::TEAMS) {
        if (taken && lane == 0) *w.taken = 1;
        __syncthreads();
        taken = *w.taken != 0;
    }
    if (WINDOW && taken) {
#pragma unroll 1
        for (int it = 0; it < w.nt; ++it) {
            const int t0 = tile_t0(it);
            if (masked(t0)) add_not_finite_shown<G, RB, PAGED>(st, w.addr, t0, min(t0 + G::TT - 1, w.last_tok), hidden, lane);
        }
    } else if (taken) {
        const int it = (max(first_masked_t0 - tile_t0(0), 0) + G::QUANTUM - 1) / G::QUANTUM;
        add_not_finite<G, RB, PAGED>(st, w.addr, tile_t0(it), w.c1, G::QUANTUM, lim, lane);
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) st.l[rb] = sum_over_groups(st.l[rb]);

    // ---- join the streams, in a fixed order
    float* obuf = reinterpret_cast<float*>(smem);                              // [NP][RP][OROW]
    float* mlbuf = reinterpret_cast<float*>(smem + G::ML);                     // [NW][MLS][2]
    if (lg == 0) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            mlbuf[(w.wave * MLS + rb * 16 + ln) * 2 + 0] = st.m[rb];
            mlbuf[(w.wave * MLS + rb * 16 + ln) * 2 + 1] = st.l[rb];
        }
    }
    __syncthreads();                                     // all rings are dead from here on
    float own[RB];
    float* sums = mlbuf + G::NW * MLS * 2;               // [RP], direct: the rows' sums
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float mw[G::NP], mm = kNoMaximum, ll = 0.f;
#pragma unroll
        for (int p = 0; p < G::NP; ++p) {
            mw[p] = mlbuf[((w.team * G::NP + p) * MLS + rb * 16 + ln) * 2];
            mm = fmaxf(mm, mw[p]);
        }
#pragma unroll
        for (int p = 0; p < G::NP; ++p) ll += mlbuf[((w.team * G::NP + p) * MLS + rb * 16 + ln) * 2 + 1] * fast_exp2(mw[p] - mm);
        own[rb] = fast_exp2(st.m[rb] - mm);
        const int row = row0 + rb * 16 + ln;
        if (w.part == 0 && lg == 0 && row < w.R) {
            if (a.direct) {
                sums[row] = ll;
                if (a.lse_out) a.lse_out[lse_index(a, w.b, w.h, WINDOW ? w.r0 + row : row)] = (mm + log2f(ll)) * 0.6931471805599453f;
            } else {
                a.part_ml[(pbase + row) * 2 + 0] = mm;
                a.part_ml[(pbase + row) * 2 + 1] = ll;
            }
        }
    }
    constexpr int DH = G::D / G::NH;
#pragma unroll
    for (int half = 0; half < G::NH; ++half) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int x = 0; x < G::DB / G::NH; ++x)
                *reinterpret_cast<floatx4*>(obuf + (w.part * G::RP + row0 + rb * 16 + ln) * G::OROW + x * 16 + lg * 4) =
                    st.acc[half * (G::DB / G::NH) + x][rb] * own[rb];
        __syncthreads();
        for (int f = threadIdx.x; f < w.R * (DH / 4); f += G::NW * 64) {
            const int row = f / (DH / 4), x = f % (DH / 4) * 4;
            floatx4 sum = *reinterpret_cast<const floatx4*>(obuf + row * G::OROW + x);
#pragma unroll
            for (int p = 1; p < G::NP; ++p) sum += *reinterpret_cast<const floatx4*>(obuf + (p * G::RP + row) * G::OROW + x);
            if (a.direct) {
                const float l = sums[row];
                if (l != 0.f) sum /= l;
                const bf16x4 o = {(__bf16)sum[0], (__bf16)sum[1], (__bf16)sum[2], (__bf16)sum[3]};
                *reinterpret_cast<bf16x4*>(a.out + out_index<G::D>(a, w.b, w.h, WINDOW ? w.r0 + row : row) + half * DH + x) = o;
            } else {
                *reinterpret_cast<floatx4*>(a.part_o + (pbase + row) * G::D + half * DH + x) = sum;
            }
        }
        __syncthreads();                                 // before the buffer is written again, or becomes rings
    }
}

template <class G, bool PAGED, bool WINDOW>
__device__ __forceinline__ void stream_piece(const StreamLaunch& a, char* smem, int b, int h, int L, int c0, int c1, int64_t pbase, int r0)
{                                                        // r0: the first of the packed rows (of a shared prefix, there may be more than RP)
    Piece w;
    const int tid = opaque(threadIdx.x);
    w.lane = tid & 63;
    w.wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    w.part = w.wave % G::NP;
    w.team = w.wave / G::NP;
    w.b = b;
    w.h = h;
    w.L = L;
    w.Q = seq_queries(a, b);
    w.R = min(w.Q * a.G - r0, G::RP);
    w.c0 = c0;
    w.c1 = c1;
    const int ntile = (c1 - c0 + G::TT - 1) / G::TT;
    // The streams take the tiles in turn, so that what a workgroup reads at a time lies together.  (A contiguous range for each, beginning powers of two
    // apart: 128K tokens at 4 rows 48.4 us instead of 46.2, at 36 rows 61 instead of 59, at 72 rows 75 instead of 72.5.)
    // Teams meet at barriers, so there every stream runs as many tiles; those past the end are masked.
    w.nt = (ntile + G::NP - 1 - (G::TEAMS ? 0 : w.part)) / G::NP;
    if (WINDOW) {
        static_assert(!WINDOW || G::TT == kWindowStep, "");
        const WindowRows rows(a, b, r0);
        const WindowSpan span = rows.span(a);
        w.joint = span.joint;
        w.gap = span.gap;
        w.r0 = r0;
        w.first = rows.first;
        w.last = rows.last;
    }
    w.last_tok = tile_token<WINDOW>(w, c1 - 1);
    w.addr = make_row_addr<G, PAGED>(a.own, b, h);
    const int ring = w.part * G::RING;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    w.kring = smem + ring;
    w.vring = w.kring + G::S * G::SLOT;
    w.sring = w.kring + 2 * G::S * G::SLOT;
    w.kring_lds = lds + ring;
    w.vring_lds = w.kring_lds + G::S * G::SLOT;
    w.sring_lds = w.kring_lds + 2 * G::S * G::SLOT;
    w.qlds = smem + G::NP * G::RING;
    w.taken = reinterpret_cast<int*>(smem + G::TAKEN) + w.part;
    if (G::TEAMS && w.lane == 0) *w.taken = 0;

    // The Q block, ahead of the first tiles: complete as soon as only they are outstanding.  Rows past the real ones repeat one.
    {
        const int last_row = a.Qmax * a.G - 1;
        for (int e = w.wave; e < G::RP / G::QRPI; e += G::NW) {
            const int row = e * G::QRPI + w.lane / G::QCPR;
            const int rr = min(r0 + row, last_row);
            const int ch = (w.lane % G::QCPR) ^ k_swz<G::QROWB>(row);
            const uint32_t off = (uint32_t)(((((int64_t)b * a.Qmax + rr / a.G) * a.Hq + h * a.G + rr % a.G) * G::D) * 2) + ch * 16;
            dma16_keep(reinterpret_cast<const char*>(a.q), off, lds + G::NP * G::RING + e * 1024);
        }
    }
    auto tile_t0 = [&](int it) { return tile_token<WINDOW>(w, c0 + (w.part + it * G::NP) * G::TT); };
    TilePages<G, PAGED> pages;
    constexpr int H = G::TEAMS ? G::NLD / 2 : G::NLD;
    const int e0 = G::TEAMS ? w.team * H : 0;
    if (w.nt > 0) {
        // tiles 0 .. S-1; of teams, the last is left to the first steps (bf16: its V)
        constexpr int NK = G::S - (G::TEAMS && G::QUANT ? 1 : 0), NV = G::S - (G::TEAMS ? 1 : 0);
#pragma unroll
        for (int it = 0; it < NK; ++it) {
            const int t0 = tile_t0(it);
            pages.find(w.addr, t0, w.last_tok);
            load_scales<G, PAGED>(w.addr, pages, w.sring_lds + it * 256, t0, w.last_tok, w.lane);
            load_tile<G, PAGED, false, H>(w.addr, pages, w.kring_lds + it * G::SLOT, t0, w.last_tok, w.lane, e0);
            if (it < NV) load_tile<G, PAGED, true, H>(w.addr, pages, w.vring_lds + it * G::SLOT, t0, w.last_tok, w.lane, e0);
        }
        wait_loads<(NK + NV) * H + NK * G::SC>();
    } else {
        wait_loads<0>();
    }
    __syncthreads();                                     // the whole Q block is in LDS

    if constexpr (!G::TEAMS) {
        run_piece<G, G::RB0, PAGED, WINDOW>(a, w, smem, 0, pbase);
    } else if constexpr (G::RB0 == G::RB1) {
        run_piece<G, G::RB0, PAGED, WINDOW>(a, w, smem, w.team * G::RB0 * 16, pbase);
    } else {
        // the two arms run the same barriers
        if (w.team == 0) run_piece<G, G::RB0, PAGED, WINDOW>(a, w, smem, 0, pbase);
        else run_piece<G, G::RB1, PAGED, WINDOW>(a, w, smem, G::RB0 * 16, pbase);
    }
}

// Packed rows [from, to) of a sequence, which it does not have or which attend nothing: zeros (lse: 0, and -infinity for rows that it has).
template <class G>
__device__ __forceinline__ void write_missing_rows(const StreamLaunch& a, int b, int h, int from, int to)
{
    const int R = seq_queries(a, b) * a.G;
    for (int f = threadIdx.x; f < (to - from) * (G::D / 8); f += G::NW * 64)
        *reinterpret_cast<u32x4*>(a.out + out_index<G::D>(a, b, h, from + f / (G::D / 8)) + f % (G::D / 8) * 8) = u32x4{0, 0, 0, 0};
    if (a.lse_out)
        for (int row = from + threadIdx.x; row < to; row += G::NW * 64) a.lse_out[lse_index(a, b, h, row)] = row < R ? -INFINITY : 0.f;
}

// Grid: one workgroup per (kv head, share).  Partials: [kv head][g + b], which no two pieces of a head share.  Direct: per (kv head, sequence).
template <class G, bool PAGED>
__device__ __forceinline__ void stream_share(const StreamLaunch& a, char* smem, int g, int len, int rt = 0)
{                                                        // len: of sequence `lane`, 0 where there is none
    const int h = __builtin_amdgcn_readfirstlane(a.rot ? (blockIdx.x + g) % a.Hkv : blockIdx.x);     // (base addresses go through scalar registers)
    if (a.direct) {
        const int L = __builtin_amdgcn_readfirstlane(seq_len(a, g));
        write_missing_rows<G>(a, g, h, L > 0 ? seq_queries(a, g) * a.G : 0, a.Qmax * a.G);
        if (L > 0) stream_piece<G, PAGED, false>(a, smem, g, h, L, 0, L, 0, 0);
        return;
    }
    for_each_piece(a, g, threadIdx.x & 63, len, G::QUANTUM, [&](int b, int L, int c0, int c1) {
        stream_piece<G, PAGED, false>(a, smem, b, h, L, c0, c1, ((int64_t)(h * a.tiles + rt) * a.nslots + g + b) * G::RP, rt * G::RP);
        wait_loads<0>();                                 // the partial's stores are out of the load account
    });
}
__device__ __forceinline__ int first_len(const StreamLaunch& a)
{
    const int lane = threadIdx.x & 63;
    return !a.direct && lane < a.B ? seq_len(a, lane) : 0;
}
template <class G, bool PAGED>
__global__ void __launch_bounds__(G::NW * 64) attn_stream(StreamLaunch a)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    stream_share<G, PAGED>(a, smem, blockIdx.y, first_len(a));
}
// bf16, a window: one workgroup per (kv head, sequence, share, row tile).  What sequences have is alike, so each is cut by itself, and a workgroup need not
// look at the others.
template <class G, bool PAGED>
__global__ void __launch_bounds__(G::NW * 64) attn_stream_window(StreamLaunch a)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int y = blockIdx.y / a.tiles, r0 = __builtin_amdgcn_readfirstlane((blockIdx.y - y * a.tiles) * G::RP);
    const int b = __builtin_amdgcn_readfirstlane(y / a.groups), share = y - b * a.groups;
    const int h = __builtin_amdgcn_readfirstlane(a.rot ? (blockIdx.x + y) % a.Hkv : blockIdx.x);
    const WindowRows rows(a, b, r0);
    const int L = __builtin_amdgcn_readfirstlane(rows.L);
    if (a.direct) write_missing_rows<G>(a, b, h, rows.attend() ? r0 + rows.rows : r0, min(r0 + G::RP, a.Qmax * a.G));
    if (!rows.attend()) return;
    const int len = rows.span(a).len, quanta = (len + G::QUANTUM - 1) / G::QUANTUM, shares = window_shares(a, len);
    if (share >= shares) return;
    const int c0 = (int)((int64_t)quanta * share / shares) * G::QUANTUM;
    const int c1 = min((int)((int64_t)quanta * (share + 1) / shares) * G::QUANTUM, len);
    stream_piece<G, PAGED, true>(a, smem, b, h, L, c0, c1, window_slot(a, b, h, r0) + (int64_t)share * G::RP, r0);
}

// How a prefix and the sequences' own tokens divide the `units` workgroups of a kv head: by what there is to read, of the prefix once for each row tile.
// It goes by the lengths, which are device data, and by no bound of them, that a caller may set as far above them as a cache's capacity (4 sequences of
// 300 tokens in caches of 128K, 32K of prefix: 174 us by the bounds, 30 by the lengths; looking at all lengths first costs every call about 0.5 us).  A sequence costs its own part about as much as 512 tokens, besides
// those that it has (19 short ones beside 2000 tokens of prefix, 4 kv heads: 19 us, 40 without).
constexpr int kPieceTokens = 512;
// The most that the own part takes: the prefix has a workgroup for each row tile, beyond the units where the tiles are many.
__host__ __device__ constexpr int most_own_units(int units, int tiles)
{
    const int left = units - tiles, half = units / 2;
    return left > half ? left : half > 1 ? half : 1;
}
struct PairGroups { int own, prefix; };          // shares of a kv head
// quanta: the sum of the own tokens' seq_cost(), of n sequences that have any.
__device__ __forceinline__ PairGroups pair_groups(const StreamLaunch& own, const StreamLaunch& prefix, int quanta, int n, int prefix_len)
{
#pragma clang fp contract(off)
    // The merge must find what the shares were: the same operations on both sides, whose last bits do not matter.  In half quanta; a sequence's last one is half full.
    if (own.units == 0) return {own.groups, prefix.groups};
    const float mine = (float)(2 * quanta + n * (2 * kPieceTokens / own.quantum - 2 * kPieceQuanta - 1));
    const float other = (float)prefix.tiles * (float)prefix_len * __builtin_amdgcn_rcpf((float)(own.quantum / 2));
    int g = (int)((float)own.units * mine * __builtin_amdgcn_rcpf(fmaxf(mine + other, 1.f)));
    g = __builtin_amdgcn_readfirstlane(max(1, min(g, most_own_units(own.units, prefix.tiles))));
    const int left = max(own.units - g, 0), each = max(1, prefix.tiles == 1 ? left : (int)((unsigned)left / (unsigned)prefix.tiles));
    g = max(g, own.units - each * prefix.tiles);                 // what the row tiles leave over
    return {min(g, own.groups), min(each, prefix.groups)};
}
// bf16: two in one launch, the shares of a prefix (or none), then those of the sequences' own tokens; both paged or neither.
template <class G, bool PAGED>
__global__ void __launch_bounds__(G::NW * 64) attn_stream_pair(StreamLaunch own, StreamLaunch prefix)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int y = __builtin_amdgcn_readfirstlane(blockIdx.y);
    PairGroups groups{own.groups, prefix.groups};
    int len = first_len(own), P = 0;
    if (own.units) {
        P = seq_len(prefix, 0);
        int quanta = 0, n = 0;
        for (int b0 = 0, l = len; b0 < own.B; b0 += 64) {
            const int b = b0 + (threadIdx.x & 63);
            if (b0) l = b < own.B ? seq_len(own, b) : 0;
            quanta += __builtin_amdgcn_readlane(scan_costs(seq_cost(l, b, G::QUANTUM)), 63);
            n += __popcll(__ballot(l > 0));
        }
        groups = pair_groups(own, prefix, quanta, n, P);
    }
    const int shares = groups.prefix * prefix.tiles;
    const bool first = y < shares;
    StreamLaunch a = first ? prefix : own;
    a.groups = first ? groups.prefix : groups.own;
    if (first) len = (threadIdx.x & 63) == 0 ? P : 0;
    const int g = first ? y : y - shares;
    stream_share<G, PAGED>(a, smem, g / a.tiles, len, g % a.tiles);
}

// The partials of one row: `n` of them, from row slot `slot` on, RP slots apart.
struct Partials {
    int n = 0;
    int64_t slot = 0;
};
// Where a sequence stands among the batch's quanta.
struct Place {
    int before = 0, cost = 0, total = 0, n = 0;          // n: sequences that have tokens
};
__device__ __forceinline__ Place find_place(const StreamLaunch& a, int b, int lane, int len)
{                                                        // len: of sequence `lane`, 0 where there is none
    Place p;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        if (b0) len = b0 + lane < a.B ? seq_len(a, b0 + lane) : 0;
        const int mine = seq_cost(len, b0 + lane, a.quantum);
        const int end = p.total + scan_costs(mine);
        if (b >= b0 && b < b0 + 64) {
            p.cost = __builtin_amdgcn_readlane(mine, b - b0);
            p.before = __builtin_amdgcn_readlane(end, b - b0) - p.cost;
        }
        p.total = __builtin_amdgcn_readlane(end, 63);
        p.n += __popcll(__ballot(len > 0));
    }
    return p;
}
// The partials of packed row `row` of sequence b, head h, of `groups` shares.
__device__ __forceinline__ Partials find_partials(const StreamLaunch& a, const Place& at, int groups, int b, int h, int row)
{
    Partials p;
    if (at.cost > 0) {
        const Shares sh(at.total, groups);
        const int g0 = sh.owner(at.before + piece_cost(b)), g1 = sh.owner(at.before + at.cost - 1);
        p.n = g1 - g0 + 1;
        p.slot = ((int64_t)(h * a.tiles + row / a.RP) * a.nslots + g0 + b) * a.RP + row % a.RP;
    }
    return p;
}
// A block of up to kMergeBlock of them on its way: this thread's column of each, and (maximum, sum) of one.
struct PartialBlock {
    float o[kMergeBlock], m, l;
    template <int D>
    __device__ __forceinline__ void load(const StreamLaunch& a, int64_t slot, int n, int d)
    {
        const float* po = a.part_o + slot * D + d;
#pragma unroll
        for (int j = 0; j < kMergeBlock; ++j) o[j] = j < n ? po[(int64_t)j * a.RP * D] : 0.f;
        const int sl = d & (kMergeBlock - 1);
        m = -INFINITY;
        l = 0.f;
        if (sl < n) {
            const float* ml = a.part_ml + (slot + (int64_t)sl * a.RP) * 2;
            m = ml[0];
            l = ml[1];
        }
    }
    // Folds the first n into the row's state and this thread's column; the others may be anything.
    __device__ __forceinline__ void fold(int n, int d, RowMerge& r, float& num)
    {
        const bool there = (d & (kMergeBlock - 1)) < n;
        float resc;
        const float w = r.block(there ? m : -INFINITY, there ? l : 0.f, &resc);
        float acc0 = 0.f, acc1 = 0.f;
#pragma unroll
        for (int j = 0; j < kMergeBlock; j += 2) {
            acc0 = fmaf(lane_of(w, j), j < n ? o[j] : 0.f, acc0);
            acc1 = fmaf(lane_of(w, j + 1), j + 1 < n ? o[j + 1] : 0.f, acc1);
        }
        num = num * resc + (acc0 + acc1);
    }
};
template <int D>
__device__ __forceinline__ void fold_partials(const StreamLaunch& a, int64_t slot, int n, int d, RowMerge& r, float& num)
{
    for (int s0 = 0; s0 < n; s0 += kMergeBlock) {
        PartialBlock x;
        x.load<D>(a, slot + (int64_t)s0 * a.RP, n - s0, d);
        x.fold(n - s0, d, r, num);
    }
}
// Where a single sequence's begin (b = 0), whose first share is share 0 whatever its length.
__device__ __forceinline__ int64_t first_slot(const StreamLaunch& a, int h, int row)
{
    return (int64_t)(h * a.tiles + row / a.RP) * a.nslots * a.RP + row % a.RP;
}

// One workgroup of D threads per (sequence, kv head, packed row): out = sum 2^(m_s - M) O_s / sum 2^(m_s - M) l_s, over the row's partials of the
// prefix and of its own tokens.
template <int D, bool PREFIX>
__global__ void __launch_bounds__(D) attn_stream_merge(StreamLaunch a, StreamLaunch prefix)
{
    const int row = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    const int d = threadIdx.x;
    uint16_t* dst = a.out + out_index<D>(a, b, h, row) + d;
    if (row >= seq_queries(a, b) * a.G) {                 // query rows this sequence does not have
        *dst = 0;
        if (a.lse_out && d == 0) a.lse_out[lse_index(a, b, h, row)] = 0.f;
        return;
    }
    // All that can be asked for is asked for at once: the lengths, the first block of a single sequence (the prefix is one) before its length is known, the
    // other's as soon as the lengths are there.
    const int lane = d & 63;
    const int len = lane < a.B ? seq_len(a, lane) : 0, prefix_len = PREFIX ? seq_len(prefix, 0) : 0;
    const bool there = seq_len(a, b) > 0;                 // (a sequence without tokens has no rows, behind a prefix either)
    const int prefix_row = b * a.Qmax * a.G + row;
    PartialBlock x, y;
    const int64_t x_slot = PREFIX ? first_slot(prefix, h, prefix_row) : 0;
    if (PREFIX) x.load<D>(prefix, x_slot, prefix.nslots, d);
    if (a.B == 1) y.load<D>(a, first_slot(a, h, row), a.nslots, d);
    const Place at = find_place(a, b, lane, len);
    PairGroups groups{a.groups, 0};
    if (PREFIX) groups = pair_groups(a, prefix, at.total, at.n, prefix_len);
    const Partials own = find_partials(a, at, groups.own, b, h, row);
    if (a.B != 1) y.load<D>(a, own.slot, own.n, d);
    RowMerge r;
    float num = 0.f;
    if (PREFIX) {
        const int quanta = (prefix_len + prefix.quantum - 1) / prefix.quantum, n = there ? min(groups.prefix, quanta) : 0;   // a share each
        x.fold(n, d, r, num);
        fold_partials<D>(prefix, x_slot + (int64_t)kMergeBlock * prefix.RP, n - kMergeBlock, d, r, num);
    }
    y.fold(own.n, d, r, num);
    fold_partials<D>(a, own.slot + (int64_t)kMergeBlock * a.RP, own.n - kMergeBlock, d, r, num);
    const __bf16 o = (__bf16)(r.den == 0.f ? 0.f : num / r.den);
    *dst = __builtin_bit_cast(uint16_t, o);
    if (a.lse_out && d == 0) a.lse_out[lse_index(a, b, h, row)] = (r.M + log2f(r.den)) * 0.6931471805599453f;
}

// The same for a window's few rows, whose partials lie where they lie whatever the lengths are.
template <int D>
__global__ void __launch_bounds__(D) attn_window_rows_merge(StreamLaunch a, StreamLaunch)
{
    const int row = blockIdx.x, h = blockIdx.y, b = blockIdx.z, d = threadIdx.x;
    const int64_t slot = window_slot(a, b, h, row);
    PartialBlock y;
    y.load<D>(a, slot, a.groups, d);
    const WindowRows rows(a, b, row / a.RP * a.RP);
    const int n = rows.attend() ? window_shares(a, rows.span(a).len) : 0;
    const bool real = row < rows.Q * a.G;
    RowMerge r;
    float num = 0.f;
    y.fold(real ? n : 0, d, r, num);
    fold_partials<D>(a, slot + (int64_t)kMergeBlock * a.RP, (real ? n : 0) - kMergeBlock, d, r, num);
    const __bf16 o = (__bf16)(r.den == 0.f ? 0.f : num / r.den);
    a.out[out_index<D>(a, b, h, row) + d] = __builtin_bit_cast(uint16_t, o);
    if (a.lse_out && d == 0) a.lse_out[lse_index(a, b, h, row)] = real ? (n > 0 ? (r.M + log2f(r.den)) * 0.6931471805599453f : -INFINITY) : 0.f;
}

// Calls f(Geo, paged) for the kernel that a shape takes; row blocks 1..6.
template <int D, bool QUANT, class F>
hipError_t with_geo(int rb, F f)
{
    switch (rb) {
        case 1: return f(Geo<D, QUANT, 1, 0>());
        case 2: return f(Geo<D, QUANT, 2, 0>());
        case 3: return f(Geo<D, QUANT, 3, 0>());
        case 4: if constexpr (QUANT) return f(Geo<D, true, 2, 2>()); else return f(Geo<D, false, 4, 0>());
        case 5: return f(Geo<D, QUANT, 3, 2>());
        case 6: return f(Geo<D, QUANT, 3, 3>());
    }
    return hipErrorInvalidValue;
}
template <class F>
hipError_t with_geo(int D, bool quant, int rb, F f)
{
    if (D == 128) return quant ? with_geo<128, true>(rb, f) : with_geo<128, false>(rb, f);
    return quant ? with_geo<64, true>(rb, f) : with_geo<64, false>(rb, f);
}

}  // namespace

hipError_t configure_attn_stream()
{
    for (int D = 64; D <= 128; D += 64)
        for (int rb = 1; rb <= 6; ++rb)
            for (int quant = 0; quant < 2; ++quant) {
                const hipError_t e = with_geo(D, quant, rb, [](auto geo) {
                    using G = decltype(geo);
                    static_assert(G::LDS <= 160 * 1024, "LDS of a compute unit");
                    auto raise = [](auto fn) {
                        return hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
                    };
                    if constexpr (G::QUANT) {
                        const hipError_t e = raise(attn_stream<G, false>);
                        return e == hipSuccess ? raise(attn_stream<G, true>) : e;
                    } else {
                        hipError_t e = raise(attn_stream_pair<G, false>);
                        if (e == hipSuccess) e = raise(attn_stream_pair<G, true>);
                        if (e == hipSuccess) e = raise(attn_stream_window<G, false>);
                        return e == hipSuccess ? raise(attn_stream_window<G, true>) : e;
                    }
                });
                if (e != hipSuccess) return e;
            }
    return hipSuccess;
}

namespace {

// One workgroup for each sequence and kv head, which writes the result, spares a launch and the partials, and gives up sharing out the tokens.  Up to two
// quanta there is little to share (us a call, one sequence, 8 kv heads of 128, 4 and 36 rows: 512 tokens 8.4 and 12.3 instead of 11.1 and 14.0;
// 1024 tokens 10.8 and 16.6 instead of 11.0 and 14.4), and up to eight it pays where the sequences occupy at least half of the compute units anyhow, in one
// round (16 sequences, 20 rows: 512 tokens 11.4 instead of 18, 1024 14.3 instead of 20, 2048 19.7 instead of 24.5).
constexpr int kDirectQuanta = 2, kDirectBatchQuanta = 8;

void plan_shares(StreamLaunch& a, int rb, int groups)
{
    a.RP = rb * 16;
    a.tiles = 1;
    (void)with_geo(a.D, a.own.ks != nullptr, rb, [&](auto geo) {
        a.quantum = decltype(geo)::QUANTUM;
        return hipSuccess;
    });
    // no more shares than the longest possible batch has quanta
    const int64_t most = (int64_t)a.B * (((int64_t)a.max_ctx + a.quantum - 1) / a.quantum + kPieceQuanta);
    a.groups = groups < 1 ? 1 : groups;
    if (a.groups > most) a.groups = (int)most;
    a.nslots = a.groups + a.B - 1;
    // heads whose rows are contiguous are spread over the dies, heads inside a token's row run side by side
    a.rot = a.own.hstride > a.own.tstride && a.Hkv > 1;
}

}  // namespace

// A workgroup takes a compute unit's LDS.
void plan_attn_stream(StreamLaunch& a, int n_cu)
{
    plan_shares(a, (a.Qmax * a.G + 15) / 16, n_cu / a.Hkv);
    const int64_t units = (int64_t)a.B * a.Hkv;
    const int quanta = 2 * units >= n_cu && units <= n_cu ? kDirectBatchQuanta : kDirectQuanta;
    a.direct = a.max_ctx <= quanta * a.quantum;
}

// Row tiles and shares of a sequence's window: those that a simple account finds the fastest.  A workgroup takes a fixed time, of which most is code that each of
// them runs for the first time, more of it the more blocks of rows it has, and its tokens times a rate, that of its arithmetic or what the memory gives to so many workgroups;
// the chip takes as many rounds as it is filled by; more than one share cost a second launch, and the partials of many row tiles their way.  (us a call, 32 / 8 heads of
// 128: 64 sequences of 4 rows, 2000 tokens: 84 in one share; of 36 rows, 500 tokens: 43 in one share; one sequence of 36 rows, 120 tokens: 10.4 in tiles of 16 rows, 14.3
// in one of 48; of 72 rows, 2000 tokens: 13.6 and 17.5; eight of 36 rows, 8000 tokens: 55 in one tile, 61 in two; one of 400 rows, 1000 tokens, tiles of 16, 32, 48, 96: 16,
// 20, 23, 31; of 1600 rows 58, 39, 44, 31.  The division of the whole batch's tokens into equal shares, which unequal lengths ask for, takes 90 and 65 in the first two.)
float plan_attn_stream_window(StreamLaunch& a, int n_cu)
{
    const int64_t rows = (int64_t)a.Qmax * a.G;
    float best = INFINITY;
    int best_rb = 0, best_groups = 1;
    for (int rb = rows <= kStreamRows ? (int)(rows + 15) / 16 : kStreamRows / 16; rb >= 1; rb = rb > 3 ? 3 : rb - 1) {
        plan_shares(a, rb, 1);
        const int64_t tiles = (rows + rb * 16 - 1) / (rb * 16), units = a.B * tiles * a.Hkv;
        if (a.B * tiles > 65535) continue;                                 // (a grid's second dimension; B alone is at most that)
        const int64_t positions = tiles > 1 ? (rb * 16 - 1) / a.G + 2 : a.Qmax;
        const int64_t span = (int64_t)a.sinks + a.window + positions + 2 * kWindowStep, tokens = span < a.max_ctx ? span : a.max_ctx;
        const int64_t most = (tokens + a.quantum - 1) / a.quantum;
        const float fixed = rb == 1 ? (tiles > 1 ? 9.f : 7.f) : rb == 2 ? 12.f : rb == 3 ? 14.f : 17.f, a_token = 0.0055f + 0.0012f * rb;    // us
        const float bytes = 4.f * a.D * (0.35f + 0.65f / tiles);           // of which row tiles beside one another share some
        for (int64_t k = 0; k <= 4; ++k) {                                 // shares that fill k rounds
            int64_t groups = k * n_cu / units;
            groups = groups > most ? most : groups < 1 ? 1 : groups;
            const int64_t grid = units * groups, busy = grid < n_cu ? grid : n_cu, rounds = (grid + n_cu - 1) / n_cu;
            const float from_memory = bytes * (float)busy / 6.8e6f, rate = from_memory > a_token ? from_memory : a_token;
            const float partials = groups == 1 ? 0.f : 2.5f + (tiles > 1 ? (float)grid * (rb * 16 * (a.D + 2) * 8) * 0.25e-6f : 0.f);
            const float time = (float)rounds * (fixed + rate * (float)tokens / (float)groups) + partials;
            if (time >= best) continue;
            best = time;
            best_rb = rb;
            best_groups = (int)groups;
        }
    }
    if (best_rb == 0) return best;
    plan_shares(a, best_rb, 1);
    a.tiles = (int)((rows + best_rb * 16 - 1) / (best_rb * 16));
    a.groups = best_groups;
    a.nslots = a.B * a.groups;
    a.direct = a.groups == 1;
    return best;
}

void plan_attn_stream_pair(StreamLaunch& own, StreamLaunch& prefix, int n_cu)
{
    const int rows = prefix.Qmax * prefix.G, own_rows = own.Qmax * own.G, each = n_cu > own.Hkv ? n_cu / own.Hkv : 1;
    const int rb = rows <= kStreamRows ? (rows + 15) / 16 : own_rows <= 48 ? 3 : (own_rows + 15) / 16;
    const int tiles = (rows + rb * 16 - 1) / (rb * 16);
    plan_shares(own, rb, each);
    plan_shares(prefix, rb, each / tiles);
    prefix.tiles = tiles;
    own.units = !prefix.own.page_table == !own.own.page_table ? each : 0;
}

size_t attn_stream_workspace_bytes(const StreamLaunch& a)
{
    if (a.direct) return 256;
    const size_t rows = (size_t)a.Hkv * a.tiles * a.nslots * a.RP;
    return (rows * a.D * 4 + 255) / 256 * 256 + (rows * 8 + 255) / 256 * 256;
}

void bind_attn_stream(StreamLaunch& a, void* workspace)
{
    const size_t rows = (size_t)a.Hkv * a.tiles * a.nslots * a.RP;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + (rows * a.D * 4 + 255) / 256 * 256);
}

hipError_t launch_attn_stream(const StreamLaunch& a, hipStream_t stream)
{
    return with_geo(a.D, a.own.ks != nullptr, a.RP / 16, [&](auto geo) {
        using G = decltype(geo);
        const dim3 grid(a.Hkv, a.window ? a.B * a.groups * a.tiles : a.direct ? a.B : a.groups * a.tiles), block(G::NW * 64);
        if constexpr (G::QUANT) {
            auto fn = a.own.page_table ? attn_stream<G, true> : attn_stream<G, false>;
            hipLaunchKernelGGL(fn, grid, block, G::LDS, stream, a);
        } else if (a.window) {
            auto fn = a.own.page_table ? attn_stream_window<G, true> : attn_stream_window<G, false>;
            hipLaunchKernelGGL(fn, grid, block, G::LDS, stream, a);
        } else {
            auto fn = a.own.page_table ? attn_stream_pair<G, true> : attn_stream_pair<G, false>;
            hipLaunchKernelGGL(fn, grid, block, G::LDS, stream, a, StreamLaunch{});
        }
        return hipGetLastError();
    });
}

hipError_t launch_attn_stream_pair(const StreamLaunch& own, const StreamLaunch& prefix, hipStream_t stream)
{
    if (own.units == 0) {                                               // (rare: a prefix of its own beside paged sequences)
        const hipError_t e = launch_attn_stream(prefix, stream);
        return e == hipSuccess ? launch_attn_stream(own, stream) : e;
    }
    return with_geo(own.D, false, own.RP / 16, [&](auto geo) {
        using G = decltype(geo);
        if constexpr (!G::QUANT) {
            auto fn = own.own.page_table ? attn_stream_pair<G, true> : attn_stream_pair<G, false>;
            const int with_tiles = most_own_units(own.units, prefix.tiles) + prefix.tiles;
            const int shares = with_tiles > own.units ? with_tiles : own.units;
            hipLaunchKernelGGL(fn, dim3(own.Hkv, shares), dim3(G::NW * 64), G::LDS, stream, own, prefix);
            return hipGetLastError();
        }
        return hipErrorInvalidValue;
    });
}

hipError_t launch_attn_stream_merge(const StreamLaunch& a, const StreamLaunch& prefix, hipStream_t stream)
{
    auto fn = prefix.part_o ? (a.D == 128 ? attn_stream_merge<128, true> : attn_stream_merge<64, true>)
              : a.window    ? (a.D == 128 ? attn_window_rows_merge<128> : attn_window_rows_merge<64>)
                            : (a.D == 128 ? attn_stream_merge<128, false> : attn_stream_merge<64, false>);
    hipLaunchKernelGGL(fn, dim3(a.Qmax * a.G, a.Hkv, a.B), dim3(a.D), 0, stream, a, prefix);
    return hipGetLastError();
}
