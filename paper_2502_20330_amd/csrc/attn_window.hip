// Attention with a sliding window and sinks for many query rows: prompts, and pieces of prompts behind what is cached already (gfx950).
//
// A row at position p attends the tokens of (p - window, p] and the first `sinks` ones.  The rows of a (sequence, kv head), position by position with the
// G heads of a position side by side, are cut into tiles of 128 to 384; a tile's tokens are those that any of its rows attends, two runs that are taken for
// one (WindowSpan in attn_tile.h), and only tiles of tokens at the runs' ends need a mask.  So a tile of RP rows computes RP (window + sinks + RP / G)
// scores where RP (window + sinks) count.
// It takes 4 d multiply-adds and an exponential a score: matrix cores and exponentials bound it.  Waves, ring and schedule are those of
// attn_prefix.hip: eight waves hold the rows, the tokens go HBM -> LDS once a workgroup, and a row tile's neighbours, which read nearly the same
// tokens, follow it on the same die, whose L2 serves them: with the hint that a tile is read once, which serves the other kernels, 384 rows of 32K positions took
// 2272 us instead of 1949.
// Measured (32K positions, 32 / 8 heads of 128, a window of 4096 and 64 sinks, 2.09 TFLOP of scores that count): 1950 to 2030 us from card to card, 1030 to 1073 TFLOP/s, where a large
// product of the library reaches 1295.  By counters the clock is held at 2.0 GHz, the matrix cores are busy in 44 % of the cycles, LDS in 15 %, 88 % of the L2's requests hit.  What the chip
// may draw bounds it as much as anything: with 256 rows the same loop without softmax and loads takes 1520 us, without loads 1850, and a schedule that
// interleaves products and exponentials of neighbouring tiles in each wave (their issue then overlaps by the listing) 2120 like this one.
#include "attn_rows.h"

namespace {

// Row tile rt of (sequence b, kv head h).
struct RowTile {
    int b, h, r0, rows, Q, L;                            // packed rows r0 .. r0 + rows - 1 exist
    int first, last;                                     // their positions
};

// Positions [c0, c1) of the span, for this wave's RB blocks of rows from team_row on.
template <class G, int RB, bool PAGED>
__device__ __forceinline__ void window_piece(const StreamLaunch& a, char* smem, const RowTile& w, const WindowSpan& span, int c0, int c1, int64_t pbase,
                                             int team_row)
{
    const int tid = opaque(threadIdx.x), lane = tid & 63, ln = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int part = wave / G::T, team = wave % G::T;

    const int ntile = (c1 - c0 + G::TT - 1) / G::TT;
    const int nt = (ntile + G::NP - 1) / G::NP;          // tiles of a stream; all run as many, those past the end are masked
    const int begin = c0 + part * nt * G::TT;
    const int last_tok = span.token(min(c1, begin + nt * G::TT) - 1);
    auto tile_t0 = [&](int it) { return span.token(begin + it * G::TT); };
    const RowAddr addr = make_row_addr<G, PAGED>(a.own, w.b, w.h);
    char* kring = smem + part * G::RING;
    char* vring = kring + G::S * G::SLOT;
    const uint32_t kring_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + part * G::RING;
    const uint32_t vring_lds = kring_lds + G::S * G::SLOT;
    int* taken_word = reinterpret_cast<int*>(smem + G::TAKEN) + part;
    if (lane == 0) *taken_word = 0;

    // Q^T as the B operand, straight to registers: each wave has rows of its own
    bf16x8 qf[RB][G::KS];
    int pos[RB];                                         // of this lane's rows
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = team_row + rb * 16 + ln, r = w.r0 + min(row, w.rows - 1);
        pos[rb] = w.L - w.Q + r / a.G;
        const u32x4* src = reinterpret_cast<const u32x4*>(a.q + (((int64_t)w.b * a.Qmax + r / a.G) * a.Hq + w.h * a.G + r % a.G) * G::D);
#pragma unroll
        for (int ks = 0; ks < G::KS; ++ks) {
            u32x4 raw = src[ks * 4 + lg];
            if (row >= w.rows) raw = u32x4{0, 0, 0, 0};
            qf[rb][ks] = __builtin_bit_cast(bf16x8, raw);
        }
    }
    TilePages<G, PAGED> pages;
#pragma unroll
    for (int it = 0; it < G::S - G::NB; ++it) {
        pages.find(addr, tile_t0(it), last_tok);
        load_both<G, PAGED, true>(addr, pages, kring_lds + it * G::SLOT, vring_lds + it * G::SLOT, tile_t0(it), last_tok, lane, team);
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
    auto hidden = [&](int tok, int rb) { return tok > min(pos[rb], last_tok) || (tok <= pos[rb] - a.window && tok >= a.sinks); };
    auto masked = [&](int t0) { return window_masks(t0, G::TT, w.first, w.last, last_tok, a.window, a.sinks); };
    bool taken = false;
    const uint32_t no_scales[G::TB] = {};

    // (meetings and the order of a step: attn_prefix.hip)
    int fill = G::S - G::NB, fill_slot = G::S - G::NB;   // the tile that is loaded next, and its slot
    auto next_block = [&]() {
        wait_loads<(G::S - 2 * G::NB) * 2 * G::H>();
        lds_reads_done();
        meet();
#pragma unroll
        for (int x = 0; x < G::NB; ++x) {
            pages.find(addr, tile_t0(fill), last_tok);
            load_both<G, PAGED, true>(addr, pages, kring_lds + fill_slot * G::SLOT, vring_lds + fill_slot * G::SLOT, tile_t0(fill), last_tok, lane, team);
            ++fill;
            fill_slot = fill_slot + 1 == G::S ? 0 : fill_slot + 1;
        }
    };
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
        const bool some = masked(t0);
        softmax_tile<G, RB>(st, s, pb, no_scales, t0, some, hidden, 0, c, lane);
        if (some) taken |= take_not_finite<G>(vt, lane);                       // (whoever comes second finds zeros)
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
#pragma unroll 1
        for (int it = 0; it < nt; ++it) {
            const int t0 = tile_t0(it);
            if (masked(t0)) add_not_finite_shown<G, RB, PAGED>(st, addr, t0, min(t0 + G::TT - 1, last_tok), hidden, lane);
        }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) st.l[rb] = sum_over_groups(st.l[rb]);

    // ---- join the streams, in a fixed order, and write
    const int row0 = team_row + ln;
    float* obuf = reinterpret_cast<float*>(smem);                              // [NP][RP][OROW]
    float* mlbuf = reinterpret_cast<float*>(smem + G::ML);                     // [NP][RP][2]
    if (G::NP > 1) {
        if (lg == 0) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                mlbuf[(part * G::RP + row0 + rb * 16) * 2 + 0] = st.m[rb];
                mlbuf[(part * G::RP + row0 + rb * 16) * 2 + 1] = st.l[rb];
            }
        }
        __syncthreads();
    }
    float factor[RB];                                    // what this wave's part of a row is multiplied by
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = row0 + rb * 16;
        float mm = st.m[rb], ll = st.l[rb];
        if (G::NP > 1) {
            float mw[G::NP];
            mm = kNoMaximum;
            ll = 0.f;
#pragma unroll
            for (int p = 0; p < G::NP; ++p) {
                mw[p] = mlbuf[(p * G::RP + row) * 2];
                mm = fmaxf(mm, mw[p]);
            }
#pragma unroll
            for (int p = 0; p < G::NP; ++p) ll += mlbuf[(p * G::RP + row) * 2 + 1] * fast_exp2(mw[p] - mm);
        }
        factor[rb] = G::NP > 1 ? fast_exp2(st.m[rb] - mm) : 1.f;
        if (a.direct) factor[rb] = ll == 0.f ? 0.f : factor[rb] / ll;          // (a row that attends nothing: zeros)
        if (part == 0 && lg == 0 && row < w.rows) {
            if (!a.direct) {
                a.part_ml[(pbase + row) * 2 + 0] = mm;
                a.part_ml[(pbase + row) * 2 + 1] = ll;
            } else if (a.lse_out) {
                const int r = w.r0 + row;
                a.lse_out[((int64_t)w.b * a.Hq + w.h * a.G + r % a.G) * a.Qmax + r / a.G] = (mm + log2f(ll)) * 0.6931471805599453f;
            }
        }
    }
    // four columns of a row
    auto put = [&](int row, int x, floatx4 o) {
        if (a.direct) {
            const int r = w.r0 + row;
            const bf16x4 y = {(__bf16)o[0], (__bf16)o[1], (__bf16)o[2], (__bf16)o[3]};
            *reinterpret_cast<bf16x4*>(a.out + (((int64_t)w.b * a.Qmax + r / a.G) * a.Hq + w.h * a.G + r % a.G) * G::D + x) = y;
        } else {
            *reinterpret_cast<floatx4*>(a.part_o + (pbase + row) * G::D + x) = o;
        }
    };
    if constexpr (G::NP == 1) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
            if (row0 + rb * 16 < w.rows)
#pragma unroll
                for (int db = 0; db < G::DB; ++db) put(row0 + rb * 16, db * 16 + lg * 4, st.acc[db][rb] * factor[rb]);
    } else {
        constexpr int DH = G::D / G::NH;
#pragma unroll
        for (int half = 0; half < G::NH; ++half) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int x = 0; x < G::DB / G::NH; ++x)
                    *reinterpret_cast<floatx4*>(obuf + (part * G::RP + row0 + rb * 16) * G::OROW + x * 16 + lg * 4) =
                        st.acc[half * (G::DB / G::NH) + x][rb] * factor[rb];
            __syncthreads();
            for (int f = tid; f < w.rows * (DH / 4); f += G::NW * 64) {
                const int row = f / (DH / 4), x = f % (DH / 4) * 4;
                floatx4 sum = *reinterpret_cast<const floatx4*>(obuf + row * G::OROW + x);
#pragma unroll
                for (int p = 1; p < G::NP; ++p) sum += *reinterpret_cast<const floatx4*>(obuf + (p * G::RP + row) * G::OROW + x);
                put(row, half * DH + x, sum);
            }
            if (half + 1 < G::NH) __syncthreads();
        }
    }
}

// The result of packed rows [from, to) of (b, h): zeros, and `lse`.
template <int D>
__device__ __forceinline__ void write_zeros(const StreamLaunch& a, int b, int h, int from, int to, float lse)
{
    for (int f = threadIdx.x; f < (to - from) * (D / 8); f += blockDim.x) {
        const int r = from + f / (D / 8);
        *reinterpret_cast<u32x4*>(a.out + (((int64_t)b * a.Qmax + r / a.G) * a.Hq + h * a.G + r % a.G) * D + f % (D / 8) * 8) = u32x4{0, 0, 0, 0};
    }
    if (a.lse_out)
        for (int r = from + threadIdx.x; r < to; r += blockDim.x)
            a.lse_out[((int64_t)b * a.Hq + h * a.G + r % a.G) * a.Qmax + r / a.G] = lse;
}

// Unit idx of `units` groups of `each`: neighbours of a group are eight apart, on one die.
__device__ __forceinline__ void place_of(int idx, int units, int each, int* unit, int* member)
{
    const int whole = units / 8 * 8;
    if (idx < whole * each) {
        *unit = idx / (8 * each) * 8 + idx % 8;
        *member = idx / 8 % each;
    } else {
        *unit = whole + (idx - whole * each) % (units - whole);
        *member = (idx - whole * each) / (units - whole);
    }
}

// One workgroup per (sequence and kv head, row tile, share).
template <class G, bool PAGED>
__global__ void __launch_bounds__(G::NW * 64) attn_window(StreamLaunch a)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    int unit, member;
    place_of(blockIdx.x, a.B * a.Hkv, a.tiles * a.groups, &unit, &member);
    unit = __builtin_amdgcn_readfirstlane(unit);
    member = __builtin_amdgcn_readfirstlane(member);
    // the last row tiles first: those of a prompt have the most tokens
    const int rt = a.tiles - 1 - member / a.groups, share = member % a.groups;
    RowTile w;
    w.b = unit / a.Hkv;
    w.h = unit % a.Hkv;
    w.L = __builtin_amdgcn_readfirstlane(seq_len(a, w.b));
    w.Q = __builtin_amdgcn_readfirstlane(seq_queries(a, w.b));
    w.r0 = rt * G::RP;
    const int end = min(w.r0 + G::RP, a.Qmax * a.G), real = min(end, w.Q * a.G);
    w.rows = real - w.r0;
    w.first = w.L - w.Q + w.r0 / a.G;
    w.last = w.L - w.Q + (real - 1) / a.G;
    const int attending = w.L > 0 && w.last >= 0 ? w.rows : 0;                 // 0: none of them attends anything
    if (a.direct) {
        const int from = max(w.r0, real);                                      // rows that a sequence does not have
        write_zeros<G::D>(a, w.b, w.h, from, end, 0.f);
        if (attending <= 0 && w.rows > 0) write_zeros<G::D>(a, w.b, w.h, w.r0, real, -INFINITY);
    }
    if (attending <= 0) return;
    const WindowSpan span(w.first, w.last, a.window, a.sinks, G::TT);
    const int quanta = (span.len + G::QUANTUM - 1) / G::QUANTUM;
    const int c0 = (int)((int64_t)quanta * share / a.groups) * G::QUANTUM;
    const int c1 = min((int)((int64_t)quanta * (share + 1) / a.groups) * G::QUANTUM, span.len);
    const int64_t pbase = (((int64_t)unit * a.tiles + rt) * a.groups + share) * G::RP;
    if (c0 >= c1) {                                                            // (the merge looks at the sums alone)
        for (int row = threadIdx.x; row < w.rows; row += G::NW * 64) {
            a.part_ml[(pbase + row) * 2 + 0] = kNoMaximum;
            a.part_ml[(pbase + row) * 2 + 1] = 0.f;
        }
        return;
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // (the two arms run the same barriers)
    if (G::RB0 == G::RB1 || wave < 4) window_piece<G, G::RB0, PAGED>(a, smem, w, span, c0, c1, pbase, wave % G::T * G::RB0 * 16);
    else window_piece<G, G::RB1, PAGED>(a, smem, w, span, c0, c1, pbase, G::RB0 * 64 + (wave - 4) * G::RB1 * 16);
}

// Joins the shares of a row, D / 4 lanes a row, in their order.  Grid: (blocks of rows, kv heads, sequences).
template <int D>
__global__ void __launch_bounds__(256) attn_window_merge(StreamLaunch a)
{
    constexpr int LANES = D / 4, ROWS = 256 / LANES;
    const int b = blockIdx.z, h = blockIdx.y, r = blockIdx.x * ROWS + threadIdx.x / LANES, x = threadIdx.x % LANES * 4;
    if (r >= a.Qmax * a.G) return;
    const int64_t at = ((int64_t)b * a.Qmax + r / a.G) * a.Hq + h * a.G + r % a.G;
    const int L = seq_len(a, b), Q = seq_queries(a, b);
    const bool real = r < Q * a.G;
    const int rt = r / a.RP, last_of_tile = min((rt + 1) * a.RP, Q * a.G) - 1;
    float M = kNoMaximum, den = 0.f;
    floatx4 num = {0.f, 0.f, 0.f, 0.f};
    if (real && L > 0 && L - Q + last_of_tile / a.G >= 0) {                    // (else the row tile has no partials)
        const int64_t slot = ((((int64_t)b * a.Hkv + h) * a.tiles + rt) * a.groups) * a.RP + r % a.RP;
        for (int s = 0; s < a.groups; ++s) {
            const int64_t p = slot + (int64_t)s * a.RP;
            const float m = a.part_ml[p * 2], l = a.part_ml[p * 2 + 1];
            if (l == 0.f) continue;                                            // (a NaN is not)
            const floatx4 o = *reinterpret_cast<const floatx4*>(a.part_o + p * D + x);
            const float top = fmaxf(M, m), old = fast_exp2(M - top), now = fast_exp2(m - top);
            num = num * old + o * now;
            den = den * old + l * now;
            M = top;
        }
    }
    const float inv = den == 0.f ? 0.f : 1.f / den;
    const bf16x4 o = {(__bf16)(num[0] * inv), (__bf16)(num[1] * inv), (__bf16)(num[2] * inv), (__bf16)(num[3] * inv)};
    *reinterpret_cast<bf16x4*>(a.out + at * D + x) = o;
    if (a.lse_out && x == 0)
        a.lse_out[((int64_t)b * a.Hq + h * a.G + r % a.G) * a.Qmax + r / a.G] = real ? (M + log2f(den)) * 0.6931471805599453f : 0.f;
}

}  // namespace

hipError_t configure_attn_window()
{
    for (int D = 64; D <= 128; D += 64)
        for (int rows : kRowTiles) {
            const hipError_t e = with_rows(D, rows, [](auto geo) {
                using G = decltype(geo);
                static_assert(G::LDS <= 160 * 1024, "LDS of a compute unit");
                const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(attn_window<G, false>),
                                                         hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
                if (e != hipSuccess) return e;
                return hipFuncSetAttribute(reinterpret_cast<const void*>(attn_window<G, true>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
            });
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

// Rows a workgroup and shares of its tokens: those that a simple account finds the fastest.  A workgroup takes a fixed time, most of it code that it runs for the
// first time and masks, and its tokens times a rate that is 0.17 + 0.83 RP / 256 of that of 256 rows; the chip takes as many rounds as it is filled by; shares cost their
// partials' way to memory and back, and a launch.  (us a call, 32 / 8 heads of 128, tiles of 128, 256, 384 rows: 400 rows, windows of 256 and 4096: 27, 38, 53 and
// 88, 149, 202 in one share, 22.5 and 36 in eight; 6400 rows, 1000 tokens: 79, 65, 88; 24000 rows: 237, 191, 180; 32K positions, a window of 4096: 2456, 2121, 1949, and
// with 192 rows 2175, with 320 2065.  Heads of 64 take 0.6 to 0.8 of the times, in small calls, and the same in large ones.)
float plan_attn_window(StreamLaunch& a, int n_cu)
{
    const int64_t R = (int64_t)a.Qmax * a.G, units = (int64_t)a.B * a.Hkv;
    float best = INFINITY;
    for (int rows : kRowTiles) {
        int quantum = 0;
        (void)with_rows(a.D, rows, [&](auto geo) {
            quantum = decltype(geo)::QUANTUM;
            return hipSuccess;
        });
        const int64_t tiles = (R + rows - 1) / rows, grid = units * tiles;
        const int64_t span = (int64_t)a.sinks + a.window + rows / a.G + 2 * 64, tokens = span < a.max_ctx ? span : a.max_ctx;
        const int64_t most = (tokens + quantum - 1) / quantum;
        const float fixed = 13.f + rows / 16.f, a_token = (0.17f + 0.83f / 256 * rows) * 0.028f;       // us
        for (int k = 0; k <= 3; ++k) {
            int64_t groups = k * n_cu / grid;
            groups = groups > most ? most : groups < 1 ? 1 : groups;
            const int64_t rounds = (grid * groups + n_cu - 1) / n_cu;
            const float partials = groups > 1 ? 2.f + (float)(grid * groups) * (rows * (a.D + 2) * 8) * 0.04e-6f : 0.f;
            const float time = (float)rounds * (fixed + a_token * (float)tokens / (float)groups) + partials;
            if (time >= best) continue;
            best = time;
            a.RP = rows;
            a.tiles = (int)tiles;
            a.quantum = quantum;
            a.groups = (int)groups;
        }
    }
    a.nslots = a.groups;
    a.rot = 0;
    a.direct = a.groups == 1;
    return best;
}

size_t attn_window_workspace_bytes(const StreamLaunch& a)
{
    if (a.direct) return 256;
    const size_t rows = (size_t)a.B * a.Hkv * a.tiles * a.groups * a.RP;
    return (rows * a.D * 4 + 255) / 256 * 256 + (rows * 8 + 255) / 256 * 256;
}

void bind_attn_window(StreamLaunch& a, void* workspace)
{
    const size_t rows = (size_t)a.B * a.Hkv * a.tiles * a.groups * a.RP;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + (rows * a.D * 4 + 255) / 256 * 256);
}

hipError_t launch_attn_window(const StreamLaunch& a, hipStream_t stream)
{
    const hipError_t e = with_rows(a.D, a.RP, [&](auto geo) {
        using G = decltype(geo);
        auto fn = a.own.page_table ? attn_window<G, true> : attn_window<G, false>;
        hipLaunchKernelGGL(fn, dim3((unsigned)a.B * a.Hkv * a.tiles * a.groups), dim3(G::NW * 64), G::LDS, stream, a);
        return hipGetLastError();
    });
    if (e != hipSuccess || a.direct) return e;
    const int rows = 256 / (a.D / 4);
    auto fn = a.D == 128 ? attn_window_merge<128> : attn_window_merge<64>;
    hipLaunchKernelGGL(fn, dim3((a.Qmax * a.G + rows - 1) / rows, a.Hkv, a.B), dim3(256), 0, stream, a);
    return hipGetLastError();
}
