// Tiles of K and V, in bf16 or in 8 bits: how they are divided among workgroups, loaded, multiplied and weighted.  Used by the kernels of
// attn_stream.hip and attn_prefix.hip.
#pragma once
#include "attn_exchange.h"
#include "attn_primitives.h"
#include "attn_stream.h"

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

namespace {

constexpr float kRescaleLog2 = 8.0f;   // the running maximum only moves when a tile exceeds it by this (log2 units)
constexpr float kNoMaximum = -3.402823466e38f;   // a row that has met no score yet: finite, so that differences are no NaN; no score is below it
constexpr float kFar = 8388608.f;      // 2^23: from here on a reference is far from zero (softmax_tile)
constexpr int kPieceQuanta = 2;        // what a sequence costs a workgroup besides its tokens, in quanta

template <int D_, bool QUANT_, int TB_>
struct TileGeo {
    static constexpr int D = D_, TB = TB_;                        // TB: blocks of 16 tokens in a tile
    static constexpr bool QUANT = QUANT_;
    static constexpr int TT = TB * 16;                            // tokens of a tile
    static constexpr int KS = D / 32, DB = D / 16;                // steps of the QK product, blocks of the head dim
    static constexpr int ROWB = QUANT ? D : 2 * D;                // bytes of a K or V row
    static constexpr int CPR = ROWB / 16;                         // 16-byte chunks of it
    static constexpr int RPI = 64 / CPR;                          // rows that one wave-wide 1 KiB load moves
    static constexpr int NLD = TT / RPI;                          // loads of a tile
    static constexpr int SLOT = TT * ROWB;                        // bytes of a K or V tile
    static constexpr int SC = QUANT ? 1 : 0;                      // loads of a tile's scales
    static constexpr int QROWB = 2 * D;
};

// Swizzles: chunk c of row r is stored at c ^ f(r).  A 128-bit read of K or Q takes 16 consecutive rows at one logical chunk; a transposed read of
// V takes, per half of the wave, rows 0..7 and 16..23 (or 8..15 and 24..31) of 32.
template <int ROWB> __device__ __forceinline__ int k_swz(int r) { return ROWB == 256 ? r & 15 : ROWB == 128 ? (r >> 1) & 7 : (r >> 2) & 3; }
template <bool QUANT, int ROWB> __device__ __forceinline__ int v_swz(int r)
{
    if (QUANT) return ROWB == 128 ? ((r >> 1) & 3) | (r >> 4 & 1) << 2 : (r >> 2 & 1) | (r >> 4 & 1) << 1;
    return ROWB == 256 ? (r & 7) << 1 : (r >> 1 & 3) << 1;
}

// ---- shares
// Each sequence costs its tokens in quanta and, but for the first, kPieceQuanta more, which come first; the sum is cut into equal shares.  (A share
// has one piece anyhow, and a piece more for each sequence that begins in it.)
__device__ __forceinline__ int seq_len(const StreamLaunch& a, int b) { return max(min(a.ctx_lens[b], a.max_ctx), 0); }
__device__ __forceinline__ int seq_queries(const StreamLaunch& a, int b)
{
    return min(max(a.gammas ? a.gammas[b] : a.gamma, 0), a.Qmax - 1) + 1;
}
__device__ __forceinline__ int piece_cost(int b) { return b ? kPieceQuanta : 0; }
__device__ __forceinline__ int seq_cost(int L, int b, int quantum) { return L > 0 ? (L + quantum - 1) / quantum + piece_cost(b) : 0; }

struct Shares {
    int used, len, rest;                // shares in use; the first `rest` of them have len + 1 quanta
    __device__ __forceinline__ Shares(int total, int groups) : used(max(1, min(groups, total)))
    {
        len = (int)((unsigned)total / (unsigned)used);
        rest = total - len * used;
    }
    __device__ __forceinline__ int begin(int g) const { return g >= used ? 0x7fffffff : g * len + min(g, rest); }
    __device__ __forceinline__ int owner(int x) const
    {
        const int head = rest * (len + 1);
        return x < head ? (int)((unsigned)x / (unsigned)(len + 1)) : rest + (int)((unsigned)(x - head) / (unsigned)max(len, 1));
    }
};
// Calls piece(b, L, c0, c1) for every piece [c0, c1) of a sequence b in share g, in order.  Sequences are taken 64 at a time, one a lane.
template <class Piece>
__device__ __forceinline__ void for_each_piece(const StreamLaunch& a, int g, int lane, int len, int quantum, Piece piece)
{                                                        // len: of sequence `lane`, 0 where there is none
    int cost = seq_cost(len, lane, quantum);
    int end = scan_costs(cost);                          // cost of the sequences up to this one
    int total = __builtin_amdgcn_readlane(end, 63);
    for (int b0 = 64; b0 < a.B; b0 += 64)
        total += __builtin_amdgcn_readlane(scan_costs(b0 + lane < a.B ? seq_cost(seq_len(a, b0 + lane), b0 + lane, quantum) : 0), 63);
    const Shares sh(total, a.groups);
    const int x0 = sh.begin(g), x1 = min(sh.begin(g + 1), total);
    if (x0 >= x1) return;
    for (int b0 = 0;;) {
        const int tok = end - cost + piece_cost(b0 + lane);       // position of the sequence's first tokens
        const bool mine = cost > 0 && end > x0 && tok < x1;
        for (unsigned long long todo = __ballot(mine); todo; todo &= todo - 1) {
            const int l = __ffsll((long long)todo) - 1;
            const int t = __builtin_amdgcn_readlane(tok, l), L = __builtin_amdgcn_readlane(len, l);
            const int c0 = max(x0 - t, 0) * quantum;
            const int c1 = min((min(x1, __builtin_amdgcn_readlane(end, l)) - t) * quantum, L);
            if (c0 < c1) piece(b0 + l, L, c0, c1);
        }
        const int before = __builtin_amdgcn_readlane(end, 63);
        b0 += 64;
        if (b0 >= a.B || before >= x1) return;
        len = b0 + lane < a.B ? seq_len(a, b0 + lane) : 0;
        cost = seq_cost(len, b0 + lane, quantum);
        end = before + scan_costs(cost);
    }
}

// The same number, of which the compiler knows nothing: what rare paths make of it is computed there, and does not take registers from the
// main loop (a spilled one is loaded back ahead of the loop, and that load waits for all the tiles under way).  Three blocks of 16 rows a wave use all
// there are: a few kernels keep 12 bytes in scratch, written ahead of the loop or read behind it.
__device__ __forceinline__ int opaque(int lane)
{
    asm volatile("" : "+v"(lane));
    return lane;
}

// ---- loads
// Where the rows of this (sequence, kv head) start: uniform bases and a 32-bit byte offset per lane (the host checks that a
// sequence, or a page, spans less than 4 GiB).
struct RowAddr {
    const char *k, *v;
    const uint8_t *ks, *vs;
    const __attribute__((address_space(4))) int32_t* pages;      // read as scalars
    uint32_t tok_bytes;
    int64_t page_bytes, scale_page_bytes;
    int page_shift, page_mask, page_hi;
};
template <class G, bool PAGED>
__device__ __forceinline__ RowAddr make_row_addr(const AttnSource& s, int b, int h)
{
    constexpr int E = G::QUANT ? 1 : 2;
    RowAddr r;
    const int64_t at = ((int64_t)h * s.hstride + (PAGED ? 0 : (int64_t)b * s.bstride)) * E;
    r.k = static_cast<const char*>(s.k) + at;
    r.v = static_cast<const char*>(s.v) + at;
    const int64_t sat = (int64_t)h * s.shstride + (PAGED ? 0 : (int64_t)b * s.sbstride);
    r.ks = s.ks + sat;
    r.vs = s.vs + sat;
    r.pages = PAGED ? (const __attribute__((address_space(4))) int32_t*)(s.page_table + (int64_t)b * s.max_pages) : nullptr;
    r.tok_bytes = (uint32_t)(s.tstride * E);
    r.page_bytes = s.pstride * E;
    r.scale_page_bytes = s.spstride;
    r.page_shift = s.page_shift;
    r.page_mask = s.page_mask;
    r.page_hi = s.page_hi;
    return r;
}

// The pages of a tile's blocks of 16 tokens (a page holds 16 tokens at least).
template <class G, bool PAGED>
struct TilePages {
    int id[G::TB];
    __device__ __forceinline__ void find(const RowAddr& ra, int t0, int last_tok)
    {
        if (!PAGED) return;
#pragma unroll
        for (int j = 0; j < G::TB; ++j) id[j] = min(max(ra.pages[min(t0 + 16 * j, last_tok) >> ra.page_shift], 0), ra.page_hi);
    }
    // the page of block j, which may differ from lane to lane; selected, never indexed
    __device__ __forceinline__ int of(int j) const
    {
        int r = __builtin_amdgcn_readfirstlane(id[0]);
#pragma unroll
        for (int x = 1; x < G::TB; ++x) {
            const int other = __builtin_amdgcn_readfirstlane(id[x]);
            r = j == x ? other : r;
        }
        return r;
    }
};

// Loads [e0, e0 + N) of a tile of K or V into `slot`.  Rows past `last_tok` are clamped to it (always a valid address); the softmax masks them.
// Where there are none, all that varies from load to load and from tile to tile is uniform and goes into the base; a lane's own offset
// only depends on the swizzle (f(e RPI + r) = f(e RPI) ^ f(r): fields of bits).
template <class G, bool PAGED, bool IS_V, int N>
__device__ __forceinline__ void load_tile(const RowAddr& ra, const TilePages<G, PAGED>& pages, uint32_t slot, int t0, int last_tok, int lane, int e0)
{
    const char* base = IS_V ? ra.v : ra.k;
    const int r_local = lane / G::CPR, cpos = lane % G::CPR;
    auto swz = [](int row) { return IS_V ? v_swz<G::QUANT, G::ROWB>(row) : k_swz<G::ROWB>(row); };
    if (t0 + G::TT - 1 <= last_tok) {
        const uint32_t row_off = (uint32_t)r_local * ra.tok_bytes;
#pragma unroll
        for (int x = 0; x < N; ++x) {
            const int e = e0 + x;
            const uint32_t off = row_off + (uint32_t)((cpos ^ swz(r_local)) ^ swz(e * G::RPI)) * 16u;
            if (PAGED) {
                const int id = __builtin_amdgcn_readfirstlane(pages.of(e * G::RPI / 16));
                dma16(base + (int64_t)id * ra.page_bytes + (uint32_t)((t0 + e * G::RPI) & ra.page_mask) * ra.tok_bytes, off, slot + e * 1024);
            } else {
                dma16(base + (uint32_t)(t0 + e * G::RPI) * ra.tok_bytes, off, slot + e * 1024);
            }
        }
        return;
    }
    lane = opaque(lane);
#pragma unroll
    for (int x = 0; x < N; ++x) {
        const int e = e0 + x;
        const int row = e * G::RPI + lane / G::CPR;
        const int c = lane % G::CPR ^ swz(row);
        const int tok = min(t0 + row, last_tok);
        if (PAGED) {
            const int id = __builtin_amdgcn_readfirstlane(pages.of(e * G::RPI / 16));
            dma16(base + (int64_t)id * ra.page_bytes, (uint32_t)(tok & ra.page_mask) * ra.tok_bytes + (uint32_t)c * 16u, slot + e * 1024);
        } else {
            dma16(base, (uint32_t)tok * ra.tok_bytes + (uint32_t)c * 16u, slot + e * 1024);
        }
    }
}

// 4 bytes a lane, HBM -> LDS bytes [lds_addr + 4 i, + 4).
__device__ __forceinline__ void dma4(const uint8_t* at, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off"
                 :
                 : "v"(at), "s"(lds_addr)
                 : "memory", "m0");
}
// The scales of a tile: TT bytes of K's, TT of V's, four a lane (the other lanes repeat them behind).  Groups of four tokens are read
// whole; bytes past the last token, inside the row's multiple of 16, belong to tokens that the softmax masks.
template <class G, bool PAGED>
__device__ __forceinline__ void load_scales(const RowAddr& ra, const TilePages<G, PAGED>& pages, uint32_t slot, int t0, int last_tok, int lane)
{
    if (!G::QUANT) return;
    const int i = lane % (G::TT / 4);
    const int tok = min(t0 + 4 * i, last_tok & ~3);
    const uint8_t* at = (lane / (G::TT / 4)) & 1 ? ra.vs : ra.ks;
    if (PAGED) {
        at += (int64_t)pages.of(i / 4) * ra.scale_page_bytes + (tok & ra.page_mask);
    } else {
        at += tok;
    }
    dma4(at, slot);
}

// ---- mathematics
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

template <bool HI>
__device__ __forceinline__ bf16x2 two_values(uint32_t w, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI); }
__device__ __forceinline__ bf16x8 eight_values(uint32_t w0, uint32_t w1, float scale)
{
    const bf16x2 a = two_values<false>(w0, scale), b = two_values<true>(w0, scale), c = two_values<false>(w1, scale),
                 d = two_values<true>(w1, scale);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

template <class G, int RB>
struct WaveState {
    float m[RB];                     // reference maximum per query row, log2 units (score * scale * log2 e); kNoMaximum at first
    float l[RB];                     // running sum, this lane group's tokens only
    bool far = false;                // a reference is far from zero (of the wave's rows: uniform)
    floatx4 acc[G::DB][RB];          // O^T: column 16 db + 4 (lane / 16) + i, row 16 rb + lane % 16
};

// S^T[token][row] for the tile in `kt`, bf16.
template <class G, int RB>
__device__ __forceinline__ void score_tile(floatx4 (&s)[G::TB][RB], const bf16x8 (&qf)[RB][G::KS], const char* kt, int lane)
{
    const int ln = lane & 15, lg = lane >> 4;
#pragma unroll
    for (int tb = 0; tb < G::TB; ++tb) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) s[tb][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
        const int row = tb * 16 + ln;
#pragma unroll
        for (int ks = 0; ks < G::KS; ++ks) {
            const int c = (ks * 4 + lg) ^ k_swz<G::ROWB>(row);
            const bf16x8 ka = *reinterpret_cast<const bf16x8*>(kt + row * G::ROWB + c * 16);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
                s[tb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qf[rb][ks], s[tb][rb], 0, 0, 0);
        }
    }
}

// A tile in 8 bits, out of LDS: this lane's codes of K (16 at a time, which feed two steps of the product: step 2p + h of lane group lg holds
// elements 64 p + 16 lg + 8 h .. + 7, of K and of Q alike; any order of a sum's terms will do), its token's scales, its columns of V (eight
// tokens each), the scales of V's tokens (four a block).  K's reads are issued together, and V's, so that the latency of LDS is met twice a tile.
template <class G>
struct RawTile {
    u32x4 k[G::TB][G::KS / 2];
    i32x2 v[G::TB / 2][G::DB];
    uint32_t ks[G::TB], vs[G::TB];

    __device__ __forceinline__ void read_k(const char* kt, const char* sc, int lane)
    {
        const int ln = lane & 15, lg = lane >> 4;
#pragma unroll
        for (int tb = 0; tb < G::TB; ++tb) {
            const int row = tb * 16 + ln;
            ks[tb] = *reinterpret_cast<const uint8_t*>(sc + row);
#pragma unroll
            for (int p = 0; p < G::KS / 2; ++p)
                k[tb][p] = *reinterpret_cast<const u32x4*>(kt + row * G::ROWB + ((p * 4 + lg) ^ k_swz<G::ROWB>(row)) * 16);
            vs[tb] = *reinterpret_cast<const uint32_t*>(sc + G::TT + tb * 16 + lg * 4);
        }
    }
    __device__ __forceinline__ void read_v(char* vt, int lane)
    {
        const int ln = lane & 15, lg = lane >> 4;
#pragma unroll
        for (int kk = 0; kk < G::TB / 2; ++kk)
#pragma unroll
            for (int db = 0; db < G::DB; ++db) {
                // eight rows of 16 codes: lane i of a group gives the address of row i / 2, half i % 2, and gets column i
                const int r = ln >> 1, row = kk * 32 + (r >> 2) * 16 + lg * 4 + (r & 3);
                v[kk][db] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                    (i32x2 __attribute__((address_space(3)))*)(vt + row * G::ROWB + (db ^ v_swz<true, G::ROWB>(row)) * 16 + (ln & 1) * 8));
            }
    }
    template <int RB>
    __device__ __forceinline__ void scores(floatx4 (&s)[G::TB][RB], const bf16x8 (&qf)[RB][G::KS]) const
    {
#pragma unroll
        for (int tb = 0; tb < G::TB; ++tb) {
            const float scale = scale_value(ks[tb]);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) s[tb][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < G::KS / 2; ++p)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bf16x8 ka = eight_values(k[tb][p][2 * h], k[tb][p][2 * h + 1], scale);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
                        s[tb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qf[rb][2 * p + h], s[tb][rb], 0, 0, 0);
                }
        }
    }
    template <int RB>
    __device__ __forceinline__ void add_values(WaveState<G, RB>& st, const bf16x8 (&pb)[G::TB / 2][RB]) const
    {
#pragma unroll
        for (int kk = 0; kk < G::TB / 2; ++kk)
#pragma unroll
            for (int db = 0; db < G::DB; ++db) {
                const bf16x8 va = eight_values((uint32_t)v[kk][db][0], (uint32_t)v[kk][db][1], 1.0f);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
                    st.acc[db][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[kk][rb], st.acc[db][rb], 0, 0, 0);
            }
    }
};
// The order of what stands before and after stays.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }
// A barrier that waits for nothing: reads of LDS may be under way across it.
__device__ __forceinline__ void meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// s c - m with the product rounded first.
__device__ __forceinline__ float rounded_exponent(float s, float c, float m)
{
#pragma clang fp contract(off)
    const float y = s * c;
    return y - m;
}

// Mask, online softmax; leaves P^T (in 8 bits: times V's scales), rounded to bf16 as the matrix cores take it, as the B operand of PV: slot j of lane group lg in step kk is token
// 32 kk + 16 (j / 4) + 4 lg + j % 4, what this lane holds in s[2 kk + j / 4][.][j % 4].
// That is the one rounding of a weight, by at most half a step, 2^-8 of it; an operand of more bits would take a second product.  Against 64 bits a result, with its
// own rounding, is up to 1.4 times as far off as one of 32-bit weights.  The sum of the weights takes them unrounded.
// The reference maximum only moves when a score exceeds it by kRescaleLog2; until then p = 2^(s - ref) <= 2^kRescaleLog2, exact in the final
// ratio.  So a tile's own maxima are only looked at lane by lane, and brought together over the lanes of a row when one of them asks for it.
template <class G, int RB>
__device__ __forceinline__ void softmax_tile(WaveState<G, RB>& st, floatx4 (&s)[G::TB][RB], bf16x8 (&pb)[G::TB / 2][RB],
                                             const uint32_t (&vs)[G::TB], int t0, bool masked, const int (&lim)[RB], int end, float c, int lane)
{
    float vscale[G::TB][4];
    if (G::QUANT) {
#pragma unroll
        for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
            for (int i = 0; i < 4; ++i) vscale[tb][i] = scale_value(vs[tb] >> (8 * i) & 0xffu);
    }
    if (masked) {
        asm volatile("" : "+s"(t0));                       // a branch, not selects in every tile
        const int lg = opaque(lane) >> 4;
#pragma unroll
        for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int tok = t0 + tb * 16 + lg * 4 + i;
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
                    if (tok > lim[rb]) s[tb][rb][i] = -INFINITY;
                if (G::QUANT && tok >= end) vscale[tb][i] = 0.f;       // a scale that belongs to no token may be anything
            }
    }
    float mx[RB];
    bool above = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        mx[rb] = s[0][rb][0];
#pragma unroll
        for (int x = 1; x < G::TB * 4; ++x) mx[rb] = __builtin_elementwise_maximum(mx[rb], s[x / 4][rb][x % 4]);   // (a NaN stays one)
        above |= rounded_exponent(mx[rb], c, st.m[rb]) > kRescaleLog2;
    }
    if (__any(above)) {
        bool far = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const float top = max_over_groups(mx[rb]);
            const float m_new = rounded_exponent(top, c, st.m[rb]) > kRescaleLog2 ? top * c : st.m[rb];
            const float alpha = fast_exp2(st.m[rb] - m_new);
            st.m[rb] = m_new;
            far |= fabsf(m_new) >= kFar && m_new > kNoMaximum;
            st.l[rb] *= alpha;
#pragma unroll
            for (int db = 0; db < G::DB; ++db)
#pragma unroll
                for (int i = 0; i < 4; ++i) st.acc[db][rb][i] *= alpha;
        }
        st.far = __any(far);
    }
    float ref[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) ref[rb] = st.m[rb];
    if (st.far) {
        const float inv = 1.f / c;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            if (fabsf(ref[rb]) < kFar) continue;
#pragma unroll
            for (int x = 0; x < G::TB * 4; ++x) s[x / 4][rb][x % 4] = rounded_exponent(s[x / 4][rb][x % 4], c, ref[rb]) * inv;
            ref[rb] = 0.f;
        }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float sum = 0.f;
#pragma unroll
        for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = fast_exp2(fmaf(s[tb][rb][i], c, -ref[rb]));
                sum += p;
                pb[tb / 2][rb][(tb & 1) * 4 + i] = (__bf16)(G::QUANT ? p * vscale[tb][i] : p);
            }
        st.l[rb] += sum;
    }
}

// What is not finite, in four codes or two bf16 values: all bits of such an element.
template <bool QUANT>
__device__ __forceinline__ uint32_t not_finite(uint32_t w)
{
    if (QUANT) {
        const uint32_t nan = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;      // 0x7f + 1 carries into the sign's place
        return (nan >> 7) * 0xffu;
    }
    return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// O^T[column][row] += sum_token V[token][column] P[row][token], bf16.
template <class G, int RB>
__device__ __forceinline__ void pv_tile(WaveState<G, RB>& st, const bf16x8 (&pb)[G::TB / 2][RB], char* vt, int lane)
{
    const int ln = lane & 15, lg = lane >> 4;
#pragma unroll
    for (int kk = 0; kk < G::TB / 2; ++kk)
#pragma unroll
        for (int db = 0; db < G::DB; ++db) {
            s16x4 half[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = kk * 32 + h * 16 + lg * 4 + (ln >> 2);
                const int c = (db * 2) ^ v_swz<false, G::ROWB>(row);
                half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (s16x4 __attribute__((address_space(3)))*)(vt + row * G::ROWB + c * 16 + (ln & 3) * 8));
            }
            const s16x8 both = __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
            const bf16x8 va = __builtin_bit_cast(bf16x8, both);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
                st.acc[db][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[kk][rb], st.acc[db][rb], 0, 0, 0);
        }
}

// In a tile of which some rows do not attend some tokens, a weight of zero times a NaN or an infinity of V would be NaN.  Such elements
// are taken out of the tile in LDS (true: there were any) and added in the end to the rows that attend their token, whose
// positive weight does not change them.
template <class G>
__device__ __forceinline__ bool take_not_finite(char* vt, int lane)
{
    bool any = false;
    lane = opaque(lane);
#pragma unroll 1
    for (int x = 0; x < G::SLOT / 1024; ++x) {
        u32x4* at = reinterpret_cast<u32x4*>(vt + x * 1024 + lane * 16);
        u32x4 w = *at;
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t n = not_finite<G::QUANT>(w[i]);
            w[i] &= ~n;
            bad |= n;
        }
        if (bad) *at = w;
        any |= bad != 0;
    }
    return __any(any);
}
template <class G, int RB, bool PAGED>
__device__ __forceinline__ void add_not_finite(WaveState<G, RB>& st, const RowAddr& ra, int begin, int end, int step, const int (&lim)[RB], int lane)
{                                                        // tiles of a stream, `step` tokens apart, from token `begin` on
    const int lg = opaque(lane) >> 4;
#pragma unroll 1
    for (int t = begin, left = G::TT; t < end; ++t) {
        const char* row = ra.v;
        if (PAGED) row += (int64_t)min(max(ra.pages[t >> ra.page_shift], 0), ra.page_hi) * ra.page_bytes;
        row += (uint32_t)(PAGED ? t & ra.page_mask : t) * ra.tok_bytes;
#pragma unroll
        for (int db = 0; db < G::DB; ++db) {
            uint32_t bits[4];                            // columns 16 db + 4 lg .. + 3
            if (G::QUANT) {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(row + db * 16 + lg * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) bits[i] = (w >> (8 * i) & 0x7fu) == 0x7fu ? 0x7fc00000u : 0u;
            } else {
                const u32x2 w = *reinterpret_cast<const u32x2*>(row + db * 32 + lg * 8);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t x = i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16;
                    bits[i] = (x & 0x7f800000u) == 0x7f800000u ? x : 0u;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
                    if (bits[i] && t <= lim[rb]) st.acc[db][rb][i] += __uint_as_float(bits[i]);
        }
        if (--left == 0) {
            left = G::TT;
            t += step - G::TT;
        }
    }
}

}  // namespace
