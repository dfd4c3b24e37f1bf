// Verification attention over a cache in 8 bits (gfx950), and over the sequences' own tokens behind a shared prefix.
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
#include "attn_exchange.h"
#include "attn_primitives.h"
#include "attn_stream.h"

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

namespace {

constexpr float kRescaleLog2 = 8.0f;   // the running maximum only moves when a tile exceeds it by this (log2 units)
constexpr int kPieceQuanta = 2;        // what a sequence costs a workgroup besides its tokens, in quanta

// RB0: row blocks of 16 that a wave has, or team 0; RB1: those of team 1, 0 = there are no teams.
template <int D_, bool QUANT_, int RB0_, int RB1_>
struct Geo {
    static constexpr int D = D_, RB0 = RB0_, RB1 = RB1_, RB = RB0 + RB1;
    static constexpr bool QUANT = QUANT_, TEAMS = RB1 > 0;
    static constexpr int NP = QUANT && !TEAMS ? 8 : 4;            // token streams of a workgroup
    static constexpr int NW = TEAMS ? 2 * NP : NP;                // waves
    static constexpr int TB = QUANT && D == 64 ? 4 : 2;           // blocks of 16 tokens in a tile
    static constexpr int TT = TB * 16;                            // tokens of a tile
    static constexpr int QUANTUM = NP * TT;                       // tokens of a workgroup's step
    static constexpr int KS = D / 32, DB = D / 16;                // steps of the QK product, blocks of the head dim
    static constexpr int ROWB = QUANT ? D : 2 * D;                // bytes of a K or V row
    static constexpr int CPR = ROWB / 16;                         // 16-byte chunks of it
    static constexpr int RPI = 64 / CPR;                          // rows that one wave-wide 1 KiB load moves
    static constexpr int NLD = TT / RPI;                          // loads of a tile
    static constexpr int SLOT = TT * ROWB;                        // bytes of a K or V tile
    static constexpr int SC = QUANT ? 1 : 0;                      // loads of a tile's scales
    static constexpr int S = 128 * 1024 / NP / (2 * SLOT);        // tiles of a ring: the loads in flight fill 128 KiB
    static constexpr int RING = S * (2 * SLOT + SC * 256);        // S tiles of K, of V, of scales
    static constexpr int QROWB = 2 * D, QCPR = QROWB / 16, QRPI = 64 / QCPR;
    static constexpr int RP = RB * 16;
    static constexpr int NH = NP * RP * (D + 4) * 4 > 140 * 1024 ? 2 : 1;   // passes of the last exchange, D / NH columns each
    static constexpr int OROW = D / NH + 4;                       // padded row of the exchange (floats)
    static constexpr int TILES = NP * RING + RP * QROWB;
    static constexpr int MERGE = NP * RP * OROW * 4;
    static constexpr int ML = TILES > MERGE ? TILES : MERGE;      // where the waves' (m, l) lie
    static constexpr int TAKEN = ML + NW * (TEAMS ? (RB0 > RB1 ? RB0 : RB1) : RB0) * 16 * 8;   // a word for each stream
    static constexpr int LDS = TAKEN + (TEAMS ? NP * 4 : 0);
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
// Each sequence costs its tokens in quanta and kPieceQuanta more, which come first; the sum is cut into equal shares.
__device__ __forceinline__ int seq_len(const StreamLaunch& a, int b) { return max(min(a.ctx_lens[b], a.max_ctx), 0); }
__device__ __forceinline__ int seq_queries(const StreamLaunch& a, int b)
{
    return min(max(a.gammas ? a.gammas[b] : a.gamma, 0), a.Qmax - 1) + 1;
}
__device__ __forceinline__ int seq_cost(int L, int quantum) { return L > 0 ? (L + quantum - 1) / quantum + kPieceQuanta : 0; }

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
__device__ __forceinline__ int total_cost(const StreamLaunch& a, int lane, int quantum)
{
    int total = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64)
        total += __builtin_amdgcn_readlane(scan_costs(b0 + lane < a.B ? seq_cost(seq_len(a, b0 + lane), quantum) : 0), 63);
    return total;
}
// Calls piece(b, L, c0, c1) for every piece [c0, c1) of a sequence b in share g, in order.
template <class Piece>
__device__ __forceinline__ void for_each_piece(const StreamLaunch& a, int g, int lane, int quantum, Piece piece)
{
    const int total = total_cost(a, lane, quantum);
    const Shares sh(total, a.groups);
    const int x0 = sh.begin(g), x1 = min(sh.begin(g + 1), total);
    if (x0 >= x1) return;
    int before = 0;                                      // cost of the sequences before b0
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const int len = b0 + lane < a.B ? seq_len(a, b0 + lane) : 0;
        const int cost = seq_cost(len, quantum);
        const int end = before + scan_costs(cost);
        const int tok = end - cost + kPieceQuanta;       // position of the sequence's first tokens
        const bool mine = cost > 0 && end > x0 && tok < x1;
        for (unsigned long long todo = __ballot(mine); todo; todo &= todo - 1) {
            const int l = __ffsll((long long)todo) - 1;
            const int t = __builtin_amdgcn_readlane(tok, l), L = __builtin_amdgcn_readlane(len, l);
            const int c0 = max(x0 - t, 0) * quantum;
            const int c1 = min((min(x1, __builtin_amdgcn_readlane(end, l)) - t) * quantum, L);
            if (c0 < c1) piece(b0 + l, L, c0, c1);
        }
        before = __builtin_amdgcn_readlane(end, 63);
        if (before >= x1) break;
    }
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

// Loads [E0, E1) of a tile of K or V into `slot`.  Rows past `last_tok` are clamped to it (always a valid address); the softmax masks them.
template <class G, bool PAGED, bool IS_V>
__device__ __forceinline__ void load_tile(const RowAddr& ra, const TilePages<G, PAGED>& pages, uint32_t slot, int t0, int last_tok, int lane,
                                          int e0, int n)
{
    const char* base = IS_V ? ra.v : ra.k;
    const int r_local = lane / G::CPR, cpos = lane % G::CPR;
#pragma unroll
    for (int x = 0; x < G::NLD; ++x) {
        if (x >= n) break;
        const int e = e0 + x;
        const int row = e * G::RPI + r_local;
        const int c = cpos ^ (IS_V ? v_swz<G::QUANT, G::ROWB>(row) : k_swz<G::ROWB>(row));
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
    float m[RB];                     // reference maximum per query row, log2 units (score * scale * log2 e)
    float l[RB];                     // running sum, this lane group's tokens only
    floatx4 acc[G::DB][RB];          // O^T: column 16 db + 4 (lane / 16) + i, row 16 rb + lane % 16
};

// S^T[token][row] for the tile in `kt`.  In 8 bits a lane reads 16 codes at a time, which feed two steps: step 2p + h of lane group lg holds
// elements 64 p + 16 lg + 8 h .. + 7 (of K and of Q alike; any order of a sum's terms will do).
template <class G, int RB>
__device__ __forceinline__ void score_tile(floatx4 (&s)[G::TB][RB], const bf16x8 (&qf)[RB][G::KS], const char* kt, const char* sc, int lane)
{
    const int ln = lane & 15, lg = lane >> 4;
#pragma unroll
    for (int tb = 0; tb < G::TB; ++tb) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) s[tb][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
        const int row = tb * 16 + ln;
        if constexpr (G::QUANT) {
            const float scale = scale_value(*reinterpret_cast<const uint8_t*>(sc + row));
#pragma unroll
            for (int p = 0; p < G::KS / 2; ++p) {
                const int c = (p * 4 + lg) ^ k_swz<G::ROWB>(row);
                const u32x4 raw = *reinterpret_cast<const u32x4*>(kt + row * G::ROWB + c * 16);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bf16x8 ka = eight_values(raw[2 * h], raw[2 * h + 1], scale);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
                        s[tb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qf[rb][2 * p + h], s[tb][rb], 0, 0, 0);
                }
            }
        } else {
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
}

// The scales of V's tokens, four a block: those of this lane group.
template <class G>
__device__ __forceinline__ void value_scales(uint32_t (&vs)[G::TB], const char* sc, int lane)
{
    if (!G::QUANT) return;
#pragma unroll
    for (int tb = 0; tb < G::TB; ++tb) vs[tb] = *reinterpret_cast<const uint32_t*>(sc + G::TT + tb * 16 + (lane >> 4) * 4);
}

// Mask, online softmax; leaves P^T (in 8 bits: times V's scales) as the B operand of PV: slot j of lane group lg in step kk is token
// 32 kk + 16 (j / 4) + 4 lg + j % 4, what this lane holds in s[2 kk + j / 4][.][j % 4].
template <class G, int RB>
__device__ __forceinline__ void softmax_tile(WaveState<G, RB>& st, floatx4 (&s)[G::TB][RB], bf16x8 (&pb)[G::TB / 2][RB],
                                             const uint32_t (&vs)[G::TB], int t0, bool masked, const int (&lim)[RB], int end, float c, int lane)
{
    const int lg = lane >> 4;
    float vscale[G::TB][4];
    if (G::QUANT) {
#pragma unroll
        for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
            for (int i = 0; i < 4; ++i) vscale[tb][i] = scale_value(vs[tb] >> (8 * i) & 0xffu);
    }
    if (masked) {
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
    float alpha[RB];
    bool changed = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float mx = -INFINITY;
#pragma unroll
        for (int tb = 0; tb < G::TB; ++tb)
            mx = fmaxf(mx, fmaxf(fmaxf(s[tb][rb][0], s[tb][rb][1]), fmaxf(s[tb][rb][2], s[tb][rb][3])));
        mx = max_over_groups(mx);
        const float m_new = (mx * c > st.m[rb] + kRescaleLog2) ? mx * c : st.m[rb];
        const float m_use = (m_new == -INFINITY) ? 0.f : m_new;
        alpha[rb] = fast_exp2(st.m[rb] - m_use);
        changed |= (m_new != st.m[rb]);
        st.m[rb] = m_new;
        float sum = 0.f;
#pragma unroll
        for (int tb = 0; tb < G::TB; ++tb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = fast_exp2(fmaf(s[tb][rb][i], c, -m_use));
                sum += p;
                pb[tb / 2][rb][(tb & 1) * 4 + i] = (__bf16)(G::QUANT ? p * vscale[tb][i] : p);
            }
        st.l[rb] = st.l[rb] * alpha[rb] + sum;
    }
    if (__any(changed)) {
#pragma unroll
        for (int db = 0; db < G::DB; ++db)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int i = 0; i < 4; ++i) st.acc[db][rb][i] *= alpha[rb];
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

// O^T[column][row] += sum_token V[token][column] P[row][token].
template <class G, int RB>
__device__ __forceinline__ void pv_tile(WaveState<G, RB>& st, const bf16x8 (&pb)[G::TB / 2][RB], char* vt, int lane)
{
    const int ln = lane & 15, lg = lane >> 4;
#pragma unroll
    for (int kk = 0; kk < G::TB / 2; ++kk)
#pragma unroll
        for (int db = 0; db < G::DB; ++db) {
            bf16x8 va;
            if constexpr (G::QUANT) {
                // eight rows of 16 codes: lane i of a group gives the address of row i / 2, half i % 2, and gets column i
                const int r = ln >> 1, row = kk * 32 + (r >> 2) * 16 + lg * 4 + (r & 3);
                const int c = db ^ v_swz<true, G::ROWB>(row);
                const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                    (i32x2 __attribute__((address_space(3)))*)(vt + row * G::ROWB + c * 16 + (ln & 1) * 8));
                va = eight_values((uint32_t)w[0], (uint32_t)w[1], 1.0f);
            } else {
                s16x4 half[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int row = kk * 32 + h * 16 + lg * 4 + (ln >> 2);
                    const int c = (db * 2) ^ v_swz<false, G::ROWB>(row);
                    half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (s16x4 __attribute__((address_space(3)))*)(vt + row * G::ROWB + c * 16 + (ln & 3) * 8));
                }
                const s16x8 both = __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
                va = __builtin_bit_cast(bf16x8, both);
            }
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
__device__ __forceinline__ void add_not_finite(WaveState<G, RB>& st, const RowAddr& ra, int begin, int end, const int (&lim)[RB], int lane)
{
    const int lg = lane >> 4;
#pragma unroll 1
    for (int t = begin; t < end; ++t) {
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
    }
}

// ---- one piece: tokens [c0, c1) of one (sequence, kv head)
struct Piece {
    RowAddr addr;
    char *kring, *vring, *sring, *qlds;
    int* taken;                                   // teams: the stream's word for take_not_finite
    uint32_t kring_lds, vring_lds, sring_lds;
    int L, Q, R, c0, c1, first, nt, last_tok;     // first, nt: this stream's tiles (tokens c0 + (first + i) TT ..)
    int lane, wave, part, team;
};

// Row blocks row0 / 16 .. of the workgroup, over this wave's stream.
template <class G, int RB, bool PAGED>
__device__ __forceinline__ void run_piece(const StreamLaunch& a, const Piece& w, char* smem, int row0, int64_t pbase)
{
    constexpr int MLS = (G::TEAMS && G::RB1 > G::RB0 ? G::RB1 : G::RB0) * 16;
    const int lane = w.lane, ln = lane & 15, lg = lane >> 4;
    auto tile_t0 = [&](int it) { return w.c0 + (w.first + it) * G::TT; };

    bf16x8 qf[RB][G::KS];
    int lim[RB];                                         // last token that a row attends in this piece
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = row0 + rb * 16 + ln;
        const bool real = row < w.R;
        lim[rb] = min(real ? w.L - w.Q + row / a.G : w.L - 1, w.c1 - 1);
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
        st.m[rb] = -INFINITY;
        st.l[rb] = 0.f;
#pragma unroll
        for (int db = 0; db < G::DB; ++db) st.acc[db][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const float c = a.scale_log2e;
    const int first_masked_t0 = min(w.L - w.Q, w.c1) - (G::TT - 1);     // tiles from here on hold tokens that some row does not attend
    TilePages<G, PAGED> pages;
    bool taken = false;

    // Ring slots of tile `it`, and of the one that takes a slot next.
    int slot = 0;
    auto next = [](int s) { return s + 1 == G::S ? 0 : s + 1; };
    if constexpr (!G::TEAMS) {
        // oldest load first: K(it) V(it) K(it+1) V(it+1) .., the scales ahead of K
        for (int it = 0; it < w.nt; ++it, slot = next(slot)) {
            char* kt = w.kring + slot * G::SLOT;
            char* vt = w.vring + slot * G::SLOT;
            char* sc = w.sring + slot * 256;
            const int t0 = tile_t0(it), t_next = tile_t0(it + G::S);
            floatx4 s[G::TB][RB];
            bf16x8 pb[G::TB / 2][RB];
            uint32_t vs[G::TB];

            pages.find(w.addr, t_next, w.last_tok);
            wait_loads<(2 * G::S - 1) * G::NLD + (G::S - 1) * G::SC>();        // K(it)
            score_tile<G, RB>(s, qf, kt, sc, lane);
            value_scales<G>(vs, sc, lane);
            lds_reads_done();
            load_scales<G, PAGED>(w.addr, pages, w.sring_lds + slot * 256, t_next, w.last_tok, lane);
            load_tile<G, PAGED, false>(w.addr, pages, w.kring_lds + slot * G::SLOT, t_next, w.last_tok, lane, 0, G::NLD);

            softmax_tile<G, RB>(st, s, pb, vs, t0, t0 >= first_masked_t0, lim, w.c1, c, lane);

            wait_loads<(2 * G::S - 1) * G::NLD + G::S * G::SC>();              // V(it)
            if (t0 >= first_masked_t0) taken |= take_not_finite<G>(vt, lane);
            pv_tile<G, RB>(st, pb, vt, lane);
            lds_reads_done();
            load_tile<G, PAGED, true>(w.addr, pages, w.vring_lds + slot * G::SLOT, t_next, w.last_tok, lane, 0, G::NLD);
        }
    } else {
        // Two waves share a stream; each issues half of a tile's loads (both the scales).
        // Barrier A: K(it) is complete, and everybody has done with V(it-1), whose slot V(it+S-1) takes.
        // Barrier B: V(it) is complete, and everybody has done with K(it), whose slot K(it+S) takes.
        constexpr int H = G::NLD / 2, BEHIND = 2 * (G::S - 1) * H + (G::S - 1) * G::SC;
        TilePages<G, PAGED> vpages;
        vpages.find(w.addr, tile_t0(G::S - 1), w.last_tok);
        int before = G::S - 1;                                  // the slot of tile it - 1
        for (int it = 0; it < w.nt; ++it, before = slot, slot = next(slot)) {
            char* kt = w.kring + slot * G::SLOT;
            char* vt = w.vring + slot * G::SLOT;
            char* sc = w.sring + slot * 256;
            const int t0 = tile_t0(it), t_next = tile_t0(it + G::S);
            floatx4 s[G::TB][RB];
            bf16x8 pb[G::TB / 2][RB];
            uint32_t vs[G::TB];

            pages.find(w.addr, t_next, w.last_tok);
            wait_loads<BEHIND>();                               // own half of K(it)
            __syncthreads();                                    // A
            load_tile<G, PAGED, true>(w.addr, vpages, w.vring_lds + before * G::SLOT, t_next - G::TT, w.last_tok, lane, w.team * H, H);
            score_tile<G, RB>(s, qf, kt, sc, lane);
            value_scales<G>(vs, sc, lane);
            softmax_tile<G, RB>(st, s, pb, vs, t0, t0 >= first_masked_t0, lim, w.c1, c, lane);

            wait_loads<BEHIND>();                               // own half of V(it)
            lds_reads_done();
            __syncthreads();                                    // B
            load_scales<G, PAGED>(w.addr, pages, w.sring_lds + slot * 256, t_next, w.last_tok, lane);
            load_tile<G, PAGED, false>(w.addr, pages, w.kring_lds + slot * G::SLOT, t_next, w.last_tok, lane, w.team * H, H);
            if (t0 >= first_masked_t0) taken |= take_not_finite<G>(vt, lane);      // (whoever comes second finds zeros)
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
    if (taken) {
        const int it = max(0, (max(first_masked_t0 - w.c0, 0) + G::TT - 1) / G::TT - w.first);
        add_not_finite<G, RB, PAGED>(st, w.addr, tile_t0(it), min(w.c1, tile_t0(w.nt)), lim, lane);
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
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float mw[G::NP], mm = -INFINITY, ll = 0.f;
#pragma unroll
        for (int p = 0; p < G::NP; ++p) {
            mw[p] = mlbuf[((w.team * G::NP + p) * MLS + rb * 16 + ln) * 2];
            mm = fmaxf(mm, mw[p]);
        }
        const float m_use = (mm == -INFINITY) ? 0.f : mm;
#pragma unroll
        for (int p = 0; p < G::NP; ++p) ll += mlbuf[((w.team * G::NP + p) * MLS + rb * 16 + ln) * 2 + 1] * fast_exp2(mw[p] - m_use);
        own[rb] = fast_exp2(st.m[rb] - m_use);
        const int row = row0 + rb * 16 + ln;
        if (w.part == 0 && lg == 0 && row < w.R) {
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
                *reinterpret_cast<floatx4*>(obuf + (w.part * G::RP + row0 + rb * 16 + ln) * G::OROW + x * 16 + lg * 4) =
                    st.acc[half * (G::DB / G::NH) + x][rb] * own[rb];
        __syncthreads();
        for (int f = threadIdx.x; f < w.R * (DH / 4); f += G::NW * 64) {
            const int row = f / (DH / 4), x = f % (DH / 4) * 4;
            floatx4 sum = *reinterpret_cast<const floatx4*>(obuf + row * G::OROW + x);
#pragma unroll
            for (int p = 1; p < G::NP; ++p) sum += *reinterpret_cast<const floatx4*>(obuf + (p * G::RP + row) * G::OROW + x);
            *reinterpret_cast<floatx4*>(a.part_o + (pbase + row) * G::D + half * DH + x) = sum;
        }
        __syncthreads();                                 // before the buffer is written again, or becomes rings
    }
}

template <class G, bool PAGED>
__device__ __forceinline__ void stream_piece(const StreamLaunch& a, char* smem, int b, int h, int L, int c0, int c1, int64_t pbase)
{
    Piece w;
    const int tid = threadIdx.x;
    w.lane = tid & 63;
    w.wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    w.part = w.wave % G::NP;
    w.team = w.wave / G::NP;
    w.L = L;
    w.Q = seq_queries(a, b);
    w.R = w.Q * a.G;
    w.c0 = c0;
    w.c1 = c1;
    const int ntile = (c1 - c0 + G::TT - 1) / G::TT;
    const int each = (ntile + G::NP - 1) / G::NP;        // tiles of a stream; contiguous
    w.first = w.part * each;
    // teams meet at barriers, so there every stream runs as many tiles; those past its end are masked
    w.nt = G::TEAMS ? each : max(0, min(each, ntile - w.first));
    w.last_tok = min(c1, c0 + (w.first + each) * G::TT) - 1;
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
            const int rr = min(row, last_row);
            const int ch = (w.lane % G::QCPR) ^ k_swz<G::QROWB>(row);
            const uint32_t off = (uint32_t)(((((int64_t)b * a.Qmax + rr / a.G) * a.Hq + h * a.G + rr % a.G) * G::D) * 2) + ch * 16;
            dma16_keep(reinterpret_cast<const char*>(a.q), off, lds + G::NP * G::RING + e * 1024);
        }
    }
    auto tile_t0 = [&](int it) { return c0 + (w.first + it) * G::TT; };
    TilePages<G, PAGED> pages;
    constexpr int H = G::TEAMS ? G::NLD / 2 : G::NLD;
    const int e0 = G::TEAMS ? w.team * H : 0;
    if (w.nt > 0) {
#pragma unroll
        for (int it = 0; it < G::S; ++it) {
            const int t0 = tile_t0(it);
            pages.find(w.addr, t0, w.last_tok);
            load_scales<G, PAGED>(w.addr, pages, w.sring_lds + it * 256, t0, w.last_tok, w.lane);
            load_tile<G, PAGED, false>(w.addr, pages, w.kring_lds + it * G::SLOT, t0, w.last_tok, w.lane, e0, H);
            // (teams: the last V follows barrier A)
            if (!G::TEAMS || it + 1 < G::S) load_tile<G, PAGED, true>(w.addr, pages, w.vring_lds + it * G::SLOT, t0, w.last_tok, w.lane, e0, H);
        }
        wait_loads<(2 * G::S - (G::TEAMS ? 1 : 0)) * H + G::S * G::SC>();
    } else {
        wait_loads<0>();
    }
    __syncthreads();                                     // the whole Q block is in LDS

    if constexpr (!G::TEAMS) {
        run_piece<G, G::RB0, PAGED>(a, w, smem, 0, pbase);
    } else if constexpr (G::RB0 == G::RB1) {
        run_piece<G, G::RB0, PAGED>(a, w, smem, w.team * G::RB0 * 16, pbase);
    } else {
        // the two arms run the same barriers
        if (w.team == 0) run_piece<G, G::RB0, PAGED>(a, w, smem, 0, pbase);
        else run_piece<G, G::RB1, PAGED>(a, w, smem, G::RB0 * 16, pbase);
    }
}

// Grid: one workgroup per (kv head, share).  Partials: [kv head][g + b], which no two pieces of a head share.
template <class G, bool PAGED>
__global__ void __launch_bounds__(G::NW * 64) attn_stream(StreamLaunch a)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int g = __builtin_amdgcn_readfirstlane(blockIdx.x / a.Hkv), x = blockIdx.x % a.Hkv;
    const int h = __builtin_amdgcn_readfirstlane(a.rot ? (x + g) % a.Hkv : x);     // (base addresses go through scalar registers)
    for_each_piece(a, g, threadIdx.x & 63, G::QUANTUM, [&](int b, int L, int c0, int c1) {
        stream_piece<G, PAGED>(a, smem, b, h, L, c0, c1, ((int64_t)h * a.nslots + g + b) * G::RP);
        wait_loads<0>();                                 // the partial's stores are out of the load account
    });
}

// One workgroup of D threads per (sequence, kv head, packed row): out = sum 2^(m_s - M) O_s / sum 2^(m_s - M) l_s, over the row's partials.
template <int D>
__global__ void __launch_bounds__(D) attn_stream_merge(StreamLaunch a)
{
    constexpr int SB = kMergeBlock;
    const int row = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    const int d = threadIdx.x, lane = d & 63;
    const int Q = seq_queries(a, b), R = Q * a.G;
    const int qi = row / a.G, hq = h * a.G + row % a.G;
    uint16_t* dst = a.out + (((int64_t)b * a.Qmax + qi) * a.Hq + hq) * D + d;
    if (row >= R) {                                       // query rows this sequence does not have
        *dst = 0;
        if (a.lse_out && d == 0) a.lse_out[((int64_t)b * a.Hq + hq) * a.Qmax + qi] = 0.f;
        return;
    }
    int before = 0, total = 0, cost = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const int mine = b0 + lane < a.B ? seq_cost(seq_len(a, b0 + lane), a.quantum) : 0;
        const int end = total + scan_costs(mine);
        if (b >= b0 && b < b0 + 64) {
            cost = __builtin_amdgcn_readlane(mine, b - b0);
            before = __builtin_amdgcn_readlane(end, b - b0) - cost;
        }
        total = __builtin_amdgcn_readlane(end, 63);
    }
    int ns = 0;
    int64_t slot = 0;
    if (cost > 0) {
        const Shares sh(total, a.groups);
        const int g0 = sh.owner(before + kPieceQuanta), g1 = sh.owner(before + cost - 1);
        ns = g1 - g0 + 1;
        slot = ((int64_t)h * a.nslots + g0 + b) * a.RP + row;
    }
    RowMerge r;
    float num = 0.f;
    for (int s0 = 0; s0 < ns; s0 += SB) {
        const int nb = min(SB, ns - s0), sl = d & (SB - 1);
        const float* po = a.part_o + (slot + (int64_t)s0 * a.RP) * D + d;
        float o[SB];
#pragma unroll
        for (int j = 0; j < SB; ++j) o[j] = j < nb ? po[(int64_t)j * a.RP * D] : 0.f;
        float ms = -INFINITY, ls = 0.f;
        if (sl < nb) {
            const float* ml = a.part_ml + (slot + (int64_t)(s0 + sl) * a.RP) * 2;
            ms = ml[0];
            ls = ml[1];
        }
        float resc;
        const float w = r.block(ms, ls, &resc);
        float acc0 = 0.f, acc1 = 0.f;
#pragma unroll
        for (int j = 0; j < SB; j += 2) {
            acc0 = fmaf(lane_of(w, j), o[j], acc0);
            acc1 = fmaf(lane_of(w, j + 1), o[j + 1], acc1);
        }
        num = num * resc + (acc0 + acc1);
    }
    const __bf16 o = (__bf16)(r.den == 0.f ? 0.f : num / r.den);
    *dst = __builtin_bit_cast(uint16_t, o);
    if (a.lse_out && d == 0) a.lse_out[((int64_t)b * a.Hq + hq) * a.Qmax + qi] = (r.M + log2f(r.den)) * 0.6931471805599453f;
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
                    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(attn_stream<G, false>),
                                                             hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
                    if (e != hipSuccess) return e;
                    return hipFuncSetAttribute(reinterpret_cast<const void*>(attn_stream<G, true>),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
                });
                if (e != hipSuccess) return e;
            }
    return hipSuccess;
}

void plan_attn_stream(StreamLaunch& a, int n_cu)
{
    const int rb = (a.Qmax * a.G + 15) / 16;
    a.RP = rb * 16;
    a.groups = n_cu > a.Hkv ? n_cu / a.Hkv : 1;          // a workgroup takes a compute unit's LDS
    // no more shares than the longest possible batch has quanta
    (void)with_geo(a.D, a.own.ks != nullptr, rb, [&](auto geo) {
        a.quantum = decltype(geo)::QUANTUM;
        return hipSuccess;
    });
    const int64_t most = (int64_t)a.B * (((int64_t)a.max_ctx + a.quantum - 1) / a.quantum + kPieceQuanta);
    if (a.groups > most) a.groups = (int)most;
    a.nslots = a.groups + a.B - 1;
    // heads whose rows are contiguous are spread over the dies, heads inside a token's row run side by side
    a.rot = a.own.hstride > a.own.tstride && a.Hkv > 1;
}

size_t attn_stream_workspace_bytes(const StreamLaunch& a)
{
    const size_t rows = (size_t)a.Hkv * a.nslots * a.RP;
    return (rows * a.D * 4 + 255) / 256 * 256 + (rows * 8 + 255) / 256 * 256;
}

void bind_attn_stream(StreamLaunch& a, void* workspace)
{
    const size_t rows = (size_t)a.Hkv * a.nslots * a.RP;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + (rows * a.D * 4 + 255) / 256 * 256);
}

hipError_t launch_attn_stream(const StreamLaunch& a, hipStream_t stream)
{
    return with_geo(a.D, a.own.ks != nullptr, a.RP / 16, [&](auto geo) {
        using G = decltype(geo);
        auto fn = a.own.page_table ? attn_stream<G, true> : attn_stream<G, false>;
        hipLaunchKernelGGL(fn, dim3(a.Hkv * a.groups), dim3(G::NW * 64), G::LDS, stream, a);
        return hipGetLastError();
    });
}

hipError_t launch_attn_stream_merge(const StreamLaunch& a, hipStream_t stream)
{
    auto fn = a.D == 128 ? attn_stream_merge<128> : attn_stream_merge<64>;
    hipLaunchKernelGGL(fn, dim3(a.Qmax * a.G, a.Hkv, a.B), dim3(a.D), 0, stream, a);
    return hipGetLastError();
}
