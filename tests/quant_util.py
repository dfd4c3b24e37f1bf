"""What the tests of the quantised cache and of the shared prefix share: the format and the attention in 64 bits (numpy), caches
in the layouts that a caller may use, and the tolerance of an attention result."""
import numpy as np
import torch

POSITIVE = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def e4m3_values(codes: np.ndarray) -> np.ndarray:
    """The numbers that e4m3 codes stand for."""
    mag = codes & 0x7F
    v = np.where(mag == 0x7F, np.nan, POSITIVE[np.minimum(mag, 126)])
    return np.where(codes & 0x80, -v, v)


def e4m3_codes(y: np.ndarray) -> np.ndarray:
    """Nearest codes of finite numbers in [-448, 448], ties to the even code."""
    a = np.abs(y)
    hi = np.clip(np.searchsorted(POSITIVE, a), 0, 126)               # POSITIVE[hi - 1] < a <= POSITIVE[hi]
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - POSITIVE[lo], POSITIVE[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (c | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)


def quantise(x: np.ndarray):
    """Rows (last axis) of float64 values that are bf16 numbers -> (codes uint8 like x, scale bytes)."""
    finite = np.isfinite(x)
    top = np.where(finite, np.abs(x), 0.0).max(-1)
    k = np.full(top.shape, -100)
    m, e = np.frexp(top)                                             # 448 = 0.875 * 2^9
    k = np.where(top > 0, np.clip(e - 9 + (m > 0.875), -100, 119), k)
    with np.errstate(invalid="ignore"):
        y = np.clip(np.ldexp(x, -k[..., None]), -448.0, 448.0)
    codes = e4m3_codes(np.where(finite, y, 0.0))
    return np.where(finite, codes, 0x7F).astype(np.uint8), (k + 127).astype(np.uint8)


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    return np.ldexp(e4m3_values(codes), scales.astype(np.int64)[..., None] - 127)


def bf16(rng, shape, scale=1.0) -> torch.Tensor:
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(torch.bfloat16)


def attention(q, keys, vals, seen, scale):
    """q [n, d], keys and vals [t, d], seen [n, t] (who attends what) -> (out [n, d], lse [n], weight [n, d] = sum of the weights times |v|,
    reach [n] = largest sum |q||k| * scale).  Tokens that a row does not attend have no part in it, whatever they hold."""
    n, d = q.shape
    out, lse, weight = np.zeros((n, d)), np.full(n, -np.inf), np.zeros((n, d))
    reach = np.zeros(n)
    for i in range(n):
        at = np.nonzero(seen[i])[0]
        if not len(at):
            continue
        with np.errstate(invalid="ignore"):
            s = keys[at] @ q[i] * scale
            top = s.max()
            p = np.exp(s - top)
            lse[i] = top + np.log(p.sum())
            p /= p.sum()
            out[i], weight[i] = p @ vals[at], p @ np.abs(vals[at])
            reach[i] = (np.abs(keys[at]) @ np.abs(q[i])).max() * scale
    return out, lse, weight, reach


def tolerance(out, weight, reach, d, tokens):
    """How far a result may be off: the weights and the result are rounded to bf16 (half a step is 2^-8 of the value each); a score is a 32-bit
    sum of d products, times a factor, under an exponential of 32 bits: its error moves a weight by that much relative, numerator and
    denominator; 32-bit sums over the tokens."""
    score = reach[:, None] * (d + 4) * 2.0 ** -24 + 2.0 ** -21
    return (2.0 ** -8 * (1 + 2.0 ** -8) + 2 * score + tokens * 2.0 ** -24) * weight + 2.0 ** -8 * np.abs(out) + 1e-30


def lse_tolerance(lse, reach, d, tokens):
    """A score's error, the sum's, and the rounding of the result and of its two terms."""
    return reach * (d + 4) * 2.0 ** -24 + 2.0 ** -21 + tokens * 2.0 ** -24 + 4 * np.abs(np.where(np.isfinite(lse), lse, 0)) * 2.0 ** -24


def close(got, ref, tol, what=""):
    """Equal where `ref` is not finite, else within `tol`."""
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN in other places"
    inf = ~fine & ~np.isnan(ref)
    assert np.array_equal(got[inf], ref[inf]), f"{what}: other infinities"
    over = np.abs(got - ref)[fine] - np.broadcast_to(tol, ref.shape)[fine]
    assert not over.size or over.max() <= 0, f"{what}: {over.max():.3g} over the tolerance"


def page_table(rng, lens, page, extra=3):
    """(int32 [B, max_pages], pages in the pool): every sequence has pages of its own, in random order; -1 behind them."""
    need = [-(-max(n, 1) // page) for n in lens]
    perm = rng.permutation(sum(need) + extra)
    table = np.full((len(lens), max(need)), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, sum(need) + extra


def laid_out(t: torch.Tensor, layout: str) -> torch.Tensor:
    """The same [rows, tokens, heads, d] in another memory order: heads inside tokens, outside, or rows wider than they need be."""
    if layout == "head":
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "wide":
        r, n, h, d = t.shape
        w = torch.zeros((r, n + 1, h + 1, d + 16), dtype=t.dtype, device=t.device)
        w[:, :n, :h, :d] = t
        return w[:, :n, :h, :d]
    return t.contiguous()


class QuantCache:
    """A cache in 8 bits on the host (numpy) and, through dev(), on the GPU; everything that no token owns holds NaN codes and the
    scale byte 255."""

    def __init__(self, rng, lens, hkv, d, page=0, cap=None, spread=3.0):
        self.lens, self.hkv, self.d, self.page = list(lens), hkv, d, page
        self.cap = cap or max(max(lens), 1)
        B = len(lens)
        self.x = {}
        if page:
            self.table, n = page_table(rng, [self.cap] * B, page)
            rows, tokens, slots = n, page, page
        else:
            self.table, rows, tokens, slots = None, B, self.cap, -(-self.cap // 16) * 16
        self.codes = {n: np.full((rows, tokens, hkv, d), 0x7F, np.uint8) for n in "kv"}
        self.scales = {n: np.full((rows, hkv, slots), 255, np.uint8) for n in "kv"}
        for n in "kv":
            for b, length in enumerate(lens):
                x = bf16(rng, (length, hkv, d)).double().numpy() * 2.0 ** np.round(rng.uniform(-spread, spread, (length, hkv, 1)))
                if n == "k":
                    x = x / 2
                self.put(n, b, np.arange(length), *quantise(x))

    def at(self, b, j):
        if self.table is None:
            return np.full(len(j), b), j
        return self.table[b, j // self.page], j % self.page

    def put(self, n, b, j, codes, scales):
        r, t = self.at(b, j)
        self.codes[n][r, t] = codes
        self.scales[n][r, :, t] = scales

    def tokens(self, n, b, count=None):
        """Values [tokens, hkv, d] of sequence b."""
        r, t = self.at(b, np.arange(self.lens[b] if count is None else count))
        return values(self.codes[n][r, t], self.scales[n][r, :, t])

    def dev(self, layout="token", device="cuda"):
        """(k_codes, v_codes, k_scales, v_scales, page_table or None)"""
        c = [laid_out(torch.from_numpy(self.codes[n]).to(device), layout).view(torch.float8_e4m3fn) for n in "kv"]
        s = [torch.from_numpy(self.scales[n]).to(device).view(torch.float8_e8m0fnu) for n in "kv"]
        return (*c, *s, None if self.table is None else torch.from_numpy(self.table).to(device))


def causal(length, n, rows):
    """seen [rows, length]: row i < n of a sequence attends tokens 0 .. length - n + i."""
    return (np.arange(length)[None, :] <= length - n + np.arange(rows)[:, None]) & (np.arange(rows)[:, None] < n)


def check_attention(q, out, lse, tokens_of, gammas, scale, lens, what=""):
    """Compares out [B, Q, Hq, d] and lse [B, Hq, Q] with the 64-bit attention over tokens_of(b, kv head) = (keys, values, shared), of which
    the first `shared` are attended by every row that there is."""
    B, Q, hq, d = q.shape
    qd = q.double().cpu().numpy()
    out, lse = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    for b in range(B):
        for h in range(hq):
            keys, vals, shared = tokens_of(b, h)
            n = gammas[b] + 1
            seen = causal(lens[b], n, Q)
            seen = np.concatenate([np.broadcast_to((np.arange(Q) < n)[:, None] & (lens[b] > 0), (Q, shared)), seen], 1)
            ref, rl, w, reach = attention(qd[b, :, h], keys, vals, seen, scale)
            name = f"{what} sequence {b} head {h}"
            close(out[b, :, h], ref, tolerance(ref, w, reach, d, keys.shape[0]), name)
            if lse is not None:
                rl[n:] = 0.0
                close(lse[b, h], rl, lse_tolerance(rl, reach, d, keys.shape[0]), name + " lse")
