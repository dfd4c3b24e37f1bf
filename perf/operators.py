"""Attention over a quantised or a shared context: the operators' cases, their plain form and their exact values.

Four operators of the verification step:

  append   the keys and values of new tokens are quantised as they are written into the cache (rapid_kv_append_quant)
  read     rows of such a cache are read back as bf16 (rapid_kv_read_quant)
  attn     attention of the verification positions, or of one decoded position, over such a cache
           (rapid_verify_attn_quant)
  prefix   the same attention over bf16 caches for a batch whose sequences share one long prefix
           (rapid_verify_attn_prefix)

A quantised cache holds, for each token and kv head of K and of V, d codes in e4m3 and one byte E that stands for the
scale 2^(E - 127): the smallest power of two s with max |x| <= 448 s over the finite x of the row, no smaller than
2^-100 and no larger than 2^119.  Non-finite values become NaN.

Lengths and draft counts of a ragged batch are a fixed spread over the case's range, so that work() is a function of the
case alone; all values come from the seed.
"""
from __future__ import annotations

import math

import torch

own = False


def listed():
    return [
        # one validation round of a served batch: nine rows at most for each of eight sequences, on 16-token pages
        dict(name="append_step_b8", op="append", batch=8, hq=32, hkv=8, d=128, lo=1024, ctx=4096, rows_lo=5, rows=9, page=16,
             layout="token"),
        # a whole 64K-token prompt of one layer is written at once
        dict(name="append_prompt_64k", op="append", batch=1, hq=32, hkv=8, d=128, lo=65536, ctx=65536, rows_lo=65536,
             rows=65536, page=0, layout="head"),
        # the tails of a ragged batch are handed to a program that works in bf16
        dict(name="read_tails_b4", op="read", batch=4, hq=16, hkv=8, d=64, lo=2000, ctx=5001, rows_lo=300, rows=1111, page=16,
             layout="token"),
        # a whole 32K-token sequence is read back
        dict(name="read_all_32k", op="read", batch=1, hq=32, hkv=8, d=128, lo=32768, ctx=32768, rows_lo=32768, rows=32768,
             page=0, layout="head"),
        # the smallest call: 4 query heads on one kv head of 64, a 2K-token context; latency and launches
        dict(name="attn_2k_4h", op="attn", batch=1, hq=4, hkv=1, d=64, lo=2048, ctx=2048, rows_lo=5, rows=5, page=0,
             layout="token", lse=False),
        # the drafter's decode step: one position on a retrieved 8K context
        dict(name="attn_decode_8k", op="attn", batch=1, hq=32, hkv=8, d=128, lo=8192, ctx=8192, rows_lo=1, rows=1, page=0,
             layout="head", lse=False),
        # the headline configuration's layer: nine positions of 32 heads over 128K tokens
        dict(name="attn_128k", op="attn", batch=1, hq=32, hkv=8, d=128, lo=131072, ctx=131072, rows_lo=9, rows=9, page=0,
             layout="head", lse=False),
        # a served batch: eight sequences of 16K..128K tokens, 4..8 drafts each, 16-token pages in random order
        dict(name="attn_paged_ragged_b8", op="attn", batch=8, hq=32, hkv=8, d=128, lo=16385, ctx=131071, rows_lo=5, rows=9,
             page=16, layout="head", lse=True),
        # 72 packed query rows per kv head
        dict(name="attn_128k_72rows", op="attn", batch=1, hq=64, hkv=8, d=128, lo=131072, ctx=131072, rows_lo=9, rows=9,
             page=0, layout="head", lse=False),
        # four requests about one short document, one position each
        dict(name="prefix_2k_b4_decode", op="prefix", batch=4, hq=32, hkv=8, d=128, prefix=2048, lo=33, ctx=300, rows_lo=1,
             rows=1, page=0, layout="head", lse=False),
        # eight requests about one 32K-token document, up to eight drafts each
        dict(name="prefix_32k_b8", op="prefix", batch=8, hq=32, hkv=8, d=128, prefix=32768, lo=200, ctx=1500, rows_lo=5,
             rows=9, page=0, layout="token", lse=True),
        # sixteen requests about one 128K-token document on a paged pool
        dict(name="prefix_128k_b16_paged", op="prefix", batch=16, hq=32, hkv=8, d=128, prefix=131000, lo=100, ctx=2100,
             rows_lo=3, rows=5, page=16, layout="token", lse=False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "append", "read", "read", "attn", "attn", "attn", "attn", "prefix", "prefix", "prefix"])
    hq, hkv, d = rng.choice([(4, 1, 64), (32, 8, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128), (16, 8, 64), (24, 3, 128)])
    case = dict(op=op, hq=hq, hkv=hkv, d=d, page=rng.choice([0, 0, 16, 64]), layout=rng.choice(["head", "token"]))
    per_token = 2 * hkv * d
    if op in ("append", "read"):
        rows = _log_int(rng, 1, 32768)
        ctx = max(rows, _log_int(rng, 1024, 32768))
        batch = min(_log_int(rng, 1, 16), max(1, int(6.7e7 // (per_token * ctx))))
        return dict(case, batch=batch, lo=max(rows, ctx // rng.randint(1, 4)), ctx=ctx, rows_lo=rng.randint((rows + 1) // 2, rows),
                    rows=rows)
    rows = rng.randint(1, min(11, 96 // (hq // hkv)))
    if op == "attn":
        ctx = _log_int(rng, 512, 131072)
        batch = min(_log_int(rng, 1, 32), max(1, int(1.1e9 // (per_token * ctx))), max(1, int(1.2e11 // (4 * rows * hq * d * ctx))))
        ragged = batch > 1 and rng.random() < 0.7
        return dict(case, batch=batch, lo=max(256, ctx // rng.randint(2, 8)) if ragged else ctx, ctx=ctx,
                    rows_lo=(rows + 1) // 2 if ragged else rows, rows=rows, lse=rng.random() < 0.5)
    prefix = _log_int(rng, 1024, 131072)
    batch = min(_log_int(rng, 2, 32), max(2, int(1.68e8 // (rows * hq * prefix))))
    ctx = max(rows, _log_int(rng, 32, 2100))
    return dict(case, batch=batch, prefix=prefix, lo=max(rows, ctx // rng.randint(1, 8)), ctx=ctx,
                rows_lo=(rows + 1) // 2, rows=rows, lse=rng.random() < 0.5)


# ---------------------------------------------------------------- sizes that follow from a case
def _spread(lo, hi, n):
    """n whole numbers spread over [lo, hi], not sorted; the first one is hi (caches are sized for it)."""
    return [hi if i == 0 else lo + int((hi - lo) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _lens(case):
    return _spread(min(case["lo"], case["ctx"]), case["ctx"], case["batch"])


def _rows(case):
    return _spread(case["rows_lo"], case["rows"], case["batch"])


def work(case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    lens, rows = _lens(case), _rows(case)
    if case["op"] == "append":                       # rows read in bf16, codes and scales written; a multiplication a value
        n = 2 * sum(rows) * hkv
        return {"bytes": n * (2 * d + d + 1), "flops": n * d}
    if case["op"] == "read":                         # codes and scales read, every row of the outputs written
        n = 2 * hkv
        return {"bytes": n * (sum(rows) * (d + 1) + case["batch"] * case["rows"] * 2 * d), "flops": n * sum(rows) * d}
    ends = 2 * 2 * case["batch"] * case["rows"] * hq * d + (4 * case["batch"] * case["rows"] * hq if case["lse"] else 0)
    before = case["prefix"] if case["op"] == "prefix" else 0
    pairs = sum(r * (before + n - r) + r * (r + 1) // 2 for r, n in zip(rows, lens))
    token = 2 * hkv * (2 * d if case["op"] == "prefix" else d + 1)
    return {"bytes": (before + sum(lens)) * token + ends, "flops": 4 * d * hq * pairs}


# ---------------------------------------------------------------- inputs
def _randn(g, shape, std=1.0):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=g)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _outside_in(t, layout):
    """[.., tokens, heads, d] views of memory in which heads lie outside tokens ("head") or inside."""
    return t.transpose(1, 2) if layout == "head" else t


def _cache(case, g, std):
    """A bf16 cache [rows, tokens, hkv, d] in the case's memory order: contiguous sequences, or a pool of pages."""
    n, tokens = (case["pool"], case["page"]) if case["page"] else (case["batch"], case["ctx"])
    shape = (n, case["hkv"], tokens, case["d"]) if case["layout"] == "head" else (n, tokens, case["hkv"], case["d"])
    return _outside_in(_randn(g, shape, std), case["layout"])


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case=case)
    lens, rows, page = _lens(case), _rows(case), case["page"]
    s.update(lens=_int32(lens), gammas=_int32([r - 1 for r in rows]), table=None, prefix_table=None, k_prefix=None,
             v_prefix=None)
    prefix = case["prefix"] if case["op"] == "prefix" else 0
    if page:
        need, shared = [-(-n // page) for n in lens], -(-prefix // page)
        pool = sum(need) + shared + 3                            # a few pages that nobody owns
        perm = torch.randperm(pool, device="cuda", generator=g).to(torch.int32)
        s["table"] = torch.full((case["batch"], max(need)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(need):
            s["table"][b, :n] = perm[at:at + n]
            at += n
        if prefix:
            s["prefix_table"] = perm[at:at + shared].contiguous()
        case = dict(case, pool=pool)
    if case["op"] == "prefix":
        s["k"], s["v"] = _cache(case, g, 1.5), _cache(case, g, 1.0)
        s["prefix_len"] = _int32([prefix])
        if not page:
            one = dict(case, batch=1, ctx=prefix)
            s["k_prefix"], s["v_prefix"] = _cache(one, g, 1.5)[0], _cache(one, g, 1.0)[0]
    else:
        # rows of a model differ in size from token to token and head to head: a spread over three powers of two
        for name, std in (("k", 1.5), ("v", 1.0)):
            x = _cache(case, g, std)
            x = x * torch.exp2(torch.rand(x.shape[:3], device="cuda", generator=g) * 3 - 2)[..., None].to(torch.bfloat16)
            codes, scales = _quantised(x)
            codes = codes.view(torch.uint8)
            if case["layout"] == "head":
                codes = codes.transpose(1, 2).contiguous().transpose(1, 2)
            # scales [rows, heads, tokens], in rows of a multiple of 16 bytes
            padded = torch.zeros((*scales.shape[:1], case["hkv"], -(-scales.shape[1] // 16) * 16), dtype=torch.uint8, device="cuda")
            padded[:, :, :scales.shape[1]] = scales.transpose(1, 2)
            s[name], s[name + "s"] = codes.view(torch.float8_e4m3fn), padded.view(torch.float8_e8m0fnu)
    B, Q = case["batch"], case["rows"]
    if case["op"] == "append":
        s["k_new"], s["v_new"] = (_randn(g, (B, Q, case["hkv"], case["d"]), std) for std in (1.5, 1.0))
    if case["op"] in ("attn", "prefix"):
        s["q"] = _randn(g, (B, Q, case["hq"], case["d"]))
    return s


_shared = []


def _handle():
    """The one library handle a program keeps per GPU."""
    if not _shared:
        from paper_2502_20330_amd import binding
        _shared.append(binding.Rapid(0))
    return _shared[0]


def prepare(case, seed):
    s = _inputs(case, seed)
    B, Q, hq, hkv, d = case["batch"], case["rows"], case["hq"], case["hkv"], case["d"]
    if case["op"] == "read":
        s["outs"] = tuple(torch.empty((B, Q, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if case["op"] in ("attn", "prefix"):
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((B, hq, Q), dtype=torch.float32, device="cuda") if case["lse"] else None
    return s


# ---------------------------------------------------------------- the plain form
def _power(k):
    """2^k in 32 bits for whole k in [-126, 127], exactly."""
    return ((k.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantised(x):
    """Codes (e4m3) and scale bytes of the rows (last axis) of x."""
    x = x.float()
    finite = torch.isfinite(x)
    top = torch.where(finite, x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(top)                                      # top = m 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    k = torch.where(top > 0, e - 9 + (m > 0.875).to(torch.int32), -100).clamp(-100, 119)
    y = (x * _power(-k)[..., None]).clamp(-448.0, 448.0)
    return torch.where(finite, y, math.nan).to(torch.float8_e4m3fn), (k + 127).to(torch.uint8)


def _values(s, name):
    """The values in 32 bits that the cache `name` stands for, [rows, tokens, heads, d]."""
    codes = s[name].float()
    return codes * s[name + "s"].float().transpose(1, 2)[:, :codes.shape[1], :, None]


def _own_tokens(s, x):
    """The sequences' own tokens [B, longest, heads, d] of a cache; what lies past a sequence's end is anything."""
    if s["table"] is None:
        return x
    t = x[s["table"].clamp_min(0).long()]
    return t.reshape(t.shape[0], -1, *t.shape[3:])[:, :s["case"]["ctx"]]


def _places(s):
    """For the new rows that exist: their sequence, their row, and the two indices of their token in the cache."""
    n = s["gammas"].long() + 1
    i = torch.arange(s["case"]["rows"], device="cuda")[None, :]
    b, i = torch.nonzero(i < n[:, None], as_tuple=True)
    token = s["lens"].long()[b] - n[b] + i
    if s["table"] is None:
        return b, i, b, token
    page = s["case"]["page"]
    return b, i, s["table"][b, token // page].long(), token % page


def _plain_append(s):
    b, i, x, y = _places(s)
    for name in ("k", "v"):
        codes, scales = _quantised(s[name + "_new"][b, i])
        s[name].view(torch.uint8)[x, y] = codes.view(torch.uint8)
        s[name + "s"].view(torch.uint8)[x, :, y] = scales


def _plain_read(s):
    b, i, x, y = _places(s)
    for name, out in zip(("k", "v"), s["outs"]):
        out.zero_()
        codes, scales = s[name].view(torch.uint8)[x, y], s[name + "s"].view(torch.uint8)[x, :, y]
        out[b, i] = (codes.view(torch.float8_e4m3fn).float() * _power(scales.int() - 127)[..., None]).to(torch.bfloat16)


def _plain_attn(s, k, v, prefix):
    """Softmax attention in 32 bits over the own tokens k, v [B, L, hkv, d], behind the shared ones [P, hkv, d] or none."""
    case = s["case"]
    B, Q, hq, hkv, d = case["batch"], case["rows"], case["hq"], case["hkv"], case["d"]
    group, L = hq // hkv, k.shape[1]
    n, lens = s["gammas"].long() + 1, s["lens"].long()
    i = torch.arange(Q, device="cuda")
    real = i[None, :] < n[:, None]                                                          # [B, Q]
    seen = torch.arange(L, device="cuda") <= (lens - n)[:, None, None] + i[None, :, None]   # [B, Q, L]
    seen &= real[:, :, None]
    # values past a sequence's end are anything: zeros there
    inside = (torch.arange(L, device="cuda") < lens[:, None])[:, :, None, None]
    v = torch.where(inside, v, 0.0).transpose(1, 2)                                         # [B, hkv, L, d]
    q = s["q"].float().view(B, Q, hkv, group, d).permute(0, 2, 1, 3, 4)                     # [B, hkv, Q, group, d]
    score = (q.reshape(B, hkv, Q * group, d) @ k.transpose(1, 2).transpose(2, 3)).mul_(d ** -0.5).view(B, hkv, Q, group, L)
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    if prefix is not None:
        kp, vp = (t.float().transpose(0, 1) for t in prefix)                                # [hkv, P, d]
        shared = q.transpose(0, 1).reshape(hkv, B * Q * group, d) @ kp.transpose(1, 2)
        shared = shared.mul_(d ** -0.5).view(hkv, B, Q, group, -1).transpose(0, 1)          # [B, hkv, Q, group, P]
        top = torch.maximum(top, shared.amax(-1, keepdim=True))
    top = torch.where(torch.isfinite(top), top, 0.0)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(B, hkv, Q * group, L) @ v).view(B, hkv, Q, group, d)
    if prefix is not None:
        p = shared.sub_(top).exp_()
        total = total + p.sum(-1, keepdim=True)
        o = o + (p.transpose(0, 1).reshape(hkv, B * Q * group, -1) @ vp).view(hkv, B, Q, group, d).transpose(0, 1)
    there = real[:, None, :, None, None]
    o = torch.where(there, o / total, 0.0).permute(0, 2, 1, 3, 4).reshape(B, Q, hq, d)
    s["out"].copy_(o)
    if s["lse"] is not None:
        lse = torch.where(there, top + total.log(), 0.0)[..., 0]                            # [B, hkv, Q, group]
        s["lse"].copy_(lse.permute(0, 1, 3, 2).reshape(B, hq, Q))


def _prefix_tokens(s):
    if s["prefix_table"] is None:
        return s["k_prefix"], s["v_prefix"]
    at = s["prefix_table"].long()
    return tuple(s[n][at].reshape(-1, *s[n].shape[2:])[:s["case"]["prefix"]] for n in ("k", "v"))


# ---------------------------------------------------------------- one pass
def _results(s):
    op = s["case"]["op"]
    if op == "append":
        return {n: s[n] for n in ("k", "v", "ks", "vs")}
    if op == "read":
        return {"k": s["outs"][0], "v": s["outs"][1]}
    return {"out": s["out"], "lse": s["lse"]}


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        if op == "append":
            _plain_append(s)
        elif op == "read":
            _plain_read(s)
        elif op == "attn":
            _plain_attn(s, _own_tokens(s, _values(s, "k")), _own_tokens(s, _values(s, "v")), None)
        else:
            _plain_attn(s, _own_tokens(s, s["k"]).float(), _own_tokens(s, s["v"]).float(), _prefix_tokens(s))
        return _results(s)
    r = _handle()
    more = dict(gammas=s["gammas"], page_table=s["table"], max_ctx=case["ctx"])
    if op == "append":
        r.rapid_kv_append_quant(s["k"], s["v"], s["ks"], s["vs"], s["k_new"], s["v_new"], s["lens"], **more)
    elif op == "read":
        r.rapid_kv_read_quant(s["k"], s["v"], s["ks"], s["vs"], s["lens"], case["rows"], outs=s["outs"], **more)
    elif op == "attn":
        r.rapid_verify_attn_quant(s["q"], s["k"], s["v"], s["ks"], s["vs"], s["lens"], out=s["out"], lse_out=s["lse"], **more)
    else:
        r.rapid_verify_attn_prefix(s["q"], s["k"], s["v"], s["lens"], s["prefix_len"], k_prefix=s["k_prefix"],
                                   v_prefix=s["v_prefix"], prefix_table=s["prefix_table"], max_prefix=case["prefix"],
                                   out=s["out"], lse_out=s["lse"], **more)
    return _results(s)


# ---------------------------------------------------------------- the same in 64 bits
def _exact_power(k):
    """2^k in 64 bits for whole k (given as numbers of 64 bits), by its exponent field: pow() may be off by a last place."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_rows(x):
    """Codes and scales of rows of finite values, as the 64-bit numbers that they stand for."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2(top / 448.0)).clamp(-100, 119)     # right but for rounding: two looks put that right
    k = torch.where(top <= 448.0 * _exact_power(k - 1), k - 1, k)
    k = torch.where(top > 448.0 * _exact_power(k), k + 1, k).clamp(-100, 119)
    scale = _exact_power(k)
    y = x / scale
    # four significant bits, the last place no finer than 2^-9; round() takes ties to even
    step = _exact_power(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return (torch.round(y / step) * step).clamp(-448.0, 448.0), scale[..., 0]


def _exact_token(s, b, j):
    """Where token j (a tensor) of sequence b lies."""
    if s["table"] is None:
        return torch.full_like(j, b), j
    return s["table"][b].long()[j // s["case"]["page"]], j % s["case"]["page"]


def exact(case, seed):
    s = _inputs(case, seed)
    lens, rows, hkv, d = _lens(case), _rows(case), case["hkv"], case["d"]
    if case["op"] == "append":
        got = {n: s[n].double() for n in ("k", "v", "ks", "vs")}
        for b, (length, n) in enumerate(zip(lens, rows)):
            x, y = _exact_token(s, b, torch.arange(length - n, length, device="cuda"))
            for name in ("k", "v"):
                codes, scales = _exact_rows(s[name + "_new"][b, :n])
                got[name][x, y] = codes
                got[name + "s"][x, :, y] = scales
        return got
    if case["op"] == "read":
        got = {n: torch.zeros((case["batch"], case["rows"], hkv, d), dtype=torch.float64, device="cuda") for n in ("k", "v")}
        for b, (length, n) in enumerate(zip(lens, rows)):
            x, y = _exact_token(s, b, torch.arange(length - n, length, device="cuda"))
            for name in ("k", "v"):
                codes, scales = (s[t].view(torch.uint8) for t in (name, name + "s"))
                got[name][b, :n] = (codes[x, y].view(torch.float8_e4m3fn).double()
                                    * scales[x, :, y].view(torch.float8_e8m0fnu).double()[..., None])
        return got
    B, Q, hq = case["batch"], case["rows"], case["hq"]
    out = torch.zeros((B, Q, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, hq, Q), dtype=torch.float64, device="cuda")
    for b, (length, n) in enumerate(zip(lens, rows)):
        x, y = _exact_token(s, b, torch.arange(length, device="cuda"))
        before = case["prefix"] if case["op"] == "prefix" else 0
        for h in range(hkv):
            keys, values = [], []
            for name, parts in (("k", keys), ("v", values)):
                if case["op"] == "attn":
                    scale = s[name + "s"].view(torch.uint8)[x, h, y].view(torch.float8_e8m0fnu).double()
                    parts.append(s[name].view(torch.uint8)[x, y, h].view(torch.float8_e4m3fn).double() * scale[:, None])
                    continue
                if s["prefix_table"] is None:
                    parts.append(s[name + "_prefix"][:, h].double())
                else:
                    at = torch.arange(before, device="cuda")
                    parts.append(s[name][s["prefix_table"].long()[at // case["page"]], at % case["page"], h].double())
                parts.append(s[name][x, y, h].double())
            keys, values = torch.cat(keys), torch.cat(values)
            last = before + length - n + torch.arange(n, device="cuda")
            heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            score = s["q"][b, :n, heads].double().reshape(-1, d) @ keys.t().contiguous() / math.sqrt(d)
            score = score.view(n, hq // hkv, -1)
            score.masked_fill_((torch.arange(before + length, device="cuda")[None, :] > last[:, None])[:, None, :], -math.inf)
            lse[b, heads, :n] = torch.logsumexp(score, -1).t()
            weight = torch.softmax(score, -1)
            out[b, :n, heads] = (weight.view(-1, before + length) @ values).view(n, hq // hkv, d)
    return {"out": out, "lse": lse if case["lse"] else None}
