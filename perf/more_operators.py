"""The drafter's step and prompt: the operators' cases, their plain form and their exact values.

Four operators around a draft:

  rope    the new tokens' queries and keys are rotated by their positions; keys and values go into the cache on the way
          (rapid_kv_append_rope, and rapid_kv_append_rope_quant into a cache in 8 bits)
  window  attention that sees the last `window` tokens and the first `sinks` ones, from one position to a whole prompt
          (rapid_verify_attn_window)
  codes   rows of bf16 values become 8-bit integers with a scale for each row (rapid_quant_rows)
  head    logits of the drafted rows from an output embedding that is kept that way, with the row statistics of the accept
          pass (rapid_lm_head_quant)

A row x of 8-bit integers: code[c] = 127 x[c] / max |x| to the nearest whole number, ties to even; the scale is max |x| / 127 in 32
bits.  Codes are kept in rows of a multiple of 256, zeros behind the last one.

A quantised cache holds, for each token and kv head of K and of V, d codes in e4m3 and one byte E that stands for the
scale 2^(E - 127): the smallest power of two s with max |x| <= 448 s, no smaller than 2^-100 and no larger than 2^119.

Lengths and row counts of a ragged batch are a fixed spread over the case's range, so that work() is a function of the
case alone; all values come from the seed.
"""
from __future__ import annotations

import math

import torch

own = False


def listed():
    return [
        # one round of a served batch: the queries, keys and values of nine positions at most for each of eight sequences, as
        # one projection wrote them, on 16-token pages
        dict(name="rope_step_b8", op="rope", batch=8, hq=32, hkv=8, d=128, rot=128, pairs="half", lo=1024, ctx=4096, rows_lo=5,
             rows=9, page=16, layout="token", bits=16, fused=True, jump=False),
        # a whole 64K-token prompt of one layer
        dict(name="rope_prompt_64k", op="rope", batch=1, hq=32, hkv=8, d=128, rot=128, pairs="half", lo=65536, ctx=65536,
             rows_lo=65536, rows=65536, page=0, layout="head", bits=16, fused=True, jump=False),
        # retrieved chunks that keep the positions of their document, into a cache in 8 bits; half of a head is rotated, in
        # adjacent pairs
        dict(name="rope_chunks_8bit_b4", op="rope", batch=4, hq=16, hkv=8, d=64, rot=32, pairs="adjacent", lo=2000, ctx=5001,
             rows_lo=300, rows=1111, page=16, layout="token", bits=8, fused=False, jump=True),
        # the smallest call: 4 query heads on one kv head of 64, a window of 512 in a 2K-token context; latency and launches
        dict(name="window_512_4h", op="window", batch=1, hq=4, hkv=1, d=64, lo=2048, ctx=2048, rows_lo=5, rows=5, window=512,
             sinks=4, page=0, layout="token", lse=False),
        # a served batch: eight sequences of 16K..128K tokens, 4..8 drafts each, 16-token pages in random order
        dict(name="window_8k_paged_b8", op="window", batch=8, hq=32, hkv=8, d=128, lo=16385, ctx=131071, rows_lo=5, rows=9,
             window=8192, sinks=64, page=16, layout="head", lse=True),
        # pieces of two prompts behind what is cached already, of an odd length
        dict(name="window_4k_piece_b2", op="window", batch=2, hq=28, hkv=4, d=128, lo=9000, ctx=20001, rows_lo=700, rows=1111,
             window=4096, sinks=4, page=16, layout="token", lse=False),
        # a whole 32K-token prompt
        dict(name="window_4k_prompt_32k", op="window", batch=1, hq=32, hkv=8, d=128, lo=32768, ctx=32768, rows_lo=32768,
             rows=32768, window=4096, sinks=64, page=0, layout="head", lse=True),
        # one request's hidden rows of a wide model, as a slice of a larger tensor
        dict(name="codes_77_rows", op="codes", rows=77, hidden=8192, stride=8320),
        # an output embedding, once when it is loaded
        dict(name="codes_128k_rows", op="codes", rows=128256, hidden=4096, stride=4096),
        # the drafter's decode step: one row
        dict(name="head_1_row", op="head", rows=1, hidden=4096, vocab=128256, stats=True),
        # eleven positions of a model whose vocabulary does not fill the chip in whole rounds
        dict(name="head_11_rows_152k", op="head", rows=11, hidden=3584, vocab=152064, stats=False),
        # a served batch of eight
        dict(name="head_72_rows", op="head", rows=72, hidden=4096, vocab=128256, stats=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "rope", "rope", "window", "window", "window", "window", "window", "codes", "head", "head"])
    if op == "codes":
        hidden = 8 * _log_int(rng, 16, 1024)
        return dict(op=op, rows=_log_int(rng, 1, int(5.2e8 // hidden)), hidden=hidden, stride=hidden + 8 * rng.randint(0, 32))
    if op == "head":
        hidden = rng.choice([896, 2048, 2304, 3584, 4096, 5120, 8192, 8 * rng.randint(60, 900)])
        return dict(op=op, rows=rng.randint(1, 96), hidden=hidden, vocab=_log_int(rng, 1000, int(5.4e8 // hidden)),
                    stats=rng.random() < 0.5)
    hq, hkv, d = rng.choice([(4, 1, 64), (32, 8, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128), (16, 8, 64), (24, 3, 128)])
    case = dict(op=op, hq=hq, hkv=hkv, d=d, page=rng.choice([0, 0, 16, 64]), layout=rng.choice(["head", "token"]))
    per_token = 2 * hkv * d
    if op == "rope":
        rows = _log_int(rng, 1, 32768)
        ctx = max(rows, _log_int(rng, 1024, 32768))
        batch = min(_log_int(rng, 1, 16), max(1, int(6.7e7 // (per_token * ctx))), max(1, int(3e8 // (rows * (hq + 2 * hkv) * d))))
        return dict(case, batch=batch, rot=rng.choice([d, d, d // 2, d // 4]), pairs=rng.choice(["half", "half", "adjacent"]),
                    lo=max(rows, ctx // rng.randint(1, 4)), ctx=ctx, rows_lo=rng.randint((rows + 1) // 2, rows), rows=rows,
                    bits=rng.choice([16, 16, 8]), fused=rng.random() < 0.5, jump=rng.random() < 0.3)
    window, sinks = _log_int(rng, 128, 8192), rng.choice([0, 1, 4, 16, 64, rng.randint(1, 300)])
    if rng.random() < 0.6:                           # single tokens and drafts
        rows = rng.randint(1, min(11, 96 // (hq // hkv)))
        ctx = _log_int(rng, 512, 65536)
        batch = min(_log_int(rng, 1, 64), max(1, int(1.1e9 // (per_token * ctx))))
    else:                                            # prompts and pieces of them
        rows = _log_int(rng, 30, 16384)
        ctx = max(rows, _log_int(rng, 512, 32768))
        batch = min(_log_int(rng, 1, 8), max(1, int(5e11 // (4 * rows * hq * d * min(ctx, window + 1024)))),
                    max(1, int(1.1e9 // (per_token * ctx))))
    ragged = batch > 1 and rng.random() < 0.7
    return dict(case, batch=batch, lo=max(rows, ctx // rng.randint(2, 8)) if ragged else ctx, ctx=ctx,
                rows_lo=(rows + 1) // 2 if ragged else rows, rows=rows, window=window, sinks=sinks, lse=rng.random() < 0.5)


# ---------------------------------------------------------------- sizes that follow from a case
def _spread(lo, hi, n):
    """n whole numbers spread over [lo, hi], not sorted; the first one is hi (caches are sized for it)."""
    return [hi if i == 0 else lo + int((hi - lo) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _lens(case):
    return _spread(min(case["lo"], case["ctx"]), case["ctx"], case["batch"])


def _rows(case):
    return _spread(case["rows_lo"], case["rows"], case["batch"])


def _pitch(hidden):
    return -(-hidden // 256) * 256


def _chunk(vocab):
    """Entries of a statistics chunk: whole rounds of 256 workgroups, up to 32 blocks of 16 entries each."""
    blocks = -(-vocab // 16)
    rounds = -(-blocks // (32 * 256))
    return 16 * -(-blocks // (rounds * 256))


def work(case):
    if case["op"] == "codes":                        # rows read in bf16, codes and scales written
        n = case["rows"]
        return {"bytes": n * (2 * case["hidden"] + _pitch(case["hidden"]) + 4), "flops": n * case["hidden"]}
    if case["op"] == "head":                         # codes and scales of the embedding, the rows, the logits
        n, v, k = case["rows"], case["vocab"], case["hidden"]
        return {"bytes": v * (k + 4) + n * (2 * k + 4 * v) + (8 * n * -(-v // _chunk(v)) if case["stats"] else 0),
                "flops": 2 * n * v * k}
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    lens, rows = _lens(case), _rows(case)
    if case["op"] == "rope":                         # all rows read, the queries' and the cache's written
        out = 2 * d if case["bits"] == 16 else d + 1
        return {"bytes": sum(rows) * (hq * 4 * d + 2 * hkv * (2 * d + out)), "flops": 3 * sum(rows) * (hq + hkv) * case["rot"]}
    seen = tokens = 0
    for n, r in zip(lens, rows):
        first = max(0, n - r + 1 - case["window"])                       # of the first row's window
        tokens += n - first + min(case["sinks"], first)
        for p in range(n - r, n):
            low = max(0, p + 1 - case["window"])
            seen += p + 1 - low + min(case["sinks"], low)
    ends = 2 * 2 * sum(rows) * hq * d + (4 * sum(rows) * hq if case["lse"] else 0)
    return {"bytes": tokens * 4 * hkv * d + ends, "flops": 4 * d * hq * seen}


# ---------------------------------------------------------------- inputs
def _randn(g, shape, std=1.0):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=g)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _outside_in(t, layout):
    """[.., tokens, heads, d] views of memory in which heads lie outside tokens ("head") or inside."""
    return t.transpose(1, 2) if layout == "head" else t


def _hidden_rows(g, rows, hidden, stride):
    """Rows as a model leaves them: a few channels are much larger than the others, rows differ in size."""
    x = _randn(g, (rows, stride))
    x *= torch.exp2(torch.rand((rows, 1), device="cuda", generator=g) * 3 - 2).to(torch.bfloat16)
    x[:, torch.randint(0, hidden, (max(1, hidden // 500),), device="cuda", generator=g)] *= 8
    return x[:, :hidden]


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case=case)
    if case["op"] == "codes":
        s["x"] = _hidden_rows(g, case["rows"], case["hidden"], case["stride"])
        return s
    if case["op"] == "head":
        s["h"] = _hidden_rows(g, case["rows"], case["hidden"], case["hidden"])
        w = _randn(g, (case["vocab"], case["hidden"]), 0.03)
        w *= torch.exp2(torch.rand((case["vocab"], 1), device="cuda", generator=g) * 2 - 1).to(torch.bfloat16)
        s["codes"], s["scales"] = _codes(w)
        return s
    B, Q, hq, hkv, d, page = (case[n] for n in ("batch", "rows", "hq", "hkv", "d", "page"))
    lens = _lens(case)
    s.update(lens=_int32(lens), gammas=_int32([r - 1 for r in _rows(case)]), table=None)
    n, tokens = B, case["ctx"]
    if page:
        need = [-(-x // page) for x in lens]
        n, tokens = sum(need) + 3, page                              # a few pages that nobody owns
        perm = torch.randperm(n, device="cuda", generator=g).to(torch.int32)
        s["table"] = torch.full((B, max(need)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, m in enumerate(need):
            s["table"][b, :m] = perm[at:at + m]
            at += m
    shape = (n, hkv, tokens, d) if case["layout"] == "head" else (n, tokens, hkv, d)
    if case["op"] == "window":
        s["k"], s["v"] = (_outside_in(_randn(g, shape, std), case["layout"]) for std in (1.5, 1.0))
        s["q"] = _randn(g, (B, Q, hq, d))
        return s
    # the cache before the call: empty
    if case["bits"] == 16:
        s["k"], s["v"] = (_outside_in(torch.zeros(shape, dtype=torch.bfloat16, device="cuda"), case["layout"]) for _ in "kv")
    else:
        padded = -(-tokens // 16) * 16
        for name in "kv":
            s[name] = _outside_in(torch.zeros(shape, dtype=torch.uint8, device="cuda"), case["layout"]).view(torch.float8_e4m3fn)
            s[name + "s"] = torch.full((n, hkv, padded), 27, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    if case["fused"]:
        s["q_new"], s["k_new"], s["v_new"] = _randn(g, (B, Q, hq + 2 * hkv, d)).split([hq, hkv, hkv], 2)
    else:
        s["q_new"], s["k_new"], s["v_new"] = (_randn(g, (B, Q, h, d)) for h in (hq, hkv, hkv))
    s["freq"] = 500000.0 ** (torch.arange(case["rot"] // 2, dtype=torch.float32, device="cuda") * (-2.0 / case["rot"]))
    s["positions"] = None
    if case["jump"]:                                                 # a chunk's rows follow one another in the document
        s["positions"] = torch.randint(0, 131072, (B, 1), device="cuda", generator=g, dtype=torch.int32) \
            + torch.arange(Q, dtype=torch.int32, device="cuda")
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
    if case["op"] == "codes":
        s["codes"] = torch.empty((case["rows"], _pitch(case["hidden"])), dtype=torch.int8, device="cuda")
        s["scales"] = torch.empty(case["rows"], dtype=torch.float32, device="cuda")
    elif case["op"] == "head":
        s["logits"] = torch.empty((case["rows"], case["vocab"]), dtype=torch.float32, device="cuda")
        chunks = -(-case["vocab"] // _chunk(case["vocab"]))
        s["stats"] = torch.empty((case["rows"], chunks, 2), dtype=torch.float32, device="cuda") if case["stats"] else None
    elif case["op"] == "window":
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((case["batch"], case["hq"], case["rows"]), dtype=torch.float32, device="cuda") if case["lse"] else None
    else:
        s["q_out"] = torch.zeros((case["batch"], case["rows"], case["hq"], case["d"]), dtype=torch.bfloat16, device="cuda")
    return s


# ---------------------------------------------------------------- the plain form
def _codes(x):
    """Codes (int8, rows of a multiple of 256) and scales of the rows of x."""
    x = x.float()
    top = x.abs().amax(1)
    codes = torch.round(127.0 * x / torch.where(top > 0, top, 1.0)[:, None])
    return torch.nn.functional.pad(codes.to(torch.int8), (0, _pitch(x.shape[1]) - x.shape[1])), top / 127.0


def _plain_head(s):
    case = s["case"]
    codes, scales = _codes(s["h"])
    total = codes.float() @ s["codes"].float().t()                   # whole numbers below 2^24 as long as codes are not all alike
    z = s["logits"].copy_(total * scales[:, None] * s["scales"])
    if s["stats"] is not None:
        chunk = _chunk(case["vocab"])
        z = torch.nn.functional.pad(z, (0, -case["vocab"] % chunk), value=-math.inf).view(case["rows"], -1, chunk)
        top = z.amax(-1)
        s["stats"][..., 0] = top
        s["stats"][..., 1] = (z - top[..., None]).exp().sum(-1)


def _power(k):
    """2^k in 32 bits for whole k in [-126, 127], exactly."""
    return ((k.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantised(x):
    """Codes (e4m3) and scale bytes of the rows (last axis) of x."""
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)                                          # top = m 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    k = torch.where(top > 0, e - 9 + (m > 0.875).to(torch.int32), -100).clamp(-100, 119)
    return (x * _power(-k)[..., None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), (k + 127).to(torch.uint8)


def _plain_rope(s):
    case = s["case"]
    n, lens = s["gammas"].long() + 1, s["lens"].long()
    i = torch.arange(case["rows"], device="cuda")[None, :]
    b, i = torch.nonzero(i < n[:, None], as_tuple=True)              # the rows that exist
    token = lens[b] - n[b] + i
    at = token if s["positions"] is None else s["positions"][b, i].long()
    turn = (at.double()[:, None] * s["freq"].double())[:, None, :]   # [rows, 1, rot / 2]
    cos, sin = turn.cos().float(), turn.sin().float()
    rot, half = case["rot"], case["rot"] // 2

    def rotated(x):
        x = x[b, i].float()
        first, second = (x[..., :half], x[..., half:rot]) if case["pairs"] == "half" else (x[..., 0:rot:2], x[..., 1:rot:2])
        first, second = first * cos - second * sin, second * cos + first * sin
        if case["pairs"] == "half":
            x[..., :half], x[..., half:rot] = first, second
        else:
            x[..., 0:rot:2], x[..., 1:rot:2] = first, second
        return x.to(torch.bfloat16)

    s["q_out"][b, i] = rotated(s["q_new"])
    if s["table"] is None:
        x, y = b, token
    else:
        x, y = s["table"][b, token // case["page"]].long(), token % case["page"]
    for name, rows in (("k", rotated(s["k_new"])), ("v", s["v_new"][b, i])):
        if case["bits"] == 16:
            s[name][x, y] = rows
        else:
            codes, scales = _quantised(rows.float())
            s[name].view(torch.uint8)[x, y] = codes.view(torch.uint8)
            s[name + "s"].view(torch.uint8)[x, :, y] = scales


def _plain_window(s):
    """Rows in blocks of neighbours; a block's keys are the sinks and the tokens from its first row's window to its last row."""
    case = s["case"]
    B, Q, hq, hkv, d, window = (case[n] for n in ("batch", "rows", "hq", "hkv", "d", "window"))
    sinks = min(case["sinks"], case["ctx"])
    group, T = hq // hkv, min(Q, 1024)
    blocks, span = -(-Q // T), min(window + T - 1, case["ctx"])
    n, lens = s["gammas"].long() + 1, s["lens"].long()
    i = torch.arange(blocks * T, device="cuda")
    real = (i < n[:, None]).view(B, blocks, T)
    p = ((lens - n)[:, None] + i).view(B, blocks, T)                                        # a row's token
    last = p[:, :, -1:].minimum(lens[:, None, None] - 1)
    far = last - span + 1 + torch.arange(span, device="cuda")                               # [B, blocks, span]
    first = torch.arange(sinks, device="cuda").expand(B, blocks, sinks)
    token = torch.cat([first, far], -1)
    here = token[:, :, None, :]
    seen = torch.cat([first[:, :, None, :] <= p[..., None],
                      (far[:, :, None, :] <= p[..., None]) & (far[:, :, None, :] > (p - window)[..., None])
                      & (far[:, :, None, :] >= sinks)], -1)
    seen &= real[..., None]
    at = token.clamp_min(0).minimum(lens[:, None, None] - 1).clamp_min(0)
    b = torch.arange(B, device="cuda")[:, None, None]
    x, y = (b, at) if s["table"] is None else (s["table"][b, at // case["page"]].long(), at % case["page"])
    k, v = (s[name][x, y].float().permute(0, 1, 3, 2, 4).contiguous() for name in "kv")     # [B, blocks, hkv, tokens, d]
    q = torch.nn.functional.pad(s["q"], (0, 0, 0, 0, 0, blocks * T - Q)).float()
    q = q.view(B, blocks, T, hkv, group, d).permute(0, 1, 3, 2, 4, 5).reshape(B, blocks, hkv, T * group, d)
    score = (q @ k.transpose(-1, -2)).mul_(d ** -0.5).view(B, blocks, hkv, T, group, -1)
    score.masked_fill_(~seen[:, :, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    weight = score.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    out = (weight.view(B, blocks, hkv, T * group, -1) @ v).view(B, blocks, hkv, T, group, d)
    there = real[:, :, None, :, None, None]
    out = torch.where(there, out / total, 0.0).permute(0, 1, 3, 2, 4, 5).reshape(B, blocks * T, hq, d)
    s["out"].copy_(out[:, :Q])
    if s["lse"] is not None:
        lse = torch.where(there, top + total.log(), 0.0)[..., 0]                            # [B, blocks, hkv, T, group]
        s["lse"].copy_(lse.permute(0, 2, 4, 1, 3).reshape(B, hq, blocks * T)[:, :, :Q])


# ---------------------------------------------------------------- one pass
def _results(s):
    op = s["case"]["op"]
    if op == "codes":
        return {"codes": s["codes"], "scales": s["scales"]}
    if op == "head":
        return {"logits": s["logits"], "stats": s["stats"]}
    if op == "window":
        return {"out": s["out"], "lse": s["lse"]}
    return {n: s[n] for n in ("q_out", "k", "v", "ks", "vs") if n in s}


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        if op == "codes":
            codes, scales = _codes(s["x"])
            s["codes"].copy_(codes)
            s["scales"].copy_(scales)
        elif op == "head":
            _plain_head(s)
        elif op == "window":
            _plain_window(s)
        else:
            _plain_rope(s)
        return _results(s)
    r = _handle()
    if op == "codes":
        r.rapid_quant_rows(s["x"], codes=s["codes"], scales=s["scales"])
    elif op == "head":
        r.rapid_lm_head_quant(s["h"], s["codes"], s["scales"], want_stats=case["stats"], logits=s["logits"], stats=s["stats"])
    elif op == "window":
        r.rapid_verify_attn_window(s["q"], s["k"], s["v"], s["lens"], case["window"], sinks=case["sinks"], gammas=s["gammas"],
                                   page_table=s["table"], max_ctx=case["ctx"], out=s["out"], lse_out=s["lse"])
    else:
        more = dict(q_new=s["q_new"], q_out=s["q_out"], positions=s["positions"], interleaved=case["pairs"] == "adjacent",
                    gammas=s["gammas"], page_table=s["table"], max_ctx=case["ctx"])
        if case["bits"] == 16:
            r.rapid_kv_append_rope(s["k"], s["v"], s["k_new"], s["v_new"], s["freq"], s["lens"], **more)
        else:
            r.rapid_kv_append_rope_quant(s["k"], s["v"], s["ks"], s["vs"], s["k_new"], s["v_new"], s["freq"], s["lens"], **more)
    return _results(s)


# ---------------------------------------------------------------- the same in 64 bits
def _exact_codes(x):
    """The whole numbers, in 64 bits, and the scales."""
    x = x.double()
    top = x.abs().max(1, keepdim=True).values
    return torch.round(x * 127.0 / torch.where(top > 0, top, 1.0)), (top / 127.0)[:, 0]


def _exact_power(k):
    """2^k in 64 bits for whole k (given as numbers of 64 bits), by its exponent field: pow() may be off by a last place."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_rows(x):
    """Codes and scales in e4m3 of rows of finite values, as the 64-bit numbers that they stand for."""
    top = x.abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2(top / 448.0)).clamp(-100, 119)         # right but for rounding: two looks put that right
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


def _exact_rope(s):
    case = s["case"]
    lens, rows, rot = _lens(case), _rows(case), case["rot"]
    got = {n: s[n].double() for n in ("k", "v", "ks", "vs") if n in s}
    got["q_out"] = torch.zeros((case["batch"], case["rows"], case["hq"], case["d"]), dtype=torch.float64, device="cuda")
    c = torch.arange(rot // 2, device="cuda")
    left, right = (c, c + rot // 2) if case["pairs"] == "half" else (2 * c, 2 * c + 1)
    for b, (length, n) in enumerate(zip(lens, rows)):
        j = torch.arange(length - n, length, device="cuda")
        at = j.double() if s["positions"] is None else s["positions"][b, :n].double()
        angle = torch.outer(at, s["freq"].double())[:, None, :]
        turn = torch.polar(torch.ones_like(angle), angle)
        x, y = _exact_token(s, b, j)
        for name in ("q_new", "k_new", "v_new"):
            new = s[name][b, :n].double()
            if name != "v_new":
                z = torch.complex(new[..., left], new[..., right]) * turn
                new[..., left], new[..., right] = z.real, z.imag
            if name == "q_new":
                got["q_out"][b, :n] = new
            elif case["bits"] == 16:
                got[name[0]][x, y] = new
            else:                                                    # what is quantised is the row in bf16
                codes, scales = _exact_rows(new.to(torch.bfloat16).double())
                got[name[0]][x, y] = codes
                got[name[0] + "s"][x, :, y] = scales
    return got


def _exact_window(s):
    case = s["case"]
    B, Q, hq, hkv, d, window, sinks = (case[n] for n in ("batch", "rows", "hq", "hkv", "d", "window", "sinks"))
    group = hq // hkv
    out = torch.zeros((B, Q, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, hq, Q), dtype=torch.float64, device="cuda")
    for b, (length, n) in enumerate(zip(_lens(case), _rows(case))):
        for r0 in range(0, n, 512):
            r1 = min(n, r0 + 512)
            p = length - n + torch.arange(r0, r1, device="cuda")[:, None]
            j = torch.arange(length, device="cuda")
            j = j[(j < sinks) | ((j > length - n + r0 - window) & (j < length - n + r1))]
            hidden = (j > p) | ((j <= p - window) & (j >= sinks))
            x, y = _exact_token(s, b, j)
            for h in range(hkv):
                heads = slice(h * group, (h + 1) * group)
                keys, values = s["k"][x, y, h].double(), s["v"][x, y, h].double()
                score = s["q"][b, r0:r1, heads].double().reshape(-1, d) @ keys.t().contiguous() / math.sqrt(d)
                score = score.view(r1 - r0, group, -1).masked_fill_(hidden[:, None, :], -math.inf)
                lse[b, heads, r0:r1] = torch.logsumexp(score, -1).t()
                out[b, r0:r1, heads] = (torch.softmax(score, -1).view(-1, len(j)) @ values).view(r1 - r0, group, d)
    return {"out": out, "lse": lse if case["lse"] else None}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "codes":
        codes, scales = _exact_codes(s["x"])
        pad = _pitch(case["hidden"]) - case["hidden"]
        return {"codes": torch.nn.functional.pad(codes.to(torch.int8), (0, pad)), "scales": scales}
    if case["op"] == "head":
        codes, scales = _exact_codes(s["h"])
        n, vocab, chunk = case["rows"], case["vocab"], _chunk(case["vocab"])
        z = torch.empty((n, vocab), dtype=torch.float64, device="cuda")
        for v0 in range(0, vocab, 16384):
            w = s["codes"][v0:v0 + 16384, :case["hidden"]].double()
            z[:, v0:v0 + 16384] = codes @ w.t().contiguous() * s["scales"][v0:v0 + 16384].double()
        z *= scales[:, None]
        if not case["stats"]:
            return {"logits": z, "stats": None}
        parts = z.split(chunk, 1)
        top = torch.stack([t.max(1).values for t in parts], 1)
        return {"logits": z, "stats": torch.stack([top, torch.stack([torch.logsumexp(t, 1) for t in parts], 1).sub_(top).exp_()], -1)}
    return _exact_window(s) if case["op"] == "window" else _exact_rope(s)
