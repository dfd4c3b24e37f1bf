"""rapid_verify_attn_window: every row tile of both kernels, in one share and in several, against the attention in 64 bits; and tokens that are not finite, row by row."""
import ctypes

import numpy as np
import pytest
import torch

import quant_util as qu
from paper_2502_20330_amd import binding
from test_gpu_window import i32, seen_by

# (many rows, row tile, one row tile a sequence, one share) and sequences, positions, query heads, kv heads, window of a call that is divided so, on 256 compute
# units and with heads of 64 and of 128
PLANS = {
    (0, 16, 1, 1): (1, 1, 2, 1, 40), (0, 16, 1, 0): (1, 1, 2, 1, 600), (0, 16, 0, 1): (1, 3, 6, 1, 40), (0, 16, 0, 0): (1, 3, 6, 1, 600),
    (0, 32, 1, 1): (24, 3, 48, 8, 40), (0, 32, 1, 0): (24, 3, 12, 2, 2000), (0, 32, 0, 1): (3, 200, 7, 1, 40), (0, 32, 0, 0): (1, 200, 7, 1, 3000),
    (0, 48, 1, 1): (24, 3, 96, 8, 40), (0, 48, 1, 0): (5, 3, 36, 3, 6000), (0, 48, 0, 1): (5, 170, 10, 1, 40), (0, 48, 0, 0): (1, 300, 7, 1, 4000),
    (0, 64, 1, 1): (24, 5, 80, 8, 40), (0, 64, 1, 0): (12, 5, 30, 3, 4000),
    (0, 80, 1, 1): (24, 11, 48, 8, 40), (0, 80, 1, 0): (6, 11, 18, 3, 4000),
    (0, 96, 1, 1): (24, 7, 96, 8, 40), (0, 96, 1, 0): (6, 7, 36, 3, 4000), (0, 96, 0, 1): (6, 170, 12, 1, 40), (0, 96, 0, 0): (3, 130, 10, 1, 8000),
    (1, 128, 1, 1): (24, 10, 80, 8, 40), (1, 128, 1, 0): (6, 10, 30, 3, 6000), (1, 128, 0, 1): (32, 20, 30, 3, 40), (1, 128, 0, 0): (3, 170, 12, 1, 3000),
    (1, 192, 1, 1): (24, 11, 96, 8, 40), (1, 192, 1, 0): (24, 23, 14, 2, 4000), (1, 192, 0, 1): (32, 37, 21, 3, 40), (1, 192, 0, 0): (3, 300, 10, 1, 6000),
    (1, 256, 1, 1): (24, 20, 80, 8, 40), (1, 256, 1, 0): (24, 32, 16, 2, 4000), (1, 256, 0, 1): (32, 53, 24, 3, 40), (1, 256, 0, 0): (3, 600, 7, 1, 4000),
    (1, 320, 1, 1): (24, 37, 56, 8, 40), (1, 320, 1, 0): (24, 37, 14, 2, 4000), (1, 320, 0, 1): (32, 53, 30, 3, 40), (1, 320, 0, 0): (4, 600, 7, 1, 6000),
    (1, 384, 1, 1): (24, 27, 96, 8, 40), (1, 384, 1, 0): (24, 27, 24, 2, 6000), (1, 384, 0, 1): (32, 100, 21, 3, 40), (1, 384, 0, 0): (12, 260, 10, 1, 8000),
}
SINKS = 5
DEVICE = "cuda"


def cap_of(Q, window):
    """Tokens enough for a gap between the sinks and the windows."""
    return Q + window + 150


def plan_of(context, d, B, Q, hq, hkv, window):
    cap = cap_of(Q, window)
    s = binding.AttnShape(B, Q, hq, hkv, d, cap, Q - 1, d ** -0.5, cap * hkv * d, hkv * d, d, 0, 0, 0, 0, 0, 0)
    plan = (ctypes.c_int32 * 3)()
    assert binding.load_library().rapid_verify_attn_window_plan(context, ctypes.byref(s), window, SINKS, plan) == 0
    tile, shares, many = plan
    return many, tile, int(Q * hq // hkv <= tile), int(shares == 1)


@pytest.mark.parametrize("d", [64, 128])
def test_the_shapes_are_divided_as_they_are_meant_to_be(d):
    """All tiles there are: of the streaming kernel in one and (but for 64 and 80 rows, which only calls of so few rows take) in several, of the kernel of many rows
    likewise, each with its tokens in one share and in several."""
    assert {k: plan_of(None, d, *shape) for k, shape in PLANS.items()} == {k: k for k in PLANS}
    few = {(0, t, one, direct) for t in range(16, 97, 16) for one in (0, 1) for direct in (0, 1) if one or t not in (64, 80)}
    assert set(PLANS) == few | {(1, t, one, direct) for t in range(128, 385, 64) for one in (0, 1) for direct in (0, 1)}


def test_the_plan_is_refused_like_the_call():
    lib, plan = binding.load_library(), (ctypes.c_int32 * 3)()
    s = binding.AttnShape(1, 5, 8, 2, 128, 1000, 4, 0.1, 256000, 256, 128, 0, 0, 0, 0, 0, 0)
    assert lib.rapid_verify_attn_window_plan(None, ctypes.byref(s), 100, 4, plan) == 0
    for args in ((ctypes.byref(s), 100, 4, None), (ctypes.byref(s), 0, 4, plan), (ctypes.byref(s), 100, -1, plan), (None, 100, 4, plan)):
        assert lib.rapid_verify_attn_window_plan(None, *args) == binding.RAPID_EINVAL
    s.head_dim = 96
    assert lib.rapid_verify_attn_window_plan(None, ctypes.byref(s), 100, 4, plan) == binding.RAPID_EUNSUPPORTED


def attention(q, keys, vals, seen, scale):
    """quant_util's attention in 64 bits, on tensors: (out, lse, weight, reach) as arrays.  Every token is attended by one of the rows at least."""
    n, d = q.shape
    if not keys.shape[0]:
        return np.zeros((n, d)), np.full(n, -np.inf), np.zeros((n, d)), np.zeros(n)
    s = torch.where(seen, q @ keys.T * scale, -torch.inf)
    reach = torch.where(seen, q.abs() @ keys.abs().T * scale, 0.0).amax(1)
    lse = torch.logsumexp(s, 1)
    p = torch.where(seen, torch.exp(s - lse[:, None]), 0.0)
    return tuple(x.cpu().numpy() for x in (p @ vals, lse, p @ vals.abs(), reach))


class Call:
    """A batch on the GPU whose cache holds NaN wherever nobody attends: a full sequence with as many rows as there may be, then shorter ones with fewer, one of them shorter
    than its rows and one empty where there are enough."""

    def __init__(self, d, B, Q, hq, hkv, window, page, layout):
        g = torch.Generator(device=DEVICE).manual_seed(Q * hq + d + page)
        rng = np.random.default_rng(Q * hq + d + page)
        self.d, self.B, self.Q, self.hq, self.hkv, self.window, self.page, self.layout = d, B, Q, hq, hkv, window, page, layout
        self.cap = cap_of(Q, window)
        self.gammas = [Q - 1 - (b * 7) % Q for b in range(B)]
        self.lens = [self.cap - (b * 97) % (self.cap // 2) for b in range(B)]
        if B > 2:
            self.lens[1], self.gammas[1] = max(Q // 2, 1), Q - 1
            self.lens[2] = 0
        self.q = torch.randn((B, Q, hq, d), generator=g, device=DEVICE).bfloat16()
        self.x = {n: torch.randn((B, self.cap, hkv, d), generator=g, device=DEVICE).bfloat16() for n in "kv"}
        self.seen = [seen_by(n, m + 1, Q, window, SINKS) for n, m in zip(self.lens, self.gammas)]
        for b, seen in enumerate(self.seen):
            nobody = np.ones(self.cap, bool)
            nobody[:seen.shape[1]] = ~seen.any(0)
            for n in "kv":
                self.x[n][b, torch.from_numpy(nobody).to(DEVICE)] = torch.nan
        self.table = None
        if page:
            table, self.pages = qu.page_table(rng, [self.cap] * B, page)
            self.table = torch.from_numpy(table).to(DEVICE)

    def cache(self, n):
        if not self.page:
            return qu.laid_out(self.x[n], self.layout)
        full = self.table.shape[1] * self.page
        x = torch.full((self.B, full, self.hkv, self.d), torch.nan, dtype=torch.bfloat16, device=DEVICE)
        x[:, :self.cap] = self.x[n]
        pool = torch.full((self.pages, self.page, self.hkv, self.d), torch.nan, dtype=torch.bfloat16, device=DEVICE)
        pool[self.table.long().flatten()] = x.reshape(-1, self.page, self.hkv, self.d)
        return qu.laid_out(pool, self.layout)

    def run(self):
        lse = torch.full((self.B, self.hq, self.Q), 7.0, device=DEVICE)
        out = binding_call(self.q, self.cache("k"), self.cache("v"), i32(self.lens), self.window, sinks=SINKS, gammas=i32(self.gammas), page_table=self.table,
                           max_ctx=self.cap, lse_out=lse)
        return out, lse

    def places(self):
        """Sequences, heads and rows that are compared: both ends, and every kind of sequence."""
        group = self.hq // self.hkv
        heads = sorted({0, group - 1, self.hq - 1, self.hq // 2})
        rows = np.unique(np.clip([0, 1, 2, self.Q // 3, self.Q // 2, self.Q // 2 + 1, self.Q - 2, self.Q - 1], 0, self.Q - 1))
        for b in sorted({0, min(1, self.B - 1), min(2, self.B - 1), min(3, self.B - 1), self.B - 1}):
            for h in heads:
                yield b, h, rows, f"sequence {b} head {h}"

    def check(self, out, lse, places=None, columns=None):
        """places: as of places(), by default those; columns: that are compared, by default all."""
        columns = np.arange(self.d) if columns is None else columns
        for b, h, rows, name in self.places() if places is None else places:
            seen = self.seen[b][rows]
            at = np.nonzero(seen.any(0))[0]
            k, v = (self.x[n][b, torch.from_numpy(at).to(DEVICE), h * self.hkv // self.hq].double() for n in "kv")
            ref, rl, w, reach = attention(self.q[b, rows, h].double(), k, v, torch.from_numpy(seen[:, at]).to(DEVICE), self.d ** -0.5)
            count = max(len(at), 1)
            qu.close(out[b, rows, h].double().cpu().numpy()[:, columns], ref[:, columns], qu.tolerance(ref, w, reach, self.d, count)[:, columns], name)
            rl[rows > self.gammas[b]] = 0.0
            qu.close(lse[b, h, rows], rl, qu.lse_tolerance(rl, reach, self.d, count), name + " lse")


def binding_call(*args, **kw):
    from gpu_util import rapid
    return rapid().rapid_verify_attn_window(*args, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("page,layout", [(0, "head"), (16, "token")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("plan", sorted(PLANS))
def test_every_plan(plan, d, page, layout):
    from gpu_util import rapid
    assert plan_of(rapid()._ctx, d, *PLANS[plan]) == plan
    call = Call(d, *PLANS[plan], page, layout)
    call.check(*call.run())


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("plan", sorted(PLANS))
def test_who_does_not_attend_it_does_not_see_it(plan, d, bad):
    """A sink, a token that rows lose one after another, one that they come to one after another, and a draft, in kv heads of their own: rows that attend none of their head's are
    within the tolerance of what they are without; of the others, NaN in K reaches all of a row, and anything that is not finite in V its column alone.  (An infinity in K may
    have a weight of 0 or of NaN, and says nothing of the rows that attend it.)"""
    call = Call(d, *PLANS[plan], 0, "token")
    Q, L, group = call.Q, call.cap, call.hq // call.hkv
    clean, clean_lse = call.run()
    column = 3
    others = np.array([c for c in range(d) if c != column])
    tokens = {0: [L - Q + Q // 2 - call.window, L - Q + Q // 2]}
    tokens.setdefault(call.hkv - 1, []).extend([L - 1, L - Q + Q // 3])
    if call.hkv > 2:
        tokens[1] = [2]
    tokens = {h: [t for t in ts if call.seen[0][:, t].any()] for h, ts in tokens.items()}
    some = np.zeros((call.hkv, Q), bool)                     # who attends a bad token
    for h, ts in tokens.items():
        some[h] = call.seen[0][:, ts].any(1)
    reached = torch.from_numpy(np.repeat(some, group, 0).T.copy()).to(DEVICE)                    # [Q, Hq]
    assert reached.any()
    heads = sorted({0, group - 1, min(group, call.hq - 1), call.hq - 1})
    free = [(0, h, np.flatnonzero(~some[h // group])[:: 1 + Q // 8], f"head {h}, who does not attend it") for h in heads]
    there = [(0, h, np.flatnonzero(some[h // group])[:: 1 + Q // 8], f"head {h}, who attends it") for h in heads]
    free, there = ([p for p in x if len(p[2])] for x in (free, there))
    for n in "vk":
        kept = call.x[n][0].clone()
        for h, ts in tokens.items():
            for t in ts:
                call.x[n][0, t, h, column] = bad
        out, lse = call.run()
        call.x[n][0] = kept
        assert torch.equal(out[1:], clean[1:]) and torch.equal(lse[1:], clean_lse[1:])
        assert torch.isfinite(out[0][~reached]).all() and torch.isfinite(lse[0].T[~reached]).all()
        call.check(out, lse, free)
        if n == "v":
            assert not torch.isfinite(out[0][reached][:, column]).any()
            call.check(out, lse, there, others)
        elif np.isnan(bad):
            assert torch.isnan(out[0][reached]).all() and torch.isnan(lse[0].T[reached]).all()
