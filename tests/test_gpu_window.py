"""rapid_verify_attn_window: attention with a sliding window and sinks, from one position to whole prompts, against the attention in 64 bits."""
import numpy as np
import pytest
import torch

import quant_util as qu
from gpu_util import rapid

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def seen_by(length, n, rows, window, sinks):
    """[rows, length]: who attends what."""
    p = length - n + np.arange(rows)[:, None]
    j = np.arange(length)[None, :]
    return (j <= p) & ((j > p - window) | (j < sinks)) & (np.arange(rows)[:, None] < n)


class Batch:
    """Sequences in caches of which everything that nobody attends is NaN."""

    def __init__(self, rng, lens, gammas, Q, hq, hkv, d, window, sinks, page=0, cap=None):
        self.lens, self.gammas, self.Q, self.hq, self.hkv, self.d, self.page = list(lens), list(gammas), Q, hq, hkv, d, page
        self.window, self.sinks, self.cap = window, sinks, cap or max(max(lens), Q)
        self.real = [min(x, self.cap) for x in lens]
        self.x = {n: [qu.bf16(rng, (m, hkv, d)) for m in self.real] for n in "kv"}
        self.q = qu.bf16(rng, (len(lens), Q, hq, d))
        if page:
            self.table, n = qu.page_table(rng, [self.cap] * len(lens), page)
            self.shape = (n, page, hkv, d)
        else:
            self.table, self.shape = None, (len(lens), self.cap, hkv, d)
        self.seen = [seen_by(m, g + 1, Q, window, sinks) for m, g in zip(self.real, self.gammas)]

    def caches(self, layout, device="cuda"):
        got = []
        for n in "kv":
            c = torch.full(self.shape, torch.nan, dtype=torch.bfloat16)
            for b, x in enumerate(self.x[n]):
                j = np.nonzero(self.seen[b].any(0))[0]
                at = (np.full(len(j), b), j) if self.table is None else (self.table[b, j // self.page], j % self.page)
                c[at] = x[j]
            got.append(qu.laid_out(c.to(device), layout))
        return got

    def kw(self):
        table = None if self.table is None else torch.from_numpy(self.table).cuda()
        return dict(sinks=self.sinks, gammas=i32(self.gammas), page_table=table, max_ctx=self.cap)

    def check(self, layout="token", scale=None, lse=True, rows=None):
        """rows: those that are compared (default all)."""
        B = len(self.lens)
        lse_out = torch.full((B, self.hq, self.Q), 7.0, device="cuda") if lse else None
        out = rapid().rapid_verify_attn_window(self.q.cuda(), *self.caches(layout), i32(self.lens), self.window, softmax_scale=scale,
                                               lse_out=lse_out, **self.kw())
        self.compare(out, lse_out, scale, rows)
        return out

    def compare(self, out, lse, scale=None, rows=None):
        scale = self.d ** -0.5 if scale is None else scale
        q = self.q.double().numpy()
        got, lse = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
        rows = np.arange(self.Q) if rows is None else np.unique(np.clip(rows, 0, self.Q - 1))
        for b in range(len(self.lens)):
            for h in range(self.hq):
                k, v = (self.x[n][b][:, h // (self.hq // self.hkv)].double().numpy() for n in "kv")
                ref, rl, w, reach = qu.attention(q[b, rows, h], k, v, self.seen[b][rows], scale)
                name = f"sequence {b} head {h}"
                count = min(k.shape[0], self.window + self.sinks)
                qu.close(got[b, rows, h], ref, qu.tolerance(ref, w, reach, self.d, count), name)
                if lse is not None:
                    rl[rows > self.gammas[b]] = 0.0
                    qu.close(lse[b, h, rows], rl, qu.lse_tolerance(rl, reach, self.d, count), name + " lse")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,Q", [(1, 1, 1), (4, 1, 1), (4, 1, 5), (8, 2, 8), (14, 2, 5), (7, 1, 8), (8, 1, 10), (8, 1, 12), (5, 1, 3)])
@pytest.mark.parametrize("window,sinks", [(100, 4), (512, 0)])
def test_every_count_of_few_rows(d, hq, hkv, Q, window, sinks):
    """1 to 96 packed rows, in one launch and divided among workgroups."""
    rng = np.random.default_rng(Q * hq + d)
    Batch(rng, [900, 130, Q], [Q - 1, Q // 2, Q - 1], Q, hq, hkv, d, window, sinks).check("head")
    Batch(rng, [3000], [Q - 1], Q, hq, hkv, d, 2500, sinks, page=16).check()


@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 1), (128, 6, 2)])
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 64, 100, 257])
@pytest.mark.parametrize("sinks", [0, 1, 31, 32, 33, 70, 1000])
def test_borders_of_window_and_sinks(d, hq, hkv, window, sinks):
    """Runs that end at every place of a tile, that meet, that overlap; sinks beyond the sequences; windows beyond them."""
    rng = np.random.default_rng(window + sinks)
    lens = [1, 5, 32, 33, 64, 65, 97, 200, 301, 640]
    gammas = [0, 4, 2, 4, 0, 3, 4, 1, 4, 4]
    Batch(rng, lens, gammas, 5, hq, hkv, d, window, sinks, page=16 if window % 2 else 0).check()


@pytest.mark.parametrize("page,layout", [(0, "token"), (0, "head"), (0, "wide"), (16, "token"), (16, "head"), (64, "wide")])
@pytest.mark.parametrize("d,hq,hkv,Q", [(128, 12, 3, 7), (64, 16, 2, 12), (128, 32, 4, 9), (64, 8, 2, 70), (128, 14, 2, 150)])
@pytest.mark.parametrize("window,sinks", [(150, 10), (700, 0)])
def test_ragged_batches(page, layout, d, hq, hkv, Q, window, sinks):
    """Lengths from none on, sequences shorter than their rows, rows that a sequence does not have, a length above the bound."""
    rng = np.random.default_rng(page + d + Q)
    lens, gammas = [700, 1, 0, 64, 5, 2000, 300], [Q - 1, 0, 2, Q - 2, Q - 1, 3, Q - 1]
    rows = None if Q < 20 else np.concatenate([np.arange(6), np.arange(60, 75), np.arange(Q - 4, Q), [Q // 3, Q // 2]])
    Batch(rng, lens, gammas, Q, hq, hkv, d, window, sinks, page, cap=1205).check(layout, rows=rows)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Q,hq,hkv", [(100, 1, 1), (33, 4, 1), (95, 2, 1), (127, 2, 1), (80, 4, 1), (55, 7, 1), (128, 3, 1), (200, 4, 2), (400, 1, 1)])
@pytest.mark.parametrize("window,sinks", [(90, 5), (20, 0), (1000, 40)])
def test_every_row_tile(d, Q, hq, hkv, window, sinks):
    """97 to 800 rows a kv head: every tile, one and more of them, their tokens in shares; alone, behind a cache, and from the first token on."""
    rng = np.random.default_rng(Q + d)
    some = np.concatenate([np.arange(3), Q // 2 + np.arange(3), np.arange(Q - 3, Q), rng.integers(0, Q, 12)])
    Batch(rng, [Q, Q + 777], [Q - 1, Q - 1], Q, hq, hkv, d, window, sinks).check(rows=some)


@pytest.mark.parametrize("B,Q,hq,hkv,d,window,sinks,page", [(1, 3000, 8, 2, 64, 500, 8, 0), (2, 1500, 16, 4, 128, 4000, 0, 16),
                                                             (40, 100, 8, 8, 64, 64, 3, 64), (9, 230, 32, 4, 128, 128, 64, 16)])
def test_prompts(B, Q, hq, hkv, d, window, sinks, page):
    """Row tiles that fill the chip, and some that do not exist."""
    rng = np.random.default_rng(Q)
    lens = [Q + 31 * b for b in range(B)]
    gammas = [Q - 1 - (7 * b) % (Q // 2) for b in range(B)]
    some = np.concatenate([[0, 1, Q // 2, Q // 2 + 1, Q - 2, Q - 1], rng.integers(0, Q, 6)])
    Batch(rng, lens, gammas, Q, hq, hkv, d, window, sinks, page).check("head", rows=some)


@pytest.mark.parametrize("Q", [5, 100])
@pytest.mark.parametrize("scale", [1e-3, 1.0, 30.0])
def test_scores_from_flat_to_one_key(scale, Q):
    rng = np.random.default_rng(9)
    Batch(rng, [1500, 400], [Q - 1] * 2, Q, 4, 1, 128, 300, 20).check(scale=scale, rows=np.arange(0, Q, 1 + Q // 10))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Q,hq,hkv", [(6, 4, 2), (6, 12, 1), (60, 4, 2), (200, 8, 2)])
def test_what_is_not_finite_reaches_who_attends_it_and_nobody_else(bad, d, Q, hq, hkv):
    """In V: a sink beside hidden tokens, a token that leaves the window between two rows, one that some rows do not reach yet.  In K: likewise, where
    a score may be infinite of either sign."""
    rng = np.random.default_rng(12)
    for n in "vk":
        batch = Batch(rng, [400, 300], [Q - 1, Q - 1], Q, hq, hkv, d, 50, 3)
        L = 400
        for token, head, column in ((2, 0, 5), (L - Q + 2 - 50, hkv - 1, 7), (L - Q + 4 - 50, 0, 9), (L - 2, 0, 1), (L - Q + 3, hkv - 1, 2)):
            batch.x[n][0][token, head, column] = bad
        if n == "k" and not np.isnan(bad):                   # a weight of 0 or NaN in 64 bits as well: only where it shows
            out = rapid().rapid_verify_attn_window(batch.q.cuda(), *batch.caches("token"), i32(batch.lens), 50, **batch.kw())
            assert torch.isfinite(out[1]).all()
            continue
        out = batch.check(rows=np.concatenate([np.arange(6), np.arange(Q - 4, Q)]))
        assert torch.isfinite(out[1]).all()
        if n == "v":
            g = hq // hkv
            hidden = out[0, 4:Q - 2, (hkv - 1) * g:, 7]      # the second one has left these rows' windows
            assert torch.isfinite(hidden).all() and not torch.isfinite(out[0, 0, (hkv - 1) * g:, 7]).any()
            assert not torch.isfinite(out[0, :, :g, 5]).any()


def test_a_window_over_everything_is_plain_attention():
    """The same bits as with any larger window, and within two roundings of rapid_verify_attn."""
    rng = np.random.default_rng(13)
    batch = Batch(rng, [700, 90], [4, 4], 5, 8, 2, 128, 1 << 20, 0)
    a, c = batch.check(), batch.caches("token")
    kw = dict(gammas=i32(batch.gammas), max_ctx=batch.cap)
    same = rapid().rapid_verify_attn_window(batch.q.cuda(), *c, i32(batch.lens), (1 << 31) - 1, sinks=(1 << 31) - 1, **kw)
    far = rapid().rapid_verify_attn_window(batch.q.cuda(), *c, i32(batch.lens), 1 << 40, **kw)
    plain = rapid().rapid_verify_attn(batch.q.cuda(), *c, i32(batch.lens), **kw)
    assert torch.equal(a, same) and torch.equal(a, far)
    assert (a - plain).abs().max() <= 4 * 2.0 ** -8 * max(x.abs().max() for x in batch.x["v"])


def test_offsets_past_32_bits():
    """Pages at the far end of pools of 4.6 GB, and a contiguous cache whose second sequence begins past 2^32 bytes."""
    rng = np.random.default_rng(14)
    for Q, hq, hkv in ((3, 4, 2), (60, 4, 2), (400, 32, 8)):             # (the last: the kernel of many rows)
        batch = Batch(rng, [500, 400], [Q - 1] * 2, Q, hq, hkv, 128, 200, 5, page=16)
        far = (1 << 32) // (16 * hkv * 128 * 2) + 35000
        pools = [torch.empty((far, 16, hkv, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        small = batch.caches("token")
        for pool, c in zip(pools, small):
            pool[-c.shape[0]:] = c
        table = torch.from_numpy(batch.table + (far - small[0].shape[0])).cuda()
        out = rapid().rapid_verify_attn_window(batch.q.cuda(), *pools, i32(batch.lens), 200, sinks=5, gammas=i32(batch.gammas),
                                               page_table=table, max_ctx=batch.cap)
        batch.compare(out, None, rows=np.arange(0, Q, 1 + Q // 8))
        del pools, pool
        batch = Batch(rng, [500, 400], [Q - 1] * 2, Q, hq, hkv, 128, 200, 5)
        wide = []
        for c in batch.caches("token"):
            t = torch.empty((1 << 31) + (1 << 20), dtype=torch.bfloat16, device="cuda")
            t = t.as_strided(c.shape, ((1 << 31) + 4096, *c.stride()[1:]))
            t.copy_(c)
            wide.append(t)
        out = rapid().rapid_verify_attn_window(batch.q.cuda(), *wide, i32(batch.lens), 200, sinks=5, gammas=i32(batch.gammas), max_ctx=batch.cap)
        batch.compare(out, None, rows=np.arange(0, Q, 1 + Q // 8))
        del wide, t


def test_queries_past_32_bits():
    """A prompt whose queries and results are 4.3 GB each: rows at both ends and around 2^32 bytes."""
    g = torch.Generator(device="cuda").manual_seed(15)
    Q, hq, hkv, d, window = (1 << 19) + 1000, 32, 8, 128, 70
    q, k, v = (torch.randn((1, Q, n, d), generator=g, device="cuda", dtype=torch.bfloat16) for n in (hq, hkv, hkv))
    out = rapid().rapid_verify_attn_window(q, k, v, i32([Q]), window, sinks=3)
    edge = (1 << 32) // (hq * d * 2)
    for p in (0, 5, 4000, edge - 1, edge, edge + 1, Q - 1):
        j = sorted(set(range(min(3, p + 1))) | set(range(max(0, p - window + 1), p + 1)))
        for h in (0, hq - 1):
            kk, vv = (x[0, j, h // (hq // hkv)].double().cpu().numpy() for x in (k, v))
            ref, _, w, reach = qu.attention(q[0, p:p + 1, h].double().cpu().numpy(), kk, vv, np.ones((1, len(j)), bool), d ** -0.5)
            qu.close(out[0, p:p + 1, h].double().cpu().numpy(), ref, qu.tolerance(ref, w, reach, d, len(j)), f"position {p} head {h}")


def test_pages_that_are_given_away():
    """Entries between the sinks and the windows may be anything."""
    rng = np.random.default_rng(15)
    for Q in (4, 90):
        batch = Batch(rng, [900, 1000], [Q - 1] * 2, Q, 4, 2, 64, 100, 20, page=16)
        want = batch.check(rows=np.arange(0, Q, 9))
        kept = batch.table.copy()
        for b, n in enumerate(batch.lens):
            gone = np.arange(-(-20 // 16), (n - Q - 100 + 1) // 16)
            batch.table[b, gone] = rng.choice([-7, 1 << 30, 0, 3], len(gone))
        table = torch.from_numpy(batch.table.copy()).cuda()
        batch.table = kept
        out = rapid().rapid_verify_attn_window(batch.q.cuda(), *batch.caches("token"), i32(batch.lens), 100,
                                               **dict(batch.kw(), page_table=table))
        assert torch.equal(out, want)


@pytest.mark.parametrize("Q", [4, 120])
def test_captured_calls_follow_their_lengths(Q):
    """One graph serves every length up to the bound; eager calls between its replays."""
    rng = np.random.default_rng(16)
    batch = Batch(rng, [900, 700], [Q - 1] * 2, Q, 4, 2, 128, 300, 10)
    r, lens = rapid(), i32(batch.lens)
    # all tokens exist here, since lengths change
    c = [torch.nn.utils.rnn.pad_sequence(batch.x[n], batch_first=True).contiguous().cuda() for n in "kv"]
    q, kw = batch.q.cuda(), batch.kw()
    out = torch.empty_like(q)
    r.rapid_verify_attn_window(q, *c, lens, 300, out=out, **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.rapid_verify_attn_window(q, *c, lens, 300, out=out, **kw)
    for a, b in ((900, 700), (500, 130), (Q, Q + 1), (311, 0), (900, 333)):
        lens.copy_(i32([a, b]))
        out.fill_(9.0)
        graph.replay()
        eager = r.rapid_verify_attn_window(q, *c, lens, 300, **kw)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        batch.lens = batch.real = [a, b]
        short = {n: [x[:m] for x, m in zip(batch.x[n], (a, b))] for n in "kv"}
        whole, batch.x = batch.x, short
        batch.seen = [seen_by(m, Q, Q, 300, 10) for m in (a, b)]
        batch.compare(out, None, rows=np.arange(0, Q, 1 + Q // 8))
        batch.x = whole


def test_streams_and_graphs_at_once():
    """Calls of different sizes on two streams, and replayed graphs of both, have workspaces of their own."""
    from paper_2502_20330_amd import binding
    r = binding.Rapid(0)
    rng = np.random.default_rng(17)
    some = []
    for lens, Q, window in (([20000], 9, 6000), ([3000, 900], 100, 500)):
        x = Batch(rng, lens, [Q - 1] * len(lens), Q, 8, 2, 128, window, 4)
        some.append((x.q.cuda(), *x.caches("head"), i32(lens), window, x.kw()))
    call = lambda a, **more: r.rapid_verify_attn_window(*a[:5], **a[5], **more)
    want = [call(a) for a in some]
    outs, graphs, streams = [torch.empty_like(w) for w in want], [], [torch.cuda.Stream() for _ in some]
    for a, out in zip(some, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(a, out=out)
    torch.cuda.synchronize()
    for _ in range(3):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for _ in range(10):
            for graph, stream in zip(graphs, streams):
                with torch.cuda.stream(stream):
                    graph.replay()
        eager = []
        for a, stream in zip(some, streams):
            with torch.cuda.stream(stream):
                eager.append(call(a))
        torch.cuda.synchronize()
        assert all(torch.equal(a, w) for a, w in zip(outs + eager, want + want))


# Calls that have enough row tiles to fill the chip go to the kernel of many rows; the ones above, for the most part, to that of few rows in tiles.
FULL = [(4, 200, 32, 8, 128, 0), (2, 800, 24, 8, 64, 16), (2, 800, 32, 8, 64, 0), (4, 800, 24, 8, 64, 64), (4, 800, 28, 4, 64, 0),
        (1, 600, 8, 8, 4000, 16), (4, 30, 32, 8, 4096, 0), (1, 800, 32, 8, 4000, 0)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,Q,hq,hkv,window,page", FULL)
def test_every_row_tile_of_a_full_chip(d, B, Q, hq, hkv, window, page):
    """Row tiles of 128 to 384, in one share of the tokens and in several; full sequences, ones shorter than their rows, an empty one."""
    rng = np.random.default_rng(Q + B + d)
    cap = Q + 700 if window < 700 else Q + window
    lens, gammas = [cap, Q // 2, 0, Q][:B], [Q - 1, Q - 1, 2, Q - 9][:B]
    some = np.concatenate([[0, 1, Q // 2, Q // 2 + 1, Q - 2, Q - 1], rng.integers(0, Q, 4)])
    Batch(rng, lens, gammas, Q, hq, hkv, d, window, 5, page, cap).check("head", rows=some)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("d", [64, 128])
def test_what_is_not_finite_in_many_rows(bad, d):
    rng = np.random.default_rng(21)
    Q, hq, hkv, L = 200, 32, 8, 600
    for n in "vk":
        batch = Batch(rng, [L, 500, 450, 300], [Q - 1] * 4, Q, hq, hkv, d, 50, 3)
        for token, head, column in ((2, 0, 5), (L - Q + 2 - 50, hkv - 1, 7), (L - Q + 4 - 50, 0, 9), (L - 2, 0, 1), (L - Q + 3, hkv - 1, 2)):
            batch.x[n][0][token, head, column] = bad
        if n == "k" and not np.isnan(bad):                   # (as above)
            out = rapid().rapid_verify_attn_window(batch.q.cuda(), *batch.caches("token"), i32(batch.lens), 50, **batch.kw())
        else:
            out = batch.check(rows=np.concatenate([np.arange(6), np.arange(Q - 4, Q)]))
        assert torch.isfinite(out[1:]).all()
        if n == "v":
            g = hq // hkv
            assert torch.isfinite(out[0, 4:Q - 2, (hkv - 1) * g:, 7]).all() and not torch.isfinite(out[0, 0, (hkv - 1) * g:, 7]).any()
            assert not torch.isfinite(out[0, :, :g, 5]).any()


@pytest.mark.parametrize("Q,window", [(200, 100), (30, 4096)])
def test_captured_calls_of_many_rows(Q, window):
    """One graph for every length up to the bound, rows that attend nothing among them; eager calls between its replays."""
    rng = np.random.default_rng(22)
    cap = 4200
    batch = Batch(rng, [cap] * 4, [Q - 1] * 4, Q, 32, 8, 64, window, 10)
    r, lens = rapid(), i32(batch.lens)
    c = [torch.stack(batch.x[n]).cuda() for n in "kv"]
    q, kw = batch.q.cuda(), batch.kw()
    out = torch.empty_like(q)
    r.rapid_verify_attn_window(q, *c, lens, window, out=out, **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.rapid_verify_attn_window(q, *c, lens, window, out=out, **kw)
    whole = batch.x
    for now in ([cap, 0, Q, 4100], [Q - 3, cap, 1, 2000], [1111, 33, cap, Q + 1]):
        lens.copy_(i32(now))
        out.fill_(9.0)
        graph.replay()
        eager = r.rapid_verify_attn_window(q, *c, lens, window, **kw)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        batch.lens = batch.real = now
        batch.x = {n: [x[:m] for x, m in zip(whole[n], now)] for n in "kv"}
        batch.seen = [seen_by(m, Q, Q, window, 10) for m in now]
        batch.compare(out, None, rows=np.array([0, 1, Q // 2, Q - 1]))


def test_pages_of_many_rows_that_are_given_away():
    rng = np.random.default_rng(23)
    Q = 200
    batch = Batch(rng, [900, 1000, 700, 950], [Q - 1] * 4, Q, 32, 8, 64, 100, 20, page=16)
    want = batch.check(rows=np.array([0, 1, 77, Q - 1]))
    table = batch.table.copy()
    for b, n in enumerate(batch.lens):
        gone = np.arange(-(-20 // 16), (n - Q - 100 + 1) // 16)
        table[b, gone] = rng.choice([-7, 1 << 30, 0, 3], len(gone))
    out = rapid().rapid_verify_attn_window(batch.q.cuda(), *batch.caches("token"), i32(batch.lens), 100,
                                           **dict(batch.kw(), page_table=torch.from_numpy(table).cuda()))
    assert torch.equal(out, want)


def test_a_drafters_prompt_and_steps():
    """The calls as they are used: the prompt's keys are rotated into the cache and attended, then single tokens, on the head in 8-bit integers and
    the draw; every attention is that of the rotated rows in 64 bits."""
    rng = np.random.default_rng(18)
    r, d, hq, hkv, window, sinks, vocab = rapid(), 64, 8, 2, 120, 4, 5000
    cap, page = 256, 16
    table, n = qu.page_table(rng, [cap, cap], page)
    k, v = (torch.full((n, page, hkv, d), torch.nan, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    freq = torch.tensor(10000.0 ** (-2.0 * np.arange(d // 2) / d), dtype=torch.float32, device="cuda")
    w = qu.bf16(rng, (vocab, hq * d), 0.05).cuda()
    codes, scales = r.rapid_quant_rows(w)
    lens, tab = i32([0, 0]), torch.from_numpy(table).cuda()
    whole = {x: [torch.zeros((0, hkv, d), dtype=torch.bfloat16) for _ in range(2)] for x in "kv"}
    for step, (rows, gammas) in enumerate([(200, [199, 149]), (1, [0, 0]), (1, [0, 0]), (6, [5, 2]), (1, [0, 0])]):
        x = qu.bf16(rng, (2, rows, hq + 2 * hkv, d)).cuda()
        q_new, k_new, v_new = x.split([hq, hkv, hkv], 2)
        g = i32(gammas)
        lens += g + 1
        kw = dict(gammas=g, page_table=tab, max_ctx=cap)
        q = r.rapid_kv_append_rope(k, v, k_new, v_new, freq, lens, q_new=q_new, **kw)
        out = r.rapid_verify_attn_window(q, k, v, lens, window, sinks=sinks, **kw)
        last = out[torch.arange(2), g.long()].reshape(2, hq * d).contiguous()
        logits, stats = r.rapid_lm_head_quant(last, codes, scales)
        _, tokens, _ = r.rapid_accept(logits[:, None], logits[:, None][:, :0], torch.empty((2, 0), dtype=torch.int32, device="cuda"), 0.0,
                                      torch.rand((2, 1), device="cuda"), target_stats=stats)
        assert ((tokens >= 0) & (tokens < vocab)).all()
        for b in range(2):
            m, at = gammas[b] + 1, int(lens[b])
            pos = np.arange(at - m, at)
            turns = torch.from_numpy(pos[:, None] * freq.double().cpu().numpy())[:, None]
            cos, sin = turns.cos(), turns.sin()
            for name, src, heads in (("q", q_new, hq), ("k", k_new, hkv)):
                y = src[b, :m].double().cpu()
                a, c = y[..., :d // 2], y[..., d // 2:]
                y = torch.cat([a * cos - c * sin, c * cos + a * sin], -1)
                got = q[b, :m].double().cpu() if name == "q" else k[table[b, pos // page], pos % page].double().cpu()
                assert ((got - y).abs() <= 2.0 ** -8 * y.abs() + 2.0 ** -20 * 16).all()
            whole["k"][b] = torch.cat([whole["k"][b], k[table[b, pos // page], pos % page].cpu()])
            whole["v"][b] = torch.cat([whole["v"][b], v_new[b, :m].cpu()])
            seen = seen_by(at, m, rows, window, sinks)
            for h in range(hq):
                ref, _, wt, reach = qu.attention(q[b, :, h].double().cpu().numpy()[:m], whole["k"][b][:, h // 4].double().numpy(),
                                                 whole["v"][b][:, h // 4].double().numpy(), seen[:m], d ** -0.5)
                qu.close(out[b, :m, h], ref, qu.tolerance(ref, wt, reach, d, window + sinks), f"step {step} sequence {b} head {h}")
