"""rapid_verify_attn_prefix: attention of a batch behind one shared prefix, against the attention in 64 bits."""
import numpy as np
import pytest
import torch

import quant_util as qu
from gpu_util import rapid

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


class Batch:
    """A prefix and the sequences' own caches: bf16, everything that no token owns is NaN."""

    def __init__(self, rng, prefix, lens, hkv, d, page=0, cap=None, prefix_cap=None):
        self.P, self.lens, self.hkv, self.d, self.page = prefix, list(lens), hkv, d, page
        self.cap, self.pcap = cap or max(max(lens), 1), max(prefix_cap or prefix, 1)
        self.own = {n: [qu.bf16(rng, (m, hkv, d)) for m in lens] for n in "kv"}
        self.shared = {n: qu.bf16(rng, (prefix, hkv, d)) for n in "kv"}
        if page:
            # the last row of the table is the prefix's
            self.table, n = qu.page_table(rng, [self.cap] * len(lens) + [self.pcap], page)
            shape = (n, page, hkv, d)
        else:
            shape = (len(lens), self.cap, hkv, d)
        self.cache = {n: torch.full(shape, torch.nan, dtype=torch.bfloat16) for n in "kv"}
        self.prefix = {n: torch.full((1, self.pcap, hkv, d), torch.nan, dtype=torch.bfloat16) for n in "kv"}
        self.store()

    def store(self):
        for n in "kv":
            for b, x in enumerate(self.own[n] + ([self.shared[n]] if self.page else [])):
                j = np.arange(x.shape[0])
                if self.page:
                    self.cache[n][self.table[b, j // self.page], j % self.page] = x
                else:
                    self.cache[n][b, :len(j)] = x
            self.prefix[n][0, :self.P] = self.shared[n]

    def args(self, layout, contiguous_prefix=False):
        """Positional and keyword arguments of a call, without q."""
        k, v = (qu.laid_out(self.cache[n].cuda(), layout) for n in "kv")
        kw = dict(max_ctx=self.cap, max_prefix=self.pcap)
        if self.page:
            kw["page_table"] = torch.from_numpy(self.table[:-1, :-(-self.cap // self.page)].copy()).cuda()
        if self.page and not contiguous_prefix:
            kw["prefix_table"] = torch.from_numpy(self.table[-1, :-(-self.pcap // self.page)].copy()).cuda()
        else:
            kw["k_prefix"], kw["v_prefix"] = (qu.laid_out(self.prefix[n].cuda(), layout)[0] for n in "kv")
        return (k, v, i32(self.lens), i32([self.P])), kw

    def check(self, rng, gammas, Q, hq, layout="token", scale=None, contiguous_prefix=False, lse=True, q=None):
        B = len(self.lens)
        q = qu.bf16(rng, (B, Q, hq, self.d)) if q is None else q
        args, kw = self.args(layout, contiguous_prefix)
        lse_out = torch.full((B, hq, Q), 7.0, device="cuda") if lse else None
        out = rapid().rapid_verify_attn_prefix(q.cuda(), *args, gammas=i32(gammas), softmax_scale=scale, lse_out=lse_out, **kw)
        self.compare(q, out, lse_out, gammas, scale)
        return out

    def compare(self, q, out, lse, gammas, scale=None):
        group = q.shape[2] // self.hkv
        whole = {n: [torch.cat([self.shared[n], x]).double().numpy() for x in self.own[n]] for n in "kv"}
        qu.check_attention(q, out, lse, lambda b, h: (whole["k"][b][:, h // group], whole["v"][b][:, h // group], self.P), gammas,
                           self.d ** -0.5 if scale is None else scale, self.lens)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,hq,hkv,Q", [(1, 1, 1, 1), (2, 4, 1, 1), (3, 8, 2, 4), (2, 14, 2, 7), (5, 6, 1, 9), (7, 8, 1, 5), (4, 16, 2, 12),
                                        (6, 16, 2, 12), (13, 8, 2, 9)])
def test_every_row_count(d, B, hq, hkv, Q):
    """1 to 576 rows of the batch a kv head."""
    rng = np.random.default_rng(100 * Q + d + B)
    lens = [int(x) for x in rng.integers(Q, 60, B)]
    Batch(rng, 333, lens, hkv, d).check(rng, [int(x) for x in rng.integers(0, Q, B)], Q, hq, "head")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("prefix", [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257, 1000, 5000])
def test_every_prefix_length(d, prefix):
    rng = np.random.default_rng(prefix + d)
    Batch(rng, prefix, [20, 1, 33], 1, d).check(rng, [2, 0, 2], 3, 4)


@pytest.mark.parametrize("page,layout,contiguous", [(0, "token", False), (0, "head", False), (0, "wide", False), (16, "token", False),
                                                    (16, "head", False), (64, "wide", False), (16, "token", True)])
@pytest.mark.parametrize("d,hq,hkv", [(128, 12, 3), (64, 8, 2)])
def test_ragged_batches(page, layout, contiguous, d, hq, hkv):
    """Own lengths from none to hundreds, rows that a sequence does not have, a prefix that ends inside a page and below its bound."""
    rng = np.random.default_rng(page + d)
    lens, gammas = [700, 1, 0, 64, 5, 300], [5, 0, 2, 6, 4, 6]
    Batch(rng, 601, lens, hkv, d, page, cap=705, prefix_cap=900).check(rng, gammas, 7, hq, layout, contiguous_prefix=contiguous)


def test_a_long_prefix_and_many_sequences():
    rng = np.random.default_rng(2)
    lens = [int(x) for x in rng.integers(1, 30, 70)]
    Batch(rng, 9000, lens, 1, 64).check(rng, [0] * 70, 1, 4)


@pytest.mark.parametrize("scale", [1e-3, 1.0, 30.0])
def test_scores_from_flat_to_one_key(scale):
    rng = np.random.default_rng(9)
    Batch(rng, 1500, [300, 40], 1, 128).check(rng, [4, 4], 5, 4, scale=scale)


def test_scores_that_rise_and_fall_along_the_prefix():
    rng = np.random.default_rng(10)
    d = 64
    for order in (1, -1):
        batch = Batch(rng, 2000, [90, 4], 1, d)
        batch.shared["k"] = (torch.ones((2000, 1, d)) * torch.linspace(-8, 8, 2000)[::1, None, None].flip(0 if order < 0 else 1)).to(torch.bfloat16)
        batch.store()
        batch.check(rng, [2, 2], 3, 2, scale=1.0, q=torch.ones((2, 3, 2, d), dtype=torch.bfloat16))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("d", [64, 128])
def test_what_is_not_finite_reaches_who_attends_it_and_nobody_else(bad, d):
    """A draft's K or V holds `bad`: the rows before it and the other sequences are as without; then an early token of the prefix does."""
    rng = np.random.default_rng(12)
    for n in "vk":
        batch = Batch(rng, 100, [80, 50], 2, d)
        batch.own[n][0][-1, 1, 5] = bad
        batch.own[n][0][-2, 0, 7] = bad
        batch.store()
        out = batch.check(rng, [4, 4], 5, 4)
        assert torch.isfinite(out[0, :3]).all() and torch.isfinite(out[1]).all()
        if n == "v":
            assert not torch.isfinite(out[0, 4, 2:, 5]).any()
    batch = Batch(rng, 100, [80, 50], 2, d)
    batch.shared["v"][3, 0, 9] = bad
    batch.store()
    out = batch.check(rng, [4, 4], 5, 4)
    assert not torch.isfinite(out[:, :, :2, 9]).any()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("prefix", [1, 31, 70, 333])
@pytest.mark.parametrize("B,Q", [(2, 5), (9, 12), (5, 7)])
def test_what_is_not_finite_at_the_end_of_the_prefix(bad, prefix, B, Q):
    """Its last token, in the tile that goes on behind the end: every row attends it."""
    rng = np.random.default_rng(prefix + B)
    for n in "vk":
        batch = Batch(rng, prefix, [Q + b for b in range(B)], 1, 128, prefix_cap=prefix + 40)
        batch.shared[n][-1, 0, 9] = bad
        batch.store()
        out = batch.check(rng, [Q - 1] * B, Q, 8)
        assert not torch.isfinite(out if n == "k" and bad != bad else out[..., 9]).any() or (n == "k" and bad == bad)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,Q,hq,hkv", [(9, 12, 8, 1), (30, 3, 8, 2), (20, 2, 16, 4), (40, 2, 4, 1)])
def test_many_rows_of_a_ragged_batch(d, B, Q, hq, hkv):
    """More rows than the streaming kernel takes, sequences without tokens or rows among them, paged; then with no prefix at all under the same bound."""
    rng = np.random.default_rng(B + d)
    lens = [int(x) for x in rng.integers(0, 40, B)]
    lens[1], gammas = 0, [int(x) for x in rng.integers(0, Q, B)]
    Batch(rng, 523, lens, hkv, d, 16, cap=64, prefix_cap=700).check(rng, gammas, Q, hq, "head")
    Batch(rng, 0, lens, hkv, d, 16, cap=64, prefix_cap=700).check(rng, gammas, Q, hq, "head")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,page", [(98, 0), (99, 16), (100, 0), (102, 16), (104, 64)])
def test_thousands_of_rows(d, B, page):
    """6272 to 6656 rows: tiles of 128, 192, 320, 384 and 256; sequences here and there are compared.  Then a token of the last tile is not finite."""
    rng = np.random.default_rng(B + d)
    Q, hq, some = 8, 8, [0, 1, 2, B // 2, B - 1]
    lens, gammas = [int(x) for x in rng.integers(0, 40, B)], [int(x) for x in rng.integers(0, Q, B)]
    lens[1], lens[2], gammas[2] = 0, 3, Q - 1
    batch = Batch(rng, 4201, lens, 1, d, page, cap=48, prefix_cap=4230)
    q, lse = qu.bf16(rng, (B, Q, hq, d)), torch.empty((B, hq, Q), device="cuda")
    for bad in (None, float("nan"), float("inf")):
        if bad is not None:
            batch.shared["v"][-1, 0, 9] = bad
            batch.store()
        args, kw = batch.args("head")
        out = rapid().rapid_verify_attn_prefix(q.cuda(), *args, gammas=i32(gammas), lse_out=lse, **kw)
        whole = {n: [torch.cat([batch.shared[n], batch.own[n][b]]).double().numpy() for b in some] for n in "kv"}
        qu.check_attention(q[some], out[some], lse[some], lambda b, h: (whole["k"][b][:, 0], whole["v"][b][:, 0], batch.P),
                           [gammas[b] for b in some], d ** -0.5, [lens[b] for b in some])


def test_an_empty_prefix_array_is_no_prefix():
    rng = np.random.default_rng(18)
    lens, gammas = [300, 0, 7], [2, 0, 1]
    batch = Batch(rng, 0, lens, 2, 64)
    q = qu.bf16(rng, (3, 3, 4, 64))
    (k, v, n, length), _ = batch.args("token")
    empty = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((3, 4, 3), device="cuda")
    out = rapid().rapid_verify_attn_prefix(q.cuda(), k, v, n, length, k_prefix=empty, v_prefix=empty, gammas=i32(gammas), lse_out=lse)
    batch.compare(q, out, lse, gammas)


@pytest.mark.parametrize("B", [2, 40])
def test_scores_far_below_zero(B):
    """All of a row's scores are the same number near -1e32: its weights are equal."""
    rng = np.random.default_rng(19)
    d, P, n = 64, 200, 20
    batch = Batch(rng, P, [n] * B, 1, d)
    for x in [batch.shared["k"], *batch.own["k"]]:
        x.fill_(-2.0 ** 50)
    batch.store()
    args, kw = batch.args("token")
    out = rapid().rapid_verify_attn_prefix(torch.full((B, 1, 4, d), 2.0 ** 54, dtype=torch.bfloat16, device="cuda"), *args, **kw)
    for b in (0, B - 1):
        v = torch.cat([batch.shared["v"], batch.own["v"][b]])[:, 0].double().numpy()
        tol = 2 * (P + n) * 2.0 ** -24 * np.abs(v).mean(0) + 2.0 ** -8 * np.abs(v.mean(0))     # weights of 1; sums, and the rounding of the result
        qu.close(out[b, 0, 2], v.mean(0), tol)


def test_the_prefix_is_as_if_each_sequence_held_it():
    """The same tokens as one sequence each through rapid_verify_attn: results of the two agree to their roundings."""
    rng = np.random.default_rng(13)
    batch = Batch(rng, 2000, [100, 30, 500], 2, 128)
    gammas, Q, hq = [4, 2, 0], 5, 8
    q = qu.bf16(rng, (3, Q, hq, 128))
    args, kw = batch.args("token")
    got = rapid().rapid_verify_attn_prefix(q.cuda(), *args, gammas=i32(gammas), **kw)
    k, v = torch.zeros((3, 2500, 2, 128), dtype=torch.bfloat16), torch.zeros((3, 2500, 2, 128), dtype=torch.bfloat16)
    for n, t in (("k", k), ("v", v)):
        for b, x in enumerate(batch.own[n]):
            t[b, :2000], t[b, 2000:2000 + x.shape[0]] = batch.shared[n], x
    want = rapid().rapid_verify_attn(q.cuda(), k.cuda(), v.cuda(), i32(2000 + n for n in batch.lens), gammas=i32(gammas))
    # weights and results of either are rounded to bf16: four halves of a step, of results well below 1
    assert float((got.float() - want.float()).abs().max()) < 4 * 2.0 ** -8


def test_prefix_length_is_read_on_the_device_and_clamped():
    """A graph recorded once serves prefixes of any length up to the bound."""
    from paper_2502_20330_amd import binding
    rng = np.random.default_rng(14)
    r = binding.Rapid(0)
    batch = Batch(rng, 1000, [40, 12], 2, 128)
    q = qu.bf16(rng, (2, 3, 8, 128)).cuda()
    (k, v, lens, length), kw = batch.args("head")
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r.rapid_verify_attn_prefix(q, k, v, lens, length, out=out, **kw)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.rapid_verify_attn_prefix(q, k, v, lens, length, out=out, **kw)
    for n in (1000, 0, 7, 640, 5000, -3, 1000):
        length.fill_(n)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = rapid().rapid_verify_attn_prefix(q, k, v, lens, i32([min(max(n, 0), 1000)]), **kw)
        assert torch.equal(got, want), n
        other = Batch(rng, 50, [9], 2, 128)
        a, b = other.args("token")
        r.rapid_verify_attn_prefix(q[:1].contiguous(), *a, **b)


def test_on_another_stream_and_twice():
    rng = np.random.default_rng(15)
    batch = Batch(rng, 3000, [40, 300], 2, 128)
    q = qu.bf16(rng, (2, 3, 8, 128)).cuda()
    args, kw = batch.args("token")
    want = rapid().rapid_verify_attn_prefix(q, *args, **kw)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = rapid().rapid_verify_attn_prefix(q, *args, **kw)
    s.synchronize()
    assert torch.equal(got, want)


def test_offsets_past_32_bits():
    """Own caches of more than 4 GiB: the last sequence's rows."""
    rng = np.random.default_rng(16)
    B, cap, hkv, d = 5, 500_000, 8, 128
    k, v = (torch.zeros((B, cap, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    batch = Batch(rng, 77, [30] * B, hkv, d)
    for n, t in (("k", k), ("v", v)):
        t[:, :30] = batch.cache[n].cuda()
    q = qu.bf16(rng, (B, 2, 8, d))
    args, kw = batch.args("token")
    kw["max_ctx"] = cap
    out = rapid().rapid_verify_attn_prefix(q.cuda(), k, v, *args[2:], **kw)
    batch.compare(q, out, None, [1] * B)


def test_refusals_of_the_binding():
    from paper_2502_20330_amd import binding
    rng = np.random.default_rng(17)
    r = rapid()
    batch = Batch(rng, 64, [20, 20], 2, 64)
    (k, v, lens, n), kw = batch.args("token")
    kw = {x: kw[x] for x in ("k_prefix", "v_prefix")}
    q = qu.bf16(rng, (2, 2, 4, 64)).cuda()
    table = i32([0, 1])
    bad = [
        lambda: r.rapid_verify_attn_prefix(q.float(), k, v, lens, n, **kw),
        lambda: r.rapid_verify_attn_prefix(q, k.float(), v.float(), lens, n, **kw),
        lambda: r.rapid_verify_attn_prefix(q, k, v, lens, n),
        lambda: r.rapid_verify_attn_prefix(q, k, v, lens, n, prefix_table=table),
        lambda: r.rapid_verify_attn_prefix(q, k, v, lens, n, prefix_table=table, **kw),
        lambda: r.rapid_verify_attn_prefix(q, k, v, lens, n, max_prefix=65, **kw),
        lambda: r.rapid_verify_attn_prefix(q, k, v, lens, n, max_prefix=-1, **kw),
        lambda: r.rapid_verify_attn_prefix(q, k, v, lens, n, max_ctx=21, **kw),
        lambda: r.rapid_verify_attn_prefix(q, k, v, lens, n.long(), **kw),
        lambda: r.rapid_verify_attn_prefix(q, k, v, lens, n.cpu(), **kw),
        lambda: r.rapid_verify_attn_prefix(q, k, v, lens, n, k_prefix=k[0, :, :1], v_prefix=v[0, :, :1]),
        lambda: r.rapid_verify_attn_prefix(q, k, v, lens, n, k_prefix=kw["k_prefix"].float(), v_prefix=kw["v_prefix"].float()),
        lambda: r.rapid_verify_attn_prefix(q, k, v, lens[:1], n, **kw),
        lambda: r.rapid_verify_attn_prefix(q, k, v, lens, n, 2, **kw),
        lambda: r.rapid_verify_attn_prefix(q, k, v, lens, n, softmax_scale=0.0, **kw),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(binding.RapidError):
            call()
            pytest.fail(f"call {i} was taken")
