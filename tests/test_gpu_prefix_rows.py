"""rapid_verify_attn_prefix where the batch has many rows: the kernel that takes 128 to 384 of them a workgroup (attn_prefix.hip), which bounds of
the prefix well above its length are enough to choose; and the form in one launch that a batch without a prefix takes (max_prefix = 0)."""
import ctypes

import numpy as np
import pytest
import torch

import quant_util as qu
from gpu_util import rapid
from paper_2502_20330_amd import binding
from test_gpu_prefix import Batch, i32

pytestmark = pytest.mark.gpu

N_CU = 256


def partials(hkv, slots, rows, d):
    """Bytes of the partials of `slots` slots of `rows` rows a kv head: sums, then maxima and weights, each rounded up to 256."""
    up = lambda n: -(-n // 256) * 256
    return up(hkv * slots * rows * d * 4) + up(hkv * slots * rows * 8)


def own_partials(B, Q, G, hkv, d, max_ctx):
    groups = min(max(N_CU // hkv, 1), B * (-(-max_ctx // 128) + 2))
    return partials(hkv, groups + B - 1, -(-Q * G // 16) * 16, d)


def prefix_tile(rows):
    """Rows of a workgroup and row tiles: what pads least, the larger of equals."""
    best = min((384, 320, 256, 192, 128), key=lambda t: (-(-rows // t) * t, -t))
    return best, -(-rows // best)


def prefix_partials(B, Q, G, hkv, d, max_prefix):
    tile, tiles = prefix_tile(B * Q * G)
    streams = 2 if tile <= 192 else 1
    quantum = streams * (32 if d == 128 else 64)
    groups = min(max(N_CU // (hkv * tiles), 1), -(-max_prefix // quantum))
    while groups > 1 and groups * groups * hkv * tiles > 2 * max_prefix:
        groups -= 1
    return partials(hkv, tiles * groups, tile, d)


def workspace(B, Q, hq, hkv, d, max_ctx, page, max_prefix):
    s = binding.AttnShape(B, Q, hq, hkv, d, max_ctx, Q - 1, d ** -0.5, max_ctx * hkv * d, hkv * d, d, 0, 0, 0, 0, 0, 0)
    r = rapid()
    return r.lib.rapid_verify_attn_prefix_workspace_bytes(r._ctx, ctypes.byref(s), ctypes.byref(binding.PrefixLayout(max_prefix, 0, hkv * d, d)))


def takes_the_kernel_of_many_rows(B, Q, hq, hkv, d, max_ctx, max_prefix):
    """By the size of the workspace, which is that of its plan and of no other: a change of the rule that chooses shows here."""
    if torch.cuda.get_device_properties(0).multi_processor_count != N_CU:
        return True
    G = hq // hkv
    return workspace(B, Q, hq, hkv, d, max_ctx, 0, max_prefix) == own_partials(B, Q, G, hkv, d, max_ctx) + prefix_partials(B, Q, G, hkv, d, max_prefix)


def big_prefix(batch, cap, layout):
    """The batch's prefix in memory for `cap` tokens (NaN behind it), on the GPU, in a layout."""
    out = []
    for n in "kv":
        whole = torch.full((1, cap, batch.hkv, batch.d), torch.nan, dtype=torch.bfloat16, device="cuda")
        whole[0, :batch.P] = batch.shared[n].cuda()
        out.append(qu.laid_out(whole, layout)[0])
    return dict(k_prefix=out[0], v_prefix=out[1], max_prefix=cap)


def run(batch, Q, hq, gammas, layout="token", prefix_layout=None, cap=None, pages=None, some=None, rng=None, q=None, length=None):
    """One call under a bound that takes the kernel of many rows, compared with 64 bits for the sequences `some`.  pages: a prefix table of so many
    entries, of which the batch's prefix fills the first."""
    B, d, hkv = len(batch.lens), batch.d, batch.hkv
    (k, v, lens, P), kw = batch.args(layout)
    kw = {x: kw[x] for x in ("max_ctx", "page_table") if x in kw}
    if pages:
        table = torch.full((pages,), -1, dtype=torch.int32)
        need = -(-batch.pcap // batch.page)
        table[:need] = torch.from_numpy(batch.table[-1, :need].copy())
        kw["prefix_table"], cap = table.cuda(), pages * batch.page
    else:
        kw.update(big_prefix(batch, cap, prefix_layout or layout))
    assert takes_the_kernel_of_many_rows(B, Q, hq, hkv, d, batch.cap, cap)
    q = qu.bf16(rng, (B, Q, hq, d)) if q is None else q
    lse = torch.full((B, hq, Q), 7.0, device="cuda")
    out = rapid().rapid_verify_attn_prefix(q.cuda(), k, v, lens, P if length is None else length, gammas=i32(gammas), lse_out=lse, **kw)
    some = range(B) if some is None else some
    some, group = list(some), hq // hkv
    whole = {n: {b: torch.cat([batch.shared[n], batch.own[n][b]]).double().numpy() for b in some} for n in "kv"}
    qu.check_attention(q[some], out[some], lse[some], lambda b, h: tuple(whole[n][some[b]][:, h // group] for n in "kv") + (batch.P,),
                       [gammas[b] for b in some], d ** -0.5, [batch.lens[b] for b in some])
    return out, lse


def ragged(rng, B, Q, cap):
    lens, gammas = [int(x) for x in rng.integers(0, cap, B)], [int(x) for x in rng.integers(0, Q, B)]
    lens[1 % B], gammas[2 % B], lens[2 % B] = 0, Q - 1, max(2, cap // 2)
    return lens, gammas


# 100 to 495 rows, which leave a remainder in a tile of 128, 192, 256, 320, 384, and in the second of two
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,Q,G,hkv", [(5, 5, 4, 8), (6, 7, 4, 8), (13, 5, 3, 8), (8, 9, 4, 8), (11, 8, 4, 3), (25, 5, 2, 8), (31, 3, 4, 2), (9, 11, 5, 8)])
def test_row_counts_that_leave_a_remainder(B, Q, G, hkv, d):
    rng = np.random.default_rng(B * Q + d)
    assert B * Q * G % prefix_tile(B * Q * G)[0]
    lens, gammas = ragged(rng, B, Q, 40)
    batch = Batch(rng, 523, lens, hkv, d)
    cap = 1 + (96 << 10) * N_CU // (B * Q * G * hkv)
    run(batch, Q, G * hkv, gammas, "head" if B % 2 else "token", cap=cap + 70, rng=rng, some={0, 1, 2, B // 2, B - 1})


@pytest.mark.parametrize("layout,prefix_layout", [("token", "token"), ("head", "head"), ("wide", "wide"), ("token", "head"), ("head", "wide")])
@pytest.mark.parametrize("d", [64, 128])
def test_memory_orders(layout, prefix_layout, d):
    rng = np.random.default_rng(d)
    lens, gammas = ragged(rng, 8, 9, 90)
    run(Batch(rng, 601, lens, 8, d), 9, 32, gammas, layout, prefix_layout, cap=11500, rng=rng)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("hkv", [2, 8])
@pytest.mark.parametrize("contiguous", [False, True])
def test_pages(page, hkv, contiguous):
    """The prefix in pages of the sequences' pool, or an array beside paged sequences."""
    rng = np.random.default_rng(page + hkv)
    B, Q, G = 8, 9, 4
    lens, gammas = ragged(rng, B, Q, 90)
    batch = Batch(rng, 601, lens, hkv, 128, page, prefix_cap=700)
    cap = 90 + (96 << 10) * N_CU // (B * Q * G * hkv)
    run(batch, Q, G * hkv, gammas, "head", cap=cap, pages=None if contiguous else -(-cap // page), rng=rng)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P", [0, 1, 31, 33, 129, 1000, 11500])
def test_prefix_lengths_under_one_bound(P, d):
    rng = np.random.default_rng(P + d)
    lens, gammas = ragged(rng, 8, 9, 40)
    run(Batch(rng, P, lens, 8, d), 9, 32, gammas, cap=11500, rng=rng, some=[0, 1, 2] if P > 1000 else None)


@pytest.mark.parametrize("given,P", [(20000, 11500), (-5, 0)])
def test_prefix_lengths_past_the_bound_are_clamped(given, P):
    rng = np.random.default_rng(3)
    lens, gammas = ragged(rng, 8, 9, 40)
    run(Batch(rng, P, lens, 8, 64), 9, 32, gammas, cap=11500, rng=rng, some=[0, 1, 2], length=i32([given]))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", [0, 300, -1])
@pytest.mark.parametrize("name", ["k", "v"])
def test_what_is_not_finite_in_the_prefix(bad, where, name):
    """In one kv head of one token, the last with the tile going on behind it: that head's rows feel it, the others do not."""
    rng = np.random.default_rng(7)
    B, Q = 8, 9
    batch = Batch(rng, 333, [20] * B, 8, 128)
    batch.shared[name][where, 3, 9] = bad
    out, _ = run(batch, Q, 32, [Q - 1] * B, cap=11500, rng=rng, some=[0, B - 1])
    others = [h for h in range(32) if h // 4 != 3]
    assert torch.isfinite(out[:, :, others]).all()
    if name == "v":
        assert not torch.isfinite(out[:, :, 12:16, 9]).any() and torch.isfinite(out[:, :, 12:16, :9]).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("name", ["k", "v"])
def test_what_is_not_finite_in_a_draft_behind_it(bad, name):
    rng = np.random.default_rng(8)
    B, Q = 8, 9
    batch = Batch(rng, 333, [20] * B, 8, 128)
    batch.own[name][2][-1, 3, 9] = bad
    batch.store()
    out, _ = run(batch, Q, 32, [Q - 1] * B, cap=11500, rng=rng, some=[0, 2, 3])
    assert torch.isfinite(out[[0, 1, 3, 4, 5, 6, 7]]).all() and torch.isfinite(out[2, :Q - 1]).all()


def test_scores_that_rise_and_fall():
    rng = np.random.default_rng(9)
    B, Q, P, d = 8, 9, 2000, 64
    for order in (1, -1):
        batch = Batch(rng, P, [30] * B, 8, d)
        ramp = torch.linspace(-8, 8, P)
        batch.shared["k"] = (torch.ones((P, 8, d)) * (ramp if order > 0 else ramp.flip(0))[:, None, None]).to(torch.bfloat16)
        run(batch, Q, 32, [Q - 1] * B, cap=11500, rng=rng, some=[0, 7], q=torch.ones((B, Q, 32, d), dtype=torch.bfloat16))


def test_replayed_with_a_changing_prefix():
    """One graph of the three launches, replayed over lengths of the prefix and of the sequences, eager calls of other sizes between."""
    rng = np.random.default_rng(10)
    r, B, Q, cap = binding.Rapid(0), 8, 9, 11500
    batch = Batch(rng, 3000, [60] * B, 8, 128)
    (k, v, lens, P), _ = batch.args("head")
    kw = dict(big_prefix(batch, cap, "head"), max_ctx=batch.cap)
    q = qu.bf16(rng, (B, Q, 32, 128)).cuda()
    gammas = i32([Q - 1] * B)
    assert takes_the_kernel_of_many_rows(B, Q, 32, 8, 128, batch.cap, cap)
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.rapid_verify_attn_prefix(q, k, v, lens, P, gammas=gammas, out=out, **kw)
    for n, own in ((3000, 60), (0, 60), (7, 9), (640, 33), (129, 1), (3000, 0), (3000, 60)):
        P.fill_(n)
        lens.fill_(own)
        gammas.fill_(max(min(Q, own) - 1, 0))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = rapid().rapid_verify_attn_prefix(q, k, v, lens, P, gammas=gammas, **kw)
        assert torch.equal(got, want), (n, own)
        a, b = Batch(rng, 50, [9], 8, 128).args("token")
        r.rapid_verify_attn_prefix(q[:1].contiguous(), *a, **b)
    batch.compare(q, out, None, [Q - 1] * B)


# ---- no prefix at all: one launch, a workgroup for each sequence and kv head
@pytest.mark.parametrize("page,layout", [(0, "token"), (0, "wide"), (16, "head")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,Q,hq,hkv,cap", [([256, 1, 0, 7, 33], 5, 8, 2, 256), ([1], 1, 1, 1, 1), ([100, 255], 12, 16, 2, 256),
                                               ([0, 1, 3, 1000, 1024, 16, 127, 128, 129, 31, 33, 600], 5, 32, 16, 1024)])
def test_no_prefix_and_short_sequences(lens, Q, hq, hkv, cap, d, page, layout):
    """The last occupies most of the chip, so that sequences of up to 1024 tokens take one launch as well.  No partials: a workspace of 256 bytes."""
    rng = np.random.default_rng(cap + d)
    B, gammas = len(lens), [int(x) for x in rng.integers(0, Q, len(lens))]
    if torch.cuda.get_device_properties(0).multi_processor_count == N_CU:
        assert workspace(B, Q, hq, hkv, d, max(cap, Q), 0, 0) == 256
    batch = Batch(rng, 0, lens, hkv, d, page, cap=max(cap, Q))
    (k, v, n, P), kw = batch.args(layout)
    kw = {x: kw[x] for x in ("max_ctx", "page_table") if x in kw}
    empty = torch.empty((0, hkv, d), dtype=torch.bfloat16, device="cuda")
    q, lse = qu.bf16(rng, (B, Q, hq, d)), torch.full((B, hq, Q), 7.0, device="cuda")
    out = rapid().rapid_verify_attn_prefix(q.cuda(), k, v, n, P, k_prefix=empty, v_prefix=empty, gammas=i32(gammas), lse_out=lse, **kw)
    batch.compare(q, out, lse, gammas)
