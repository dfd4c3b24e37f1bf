"""The cache in 8 bits: rapid_kv_append_quant, rapid_kv_read_quant and rapid_verify_attn_quant against the format and the attention in
64 bits."""
import numpy as np
import pytest
import torch

import quant_util as qu
from gpu_util import rapid

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def awkward_rows(rng, shape):
    """bf16 rows with what a row may hold: ordinary values, one large one, zeros, the smallest and largest numbers, NaN and infinities,
    values on the borders between two codes and between two scales."""
    x = rng.standard_normal(shape) * 2.0 ** rng.integers(-8, 9, shape[:-1])[..., None]
    flat = x.reshape(-1, shape[-1])
    for i in range(len(flat)):
        kind = i % 13
        if kind == 1: flat[i] = 0.0
        if kind == 2: flat[i, ::2] = -0.0
        if kind == 3: flat[i] *= 2.0 ** -125
        if kind == 4: flat[i] = np.sign(flat[i]) * 3.3895e38
        if kind == 5: flat[i, 3] = np.nan
        if kind == 6: flat[i, 5], flat[i, 6] = np.inf, -np.inf
        if kind == 7: flat[i] = np.inf
        if kind == 8: flat[i, 0] = 448.0; flat[i, 1:] = np.round(flat[i, 1:] * 4) / 4 + 0.125
        if kind == 9: flat[i, 0] = 1.7578125; flat[i, 1] = 1.75
        if kind == 10: flat[i] = np.arange(shape[-1]) * 2.0 ** -10
        if kind == 11: flat[i] = 2.0 ** -133
    return torch.from_numpy(x).to(torch.bfloat16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,layout", [(0, "token"), (0, "head"), (0, "wide"), (16, "token"), (64, "head")])
def test_append_writes_its_rows_and_nothing_else(d, page, layout):
    rng = np.random.default_rng(d + page)
    lens, gammas, Q, hkv = [70, 5, 33, 100, 0, 2], [6, 4, 0, 40, 3, 3], 41, 3      # the fifth and sixth have fewer tokens than rows
    cache = qu.QuantCache(rng, lens, hkv, d, page, cap=101)
    new = {n: awkward_rows(rng, (len(lens), Q, hkv, d)) for n in "kv"}
    kc, vc, ks, vs, table = cache.dev(layout)
    rapid().rapid_kv_append_quant(kc, vc, ks, vs, new["k"].cuda(), new["v"].cuda(), i32(lens), gammas=i32(gammas), page_table=table,
                                  max_ctx=101)
    for n in "kv":
        for b, (length, g) in enumerate(zip(lens, gammas)):
            i = np.arange(max(0, g + 1 - length), g + 1)
            cache.put(n, b, length - g - 1 + i, *qu.quantise(new[n][b, i].double().numpy()))
    for n, c, s in (("k", kc, ks), ("v", vc, vs)):
        assert np.array_equal(c.view(torch.uint8).cpu().numpy(), cache.codes[n])
        assert np.array_equal(s.view(torch.uint8).cpu().numpy(), cache.scales[n])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,layout", [(0, "token"), (0, "wide"), (16, "head")])
def test_read_gives_the_stored_values(d, page, layout):
    rng = np.random.default_rng(5 + d + page)
    lens, gammas, Q, hkv = [70, 5, 33, 100, 0, 2], [6, 4, 0, 98, 3, 3], 100, 3
    cache = qu.QuantCache(rng, lens, hkv, d, page, cap=101, spread=90.0)
    cache.codes["v"][:] = rng.integers(0, 256, cache.codes["v"].shape)              # every code, every scale that append writes
    cache.scales["v"][:] = rng.integers(27, 247, cache.scales["v"].shape)
    kc, vc, ks, vs, table = cache.dev(layout)
    outs = rapid().rapid_kv_read_quant(kc, vc, ks, vs, i32(lens), Q, gammas=i32(gammas), page_table=table, max_ctx=101)
    for n, out in zip("kv", outs):
        want = np.zeros((len(lens), Q, hkv, d))
        for b, (length, g) in enumerate(zip(lens, gammas)):
            i = np.arange(max(0, g + 1 - length), g + 1)
            want[b, i] = cache.tokens(n, b)[length - g - 1 + i]
        got = out.double().cpu().numpy()
        assert np.array_equal(got, want, equal_nan=True)


def test_read_back_and_written_again_keeps_the_values():
    rng = np.random.default_rng(11)
    n, hkv, d = 500, 2, 128
    cache = qu.QuantCache(rng, [n], hkv, d)
    kc, vc, ks, vs, _ = cache.dev()
    k, v = rapid().rapid_kv_read_quant(kc, vc, ks, vs, i32([n]), n)
    again = qu.QuantCache(rng, [n], hkv, d).dev()
    rapid().rapid_kv_append_quant(*again[:4], k, v, i32([n]))
    k2, v2 = rapid().rapid_kv_read_quant(*again[:4], i32([n]), n)
    assert torch.equal(k, k2) and torch.equal(v, v2)


def run_attention(cache, lens, gammas, Q, hq, layout, scale=None, q=None, seed=0, lse=True):
    rng = np.random.default_rng(seed + 1)
    B, d = len(lens), cache.d
    q = qu.bf16(rng, (B, Q, hq, d)) if q is None else q
    kc, vc, ks, vs, table = cache.dev(layout)
    lse_out = torch.full((B, hq, Q), 7.0, device="cuda") if lse else None
    out = rapid().rapid_verify_attn_quant(q.cuda(), kc, vc, ks, vs, i32(lens), gammas=i32(gammas), page_table=table,
                                          max_ctx=cache.cap, softmax_scale=scale, lse_out=lse_out)
    group = hq // cache.hkv
    qu.check_attention(q, out, lse_out, lambda b, h: (cache.tokens("k", b)[:, h // group], cache.tokens("v", b)[:, h // group], 0),
                       gammas, d ** -0.5 if scale is None else scale, lens)
    return out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,Q", [(1, 1, 1), (4, 1, 5), (8, 2, 4), (14, 2, 7), (6, 1, 11), (8, 1, 10), (16, 2, 12)])
def test_attention_of_every_row_count(d, hq, hkv, Q):
    """1 to 96 rows a kv head, one odd length."""
    rng = np.random.default_rng(100 * Q + d)
    cache = qu.QuantCache(rng, [333], hkv, d)
    run_attention(cache, [333], [Q - 1], Q, hq, "head")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1025, 5000])
def test_attention_of_every_length(d, n):
    rng = np.random.default_rng(n + d)
    cache = qu.QuantCache(rng, [n], 1, d)
    run_attention(cache, [n], [0], 1, 4, "token")
    if n >= 4:
        run_attention(cache, [n], [3], 5, 4, "token", lse=False)


@pytest.mark.parametrize("page,layout", [(0, "token"), (0, "head"), (0, "wide"), (16, "token"), (16, "head"), (64, "wide"), (256, "token")])
@pytest.mark.parametrize("d,hq,hkv", [(128, 12, 3), (64, 8, 2)])
def test_ragged_batches(page, layout, d, hq, hkv):
    """Lengths from none to thousands in one batch, as many drafts as there are tokens, rows that a sequence does not have."""
    rng = np.random.default_rng(page + d)
    lens, gammas = [700, 1, 0, 2049, 64, 5, 300], [5, 0, 2, 3, 6, 4, 6]
    cache = qu.QuantCache(rng, lens, hkv, d, page, cap=2100)
    run_attention(cache, lens, gammas, 7, hq, layout)


def test_a_long_sequence_among_short_ones():
    rng = np.random.default_rng(3)
    lens = [40, 20000, 1, 17, 300]
    cache = qu.QuantCache(rng, lens, 2, 128, 16)
    run_attention(cache, lens, [3, 8, 0, 8, 2], 9, 8, "token")


def test_many_sequences():
    """More sequences than a wave has lanes, and than the chip has compute units."""
    rng = np.random.default_rng(4)
    lens = [int(x) for x in rng.integers(0, 90, 300)]
    cache = qu.QuantCache(rng, lens, 1, 64, cap=96)
    gammas = [min(1, max(n - 1, 0)) for n in lens]
    run_attention(cache, lens, gammas, 2, 2, "token")


@pytest.mark.parametrize("scale", [1e-3, 1.0, 30.0])
def test_scores_from_flat_to_one_key(scale):
    rng = np.random.default_rng(9)
    cache = qu.QuantCache(rng, [1500], 1, 128)
    run_attention(cache, [1500], [4], 5, 4, "token", scale=scale)


def test_scores_that_rise_and_fall_along_the_sequence():
    """The running maximum moves at every tile, or never."""
    rng = np.random.default_rng(10)
    n, d = 2000, 64
    for order in (1, -1):
        cache = qu.QuantCache(rng, [n], 1, d)
        x = np.ones((n, 1, d)) * (np.linspace(-8, 8, n)[::order])[:, None, None]
        x = torch.from_numpy(x).to(torch.bfloat16).double().numpy()
        cache.put("k", 0, np.arange(n), *qu.quantise(x))
        run_attention(cache, [n], [2], 3, 2, "token", scale=1.0, q=torch.ones((1, 3, 2, d), dtype=torch.bfloat16))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [40, 130, 700])
def test_nan_reaches_who_attends_it_and_nobody_else(d, n):
    """NaN in a draft's K or V, which the rows before it do not attend; then in an early token, which all attend."""
    rng = np.random.default_rng(n)
    for name, tok in (("v", n - 1), ("v", n - 3), ("k", n - 1), ("k", n - 2)):
        cache = qu.QuantCache(rng, [n, n - 5], 2, d)
        r, t = cache.at(0, np.array([tok]))
        cache.codes[name][r, t, 1, 5:9] = [0x7F, 0xFF, 0x7F, 0xFF]
        out = run_attention(cache, [n, n - 5], [4, 4], 5, 4, "token")
        assert torch.isnan(out[0]).any() and not torch.isnan(out[0, 0]).any() and not torch.isnan(out[1]).any()
    cache = qu.QuantCache(rng, [n], 1, d)
    cache.codes["v"][0, 3, 0, 7] = 0x7F
    out = run_attention(cache, [n], [4], 5, 4, "token")
    assert torch.isnan(out[..., 7]).all() and int(torch.isnan(out).sum()) == 5 * 4


def test_page_ids_outside_the_pool_are_clamped():
    rng = np.random.default_rng(21)
    cache = qu.QuantCache(rng, [100, 60], 2, 64, 16)
    kc, vc, ks, vs, table = cache.dev()
    bad = table.clone()
    bad[0, 1], bad[1, 2] = -7, 1 << 30
    cache.table[0, 1], cache.table[1, 2] = 0, kc.shape[0] - 1
    q = qu.bf16(rng, (2, 3, 4, 64)).cuda()
    ok = torch.from_numpy(cache.table).cuda()
    args = (q, kc, vc, ks, vs, i32([100, 60]))
    assert torch.equal(rapid().rapid_verify_attn_quant(*args, page_table=bad, max_ctx=100).nan_to_num(9.0),
                       rapid().rapid_verify_attn_quant(*args, page_table=ok, max_ctx=100).nan_to_num(9.0))
    a = rapid().rapid_kv_read_quant(kc, vc, ks, vs, i32([100, 60]), 50, page_table=bad, max_ctx=100)
    b = rapid().rapid_kv_read_quant(kc, vc, ks, vs, i32([100, 60]), 50, page_table=ok, max_ctx=100)
    assert all(torch.equal(x.nan_to_num(9.0), y.nan_to_num(9.0)) for x, y in zip(a, b))


def test_lengths_and_drafts_outside_their_range_are_clamped():
    rng = np.random.default_rng(22)
    cache = qu.QuantCache(rng, [80, 80], 1, 64)
    kc, vc, ks, vs, _ = cache.dev()
    q = qu.bf16(rng, (2, 4, 2, 64)).cuda()
    r = rapid()
    one = r.rapid_verify_attn_quant(q, kc, vc, ks, vs, i32([1000, -5]), gammas=i32([99, -3]))
    two = r.rapid_verify_attn_quant(q, kc, vc, ks, vs, i32([80, 0]), gammas=i32([3, 0]))
    assert torch.equal(one, two)


def test_offsets_past_32_bits():
    """A pool of more than 4 GiB of codes: pages at its far end."""
    hkv, d, page = 8, 128, 64
    pages = (5 << 30) // (page * hkv * d)
    r, rng = rapid(), np.random.default_rng(6)
    codes = [torch.zeros((pages, page, hkv, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((pages, hkv, page), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
    table = torch.tensor([[pages - 1, 3, pages - 5]], dtype=torch.int32, device="cuda")
    n = 150
    new = [qu.bf16(rng, (1, n, hkv, d)).cuda() for _ in range(2)]
    r.rapid_kv_append_quant(*codes, *scales, *new, i32([n]), page_table=table)
    back = r.rapid_kv_read_quant(*codes, *scales, i32([n]), n, page_table=table)
    want = [qu.quantise(x.double().cpu().numpy()) for x in new]
    vals = [qu.values(*w) for w in want]
    for b, w in zip(back, vals):
        assert np.array_equal(b.double().cpu().numpy(), w)
    q = qu.bf16(rng, (1, 2, 16, d))
    out = r.rapid_verify_attn_quant(q.cuda(), *codes, *scales, i32([n]), page_table=table)
    qu.check_attention(q, out, None, lambda b, h: (vals[0][0][:, h // 2], vals[1][0][:, h // 2], 0), [1], d ** -0.5, [n])


@pytest.mark.parametrize("page", [0, 16])
def test_a_whole_generation_on_a_quantised_cache(page):
    """A prompt is written, then rounds of drafts are appended, attended, and all but some taken back; the cache is read back in the end."""
    rng = np.random.default_rng(31 + page)
    r, hq, hkv, d, Q = rapid(), 8, 2, 128, 5
    lens = [200, 37, 90]
    B, cap = len(lens), 256
    cache = qu.QuantCache(rng, [0] * B, hkv, d, page, cap=cap)
    kc, vc, ks, vs, table = cache.dev("head")
    more = dict(page_table=table, max_ctx=cap)

    def append(new, lens, gammas):
        r.rapid_kv_append_quant(kc, vc, ks, vs, new["k"].cuda(), new["v"].cuda(), ctx, gammas=i32(gammas), **more)
        for n in "kv":
            for b, (length, g) in enumerate(zip(lens, gammas)):
                cache.put(n, b, np.arange(length - g - 1, length), *qu.quantise(new[n][b, :g + 1].double().numpy()))

    ctx = i32(lens)
    append({n: qu.bf16(rng, (B, max(lens), hkv, d)) for n in "kv"}, lens, [n - 1 for n in lens])
    for _ in range(3):
        gammas = [int(x) for x in rng.integers(0, Q, B)]
        lens = [n + g + 1 for n, g in zip(lens, gammas)]
        ctx += i32(g + 1 for g in gammas)
        append({n: qu.bf16(rng, (B, Q, hkv, d)) for n in "kv"}, lens, gammas)
        q = qu.bf16(rng, (B, Q, hq, d))
        lse = torch.empty((B, hq, Q), device="cuda")
        out = r.rapid_verify_attn_quant(q.cuda(), kc, vc, ks, vs, ctx, gammas=i32(gammas), lse_out=lse, **more)
        qu.check_attention(q, out, lse, lambda b, h: (cache.tokens("k", b, lens[b])[:, h // 4], cache.tokens("v", b, lens[b])[:, h // 4], 0),
                           gammas, d ** -0.5, lens)
        accepted = [int(rng.integers(0, g + 1)) for g in gammas]
        r.rapid_kv_commit(ctx, i32(accepted), Q - 1, gammas=i32(gammas))
        lens = [n - g + a for n, g, a in zip(lens, gammas, accepted)]
        assert ctx.tolist() == lens
    back = r.rapid_kv_read_quant(kc, vc, ks, vs, ctx, max(lens), gammas=i32(n - 1 for n in lens), **more)
    for n, got in zip("kv", back):
        for b in range(B):
            assert np.array_equal(got[b, :lens[b]].double().cpu().numpy(), cache.tokens(n, b, lens[b]))
            assert not got[b, lens[b]:].any()


def test_captured_and_replayed_with_eager_calls_between():
    """One graph of append and attention, replayed over changing lengths and rows, against the eager calls; another object's larger call and this
    one's in between."""
    from paper_2502_20330_amd import binding
    rng = np.random.default_rng(41)
    r, hq, hkv, d, Q, cap = binding.Rapid(0), 8, 2, 128, 4, 900
    lens = [[500, 37], [504, 40], [899, 4], [5, 700]]
    cache = qu.QuantCache(rng, [cap, cap], hkv, d)
    state, check = cache.dev(), cache.dev()
    q, k, v = (qu.bf16(rng, (2, Q, h, d)).cuda() for h in (hq, hkv, hkv))
    ctx, out = i32(lens[0]), torch.empty((2, Q, hq, d), dtype=torch.bfloat16, device="cuda")

    def step(r, s, out):
        r.rapid_kv_append_quant(*s[:4], k, v, ctx)
        return r.rapid_verify_attn_quant(q, *s[:4], ctx, out=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(r, state, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(r, state, out)
    big = qu.QuantCache(rng, [3000] * 4, hkv, d)
    for n in lens:
        for t in (q, k, v):
            t.copy_(qu.bf16(rng, t.shape))
        ctx.copy_(i32(n))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        # the object's workspace grows; the recorded one stays
        r.rapid_verify_attn_quant(qu.bf16(rng, (4, 12, hq, d)).cuda(), *big.dev()[:4], i32([3000] * 4))
        want = step(rapid(), check, torch.empty_like(out))
        assert torch.equal(got, want)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(state[:4], check[:4]))


@pytest.mark.parametrize("d,page", [(64, 0), (64, 16), (128, 0), (128, 64)])
def test_rows_by_the_thousand(d, page):
    """So many rows that a thread takes several: whole blocks of them and a rest, fewer rows than there is room for, fewer tokens than rows."""
    rng = np.random.default_rng(70 + d + page)
    hkv = 8
    Q = (1 << 21) // (2 * hkv * 2 * (d // 8)) + 37
    lens, gammas = [Q + 5, Q - 50], [Q - 60, Q - 1]
    cache = qu.QuantCache(rng, [0, 0], hkv, d, page, cap=Q + 6)
    new = {n: awkward_rows(rng, (2, Q, hkv, d)) for n in "kv"}
    kc, vc, ks, vs, table = cache.dev()
    more = dict(gammas=i32(gammas), page_table=table, max_ctx=Q + 6)
    rapid().rapid_kv_append_quant(kc, vc, ks, vs, new["k"].cuda(), new["v"].cuda(), i32(lens), **more)
    outs = rapid().rapid_kv_read_quant(kc, vc, ks, vs, i32(lens), Q, **more)
    for n, c, s, out in (("k", kc, ks, outs[0]), ("v", vc, vs, outs[1])):
        want = np.zeros((2, Q, hkv, d), np.float32)
        for b, (length, g) in enumerate(zip(lens, gammas)):
            i = np.arange(max(0, g + 1 - length), g + 1)
            codes, scales = qu.quantise(new[n][b, i].double().numpy())
            cache.put(n, b, length - g - 1 + i, codes, scales)
            want[b, i] = qu.values(codes, scales)
        assert np.array_equal(c.view(torch.uint8).cpu().numpy(), cache.codes[n])
        assert np.array_equal(s.view(torch.uint8).cpu().numpy(), cache.scales[n])
        assert np.array_equal(out.float().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("d,page,hq,Q", [(128, 0, 8, 1), (64, 16, 16, 5), (128, 16, 16, 14), (64, 0, 16, 20), (128, 0, 16, 24)])
def test_batches_of_short_sequences(d, page, hq, Q):
    """A workgroup for each sequence and kv head: lengths from none to the bound, fewer tokens than rows, rows that a sequence does not have."""
    rng = np.random.default_rng(80 + Q + d)
    lens = [0, 1, 3, 1000, 1024, 16, 0, 127, 128, 129, 31, 33] + [int(x) for x in rng.integers(0, 300, 20)]
    gammas = [int(x) for x in rng.integers(0, Q, len(lens))]
    cache = qu.QuantCache(rng, lens, 4, d, page, cap=1024)
    r, t = cache.at(3, np.array([997]))
    cache.codes["v"][r, t, 1, 2] = 0x7F                    # for the last rows alone, if there are so many
    run_attention(cache, lens, gammas, Q, hq, "token")


def test_tens_of_thousands_of_sequences():
    rng = np.random.default_rng(90)
    B, d = 32767, 64
    r = rapid()
    codes = [torch.zeros((B, 16, 1, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros((B, 1, 16), dtype=torch.uint8, device="cuda") for _ in range(2)]
    new = [qu.bf16(rng, (B, 2, 1, d)) for _ in range(2)]
    n = torch.full((B,), 2, dtype=torch.int32, device="cuda")
    r.rapid_kv_append_quant(*codes, *scales, *(x.cuda() for x in new), n)
    back = r.rapid_kv_read_quant(*codes, *scales, n, 2)
    vals = [qu.values(*qu.quantise(x.double().numpy())) for x in new]
    for got, want in zip(back, vals):
        assert np.array_equal(got.float().cpu().numpy(), want.astype(np.float32))
    q = qu.bf16(rng, (B, 1, 1, d))
    out = r.rapid_verify_attn_quant(q.cuda(), *codes, *scales, n)
    some = [0, 1, 255, 256, 16383, 16384, 32766]
    qu.check_attention(q[some], out[some], None, lambda b, h: (vals[0][some[b]][:, 0], vals[1][some[b]][:, 0], 0), [0] * 7, d ** -0.5, [2] * 7)


@pytest.mark.parametrize("n", [100, 3000])
def test_scores_far_below_zero(n):
    """All of a row's scores are the same number near -1e32: its weights are equal."""
    rng = np.random.default_rng(91)
    d = 64
    cache = qu.QuantCache(rng, [n], 1, d)
    cache.put("k", 0, np.arange(n), *qu.quantise(np.full((n, 1, d), -2.0 ** 50)))
    kc, vc, ks, vs, _ = cache.dev()
    q = torch.full((1, 1, 4, d), 2.0 ** 54, dtype=torch.bfloat16, device="cuda")
    out = rapid().rapid_verify_attn_quant(q, kc, vc, ks, vs, i32([n]))
    v = cache.tokens("v", 0)[:, 0]
    tol = n * 2.0 ** -24 * np.abs(v).mean(0) + 2.0 ** -8 * np.abs(v.mean(0))       # weights of 1; the sum, and the rounding of the result
    qu.close(out[0, 0, 3], v.mean(0), tol)


def test_two_graphs_of_one_object_in_turn():
    """Both use the object's workspace; one after the other on a stream they do not disturb each other, nor eager calls between."""
    from paper_2502_20330_amd import binding
    rng = np.random.default_rng(92)
    r, d = binding.Rapid(0), 128
    calls, graphs, outs = [], [], []
    for lens, Q in (([2000, 300], 4), ([5000], 9)):
        cache = qu.QuantCache(rng, lens, 2, d)
        args = (qu.bf16(rng, (len(lens), Q, 8, d)).cuda(), *cache.dev()[:4], i32(lens))
        calls.append(args)
        outs.append(torch.empty_like(args[0]))
    want = [rapid().rapid_verify_attn_quant(*args) for args in calls]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for args, out in zip(calls, outs):
            r.rapid_verify_attn_quant(*args, out=out)
    torch.cuda.current_stream().wait_stream(side)
    for args, out in zip(calls, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            r.rapid_verify_attn_quant(*args, out=out)
    for turn in range(4):
        for out in outs:
            out.zero_()
        for g in graphs if turn % 2 else graphs[::-1]:
            g.replay()
            eager = r.rapid_verify_attn_quant(*calls[turn % 2])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1]) and torch.equal(eager, want[turn % 2])


def test_on_another_stream():
    rng = np.random.default_rng(51)
    cache = qu.QuantCache(rng, [3000], 2, 128)
    dev = cache.dev()
    q = qu.bf16(rng, (1, 3, 8, 128)).cuda()
    want = rapid().rapid_verify_attn_quant(q, *dev[:4], i32([3000]))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = rapid().rapid_verify_attn_quant(q, *dev[:4], i32([3000]))
    s.synchronize()
    assert torch.equal(got, want)
    assert all(torch.equal(rapid().rapid_verify_attn_quant(q, *dev[:4], i32([3000])), want) for _ in range(3))   # the same bits every time


def test_calls_on_two_streams_at_once():
    """Of one object, without waiting for one another."""
    rng = np.random.default_rng(52)
    streams, calls = [torch.cuda.Stream() for _ in range(2)], []
    for lens, Q in (([20000], 9), ([3000, 900], 4)):
        cache = qu.QuantCache(rng, lens, 2, 128)
        calls.append((qu.bf16(rng, (len(lens), Q, 8, 128)).cuda(), *cache.dev()[:4], i32(lens)))
    want = [rapid().rapid_verify_attn_quant(*c) for c in calls]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(rapid().rapid_verify_attn_quant(*calls[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


def test_refusals_of_the_binding():
    from paper_2502_20330_amd import binding
    rng = np.random.default_rng(61)
    r = rapid()
    kc, vc, ks, vs, _ = qu.QuantCache(rng, [64], 2, 64).dev()
    q = qu.bf16(rng, (1, 2, 4, 64)).cuda()
    n = i32([64])
    new = qu.bf16(rng, (1, 2, 2, 64)).cuda()
    bad = [
        lambda: r.rapid_verify_attn_quant(q.float(), kc, vc, ks, vs, n),
        lambda: r.rapid_verify_attn_quant(q, kc.float(), vc.float(), ks, vs, n),
        lambda: r.rapid_verify_attn_quant(q, kc, vc, ks[:, :1], vs[:, :1], n),
        lambda: r.rapid_verify_attn_quant(q, kc, vc, ks[..., ::2], vs[..., ::2], n),
        lambda: r.rapid_verify_attn_quant(q, kc, vc, ks[..., :40], vs[..., :40], n),
        lambda: r.rapid_verify_attn_quant(q, kc, vc, ks, vs, n.long()),
        lambda: r.rapid_verify_attn_quant(q, kc, vc, ks, vs, n.cpu()),
        lambda: r.rapid_verify_attn_quant(q, kc, vc, ks, vs, i32([64, 64])),
        lambda: r.rapid_verify_attn_quant(q, kc, vc, ks, vs, n, max_ctx=65),
        lambda: r.rapid_verify_attn_quant(q, kc, vc, ks, vs, n, out=torch.empty_like(q)[:, :1]),
        lambda: r.rapid_verify_attn_quant(q, kc, vc, ks, vs, n, lse_out=torch.empty((1, 2, 4), device="cuda")),
        lambda: r.rapid_verify_attn_quant(q, kc, vc, ks, vs, n, 2),
        lambda: r.rapid_verify_attn_quant(qu.bf16(rng, (1, 33, 6, 64)).cuda(), kc, vc, ks, vs, n),
        lambda: r.rapid_kv_append_quant(kc, vc, ks, vs, new.float(), new.float(), n),
        lambda: r.rapid_kv_append_quant(kc, vc, ks, vs, new[..., :32], new[..., :32], n),
        lambda: r.rapid_kv_read_quant(kc, vc, ks, vs, n, 65),
        lambda: r.rapid_kv_read_quant(kc, vc, ks, vs, n, 0),
        lambda: r.rapid_kv_read_quant(kc, vc, ks, vs, n, 3, outs=(new, new)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(binding.RapidError):
            call()
            pytest.fail(f"call {i} was taken")
