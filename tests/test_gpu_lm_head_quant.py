"""rapid_quant_rows and rapid_lm_head_quant: 8-bit integers with a scale for each row, and the output head on them."""
import numpy as np
import pytest
import torch

import quant_util as qu
from gpu_util import rapid

pytestmark = pytest.mark.gpu


def codes_of(x):
    """x (float64, values of bf16) -> whole numbers and scales, in 64 bits: the quotients are ratios of a 15-bit and an 8-bit number, whose
    rounding to 53 bits crosses no border between two codes."""
    m = np.abs(x).max(1)
    with np.errstate(invalid="ignore"):
        c = np.rint(127.0 * x / np.where(m > 0, m, 1.0)[:, None])
    fine = np.isfinite(m)
    return np.where(fine[:, None], c, 0), np.where(fine, m / 127.0, np.nan)


def check_rows(x, codes, scales, cols):
    want, scale = codes_of(x.double().cpu().numpy())
    got = codes.cpu().numpy()
    assert np.array_equal(got[:, :cols], want) and not got[:, cols:].any()
    # one rounding of 32 bits, or of the last place of a number below the smallest normal one
    qu.close(scales, scale, 2.0 ** -24 * np.abs(np.nan_to_num(scale)) + 2.0 ** -150)


@pytest.mark.parametrize("rows,cols", [(1, 8), (3, 256), (2, 264), (5, 2048), (4, 2056), (70, 4096), (9, 4104), (6, 8192), (3, 8200), (2, 20000),
                                       (1, 131072), (1000, 904), (3, 16384), (2, 16392), (7, 12000)])
def test_rows_of_every_length(rows, cols):
    rng = np.random.default_rng(rows + cols)
    x = qu.bf16(rng, (rows, cols + 16)) * torch.from_numpy(2.0 ** rng.integers(-30, 30, (rows, 1))).to(torch.bfloat16)
    x = x.cuda()[:, :cols]                                   # rows further apart than they are long
    codes, scales = rapid().rapid_quant_rows(x)
    assert codes.shape == (rows, -(-cols // 256) * 256)
    check_rows(x, codes, scales, cols)
    again = rapid().rapid_quant_rows(x.contiguous())
    assert torch.equal(again[0], codes) and torch.equal(again[1], scales)


@pytest.mark.parametrize("top", [128 + 127, 254, 129, 128, 192])
def test_every_border_between_codes(top):
    """All quotients of two 8-bit significands, over twelve powers of two: the borders themselves among them."""
    x = np.concatenate([[top]] + [np.arange(128, 256) * 2.0 ** -e for e in range(12)])
    x = x[np.abs(x) <= top]
    x = np.concatenate([x, -x, np.zeros(-len(x) * 2 % 8)])
    for scale in (0, 100, -110, 119, -124):
        t = torch.from_numpy(np.ldexp(x, scale)[None]).to(torch.bfloat16)
        assert np.isfinite(t.double().numpy()).all()
        check_rows(t, *(y for y in rapid().rapid_quant_rows(t.cuda())), t.shape[1])


def test_rows_that_have_no_scale():
    x = torch.zeros((5, 64), dtype=torch.bfloat16)
    x[1, 3], x[2, 63], x[3, 0], x[4, 5] = float("nan"), float("inf"), -float("inf"), 2.0
    x[1:4, 7] = 1.0
    codes, scales = (t.cpu() for t in rapid().rapid_quant_rows(x.cuda()))
    assert scales[0] == 0 and torch.isnan(scales[1:4]).all() and scales[4] == np.float32(2.0) / np.float32(127.0)
    assert not codes[:4].any() and codes[4, 5] == 127 and codes[4].count_nonzero() == 1


class Head:
    def __init__(self, rng, rows, hidden, vocab):
        self.h = qu.bf16(rng, (rows, hidden)) * torch.from_numpy(2.0 ** rng.integers(-3, 3, (rows, 1))).to(torch.bfloat16)
        self.w = qu.bf16(rng, (vocab, hidden), 0.05)
        self.h[:, rng.integers(0, hidden)] *= 8
        self.codes, self.scales = rapid().rapid_quant_rows(self.w.cuda())

    def reference(self):
        """(logits in 64 bits, from the codes' exact sums and the scales as they are kept in 32)"""
        c, s = codes_of(self.h.double().numpy())
        cw, sw = codes_of(self.w.double().numpy())
        total = torch.from_numpy(c) @ torch.from_numpy(cw).t().contiguous()        # whole numbers: exact
        return total.numpy() * s.astype(np.float32).astype(np.float64)[:, None] * sw.astype(np.float32).astype(np.float64)

    def check(self, logits, stats=None, temperature=1.0):
        z = self.reference()
        got = logits.double().cpu().numpy()
        qu.close(got, z, 3.01 * 2.0 ** -24 * np.abs(np.nan_to_num(z)), "logits")
        if stats is not None:
            chunk = rapid().lm_head_chunk(z.shape[1], z.shape[0])
            s = stats.double().cpu().numpy()
            for j, v0 in enumerate(range(0, z.shape[1], chunk)):
                part = got[:, v0:v0 + chunk]
                assert np.array_equal(s[:, j, 0], part.max(1))
                ref = np.exp((part - part.max(1, keepdims=True)) / temperature).sum(1)
                # a difference, a product with 1/T log2 e and an exponential of 32 bits; at most 512 additions
                reach = (part.max(1) - part.min(1)) / temperature
                assert (np.abs(s[:, j, 1] - ref) <= ref * ((reach + 4) * 2.0 ** -22 + 520 * 2.0 ** -24)).all()


@pytest.mark.parametrize("rows", [1, 2, 9, 16, 17, 32, 33, 48, 49, 64, 65, 72, 80, 81, 96])
@pytest.mark.parametrize("hidden,vocab", [(512, 8192), (768, 1000)])
def test_row_counts(rows, hidden, vocab):
    head = Head(np.random.default_rng(rows), rows, hidden, vocab)
    head.check(*rapid().rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales))


@pytest.mark.parametrize("hidden", [8, 64, 248, 256, 264, 896, 1016, 1024, 2304, 3584, 4096, 4104, 5120, 8192])
@pytest.mark.parametrize("rows", [3, 50])
def test_widths(hidden, rows):
    """Slabs of 256 and of 512 bytes, rows that end inside one, fewer slabs than workgroups begin at."""
    head = Head(np.random.default_rng(hidden), rows, hidden, 5003)
    head.check(*rapid().rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales, temperature=0.7), temperature=0.7)


@pytest.mark.parametrize("vocab", [16, 17, 31, 100, 4095, 4097, 50257, 131073])
@pytest.mark.parametrize("rows", [1, 70])
def test_vocabularies(vocab, rows):
    head = Head(np.random.default_rng(vocab), rows, 256, vocab)
    wide = torch.full((rows, vocab + 3), 7.0, device="cuda")
    logits, stats = rapid().rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales, logits=wide[:, :vocab])
    head.check(logits, stats)
    assert (wide[:, vocab:] == 7.0).all()
    again, none = rapid().rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales, want_stats=False)
    assert none is None and torch.equal(again, logits)


# Short rows of which there are few are brought to codes by the product's own workgroups, where the vocabulary gives each of them more than 32 entries.
SHORT = [(1, 512), (16, 512), (17, 512), (8, 1024), (9, 1024), (1, 4096), (2, 4096), (3, 4096), (1, 5120), (4, 2048), (5, 1536), (6, 1536), (1, 8192), (1, 8704)]


@pytest.mark.parametrize("vocab", [12001, 17000])
@pytest.mark.parametrize("rows,hidden", SHORT)
def test_few_short_rows(rows, hidden, vocab):
    """Either side of both limits; waves without a block; vocabularies that end inside one."""
    head = Head(np.random.default_rng(rows * hidden + vocab), rows, hidden, vocab)
    logits, stats = rapid().rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales, temperature=1.3)
    head.check(logits, stats, temperature=1.3)


@pytest.mark.parametrize("rows,hidden", [(4, 512), (8, 1024), (4, 2048)])
def test_few_short_rows_without_a_scale(rows, hidden):
    """Zeros, not a number and infinity, each in a row of its own and at either end; the last row is as ever."""
    head = Head(np.random.default_rng(8), rows, hidden, 10000)
    head.h[0] = 0
    head.h[1, hidden - 1], head.h[2, 0] = float("nan"), -float("inf")
    logits, stats = rapid().rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales)
    head.check(logits)
    assert (logits[0] == 0).all() and torch.isnan(logits[1:3]).all() and torch.isfinite(logits[3:]).all() and torch.isfinite(stats[3:]).all()


def test_few_short_rows_in_a_graph():
    """The rows are read by every replay, with eager calls of other sizes between them."""
    rng = np.random.default_rng(9)
    head, other = Head(rng, 3, 1024, 20000), Head(rng, 40, 512, 20000)
    r, h = rapid(), head.h.cuda()
    logits, _ = r.rapid_lm_head_quant(h, head.codes, head.scales, want_stats=False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.rapid_lm_head_quant(h, head.codes, head.scales, want_stats=False, logits=logits)
    for k in range(3):
        head.h = qu.bf16(rng, (3, 1024)) * 2.0 ** k
        h.copy_(head.h)
        logits.zero_()
        graph.replay()
        eager, _ = r.rapid_lm_head_quant(other.h.cuda(), other.codes, other.scales, want_stats=False)
        torch.cuda.synchronize()
        head.check(logits)
        other.check(eager)


def test_sums_beyond_24_bits():
    """All codes 127, the longest rows: 2^17 * 127^2, just below 2^31; and the same with one sign less."""
    h = torch.ones((2, 1 << 17), dtype=torch.bfloat16)
    w = torch.ones((32, 1 << 17), dtype=torch.bfloat16)
    w[1] = -1
    w[2, ::2] = -1
    codes, scales = rapid().rapid_quant_rows(w.cuda())
    z = rapid().rapid_lm_head_quant(h.cuda(), codes, scales)[0].double().cpu().numpy()
    want = np.full(32, 2.0 ** 17)
    want[1], want[2] = -want[1], 0
    # (scales of 1/127 are off by 2^-24 each, besides the three roundings)
    assert (np.abs(z - want) <= 5.01 * 2.0 ** -24 * np.abs(want)).all()


def test_what_lies_behind_hidden_has_no_effect():
    head = Head(np.random.default_rng(5), 20, 264, 300)
    want, _ = rapid().rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales)
    head.codes[:, 264:] = 99
    got, _ = rapid().rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales)
    assert torch.equal(got, want)


def test_rows_and_entries_without_a_scale():
    head = Head(np.random.default_rng(6), 20, 256, 600)
    head.h[3, 7], head.h[17, 0] = float("nan"), float("inf")
    head.w[11, 5] = float("nan")
    head.codes, head.scales = rapid().rapid_quant_rows(head.w.cuda())
    head.check(rapid().rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales, want_stats=False)[0])


def test_equal_entries_are_equal_wherever_they_lie():
    """Sums are exact, so that ties stay ties although workgroups sum in different orders."""
    head = Head(np.random.default_rng(7), 9, 4096, 20000)
    head.w[:] = head.w[0]
    head.codes, head.scales = rapid().rapid_quant_rows(head.w.cuda())
    z, _ = rapid().rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales)
    assert (z == z[:, :1]).all()


def test_streams_and_graphs_have_workspaces_of_their_own():
    from paper_2502_20330_amd import binding
    r = binding.Rapid(0)
    rng = np.random.default_rng(8)
    heads = [Head(rng, n, 4096, 30000) for n in (5, 70)]
    args = [(x.h.cuda(), x.codes, x.scales) for x in heads]
    want = [r.rapid_lm_head_quant(*a)[0] for a in args]
    streams = [torch.cuda.Stream() for _ in args]
    outs = [torch.empty_like(w) for w in want]
    graphs = []
    for a, out in zip(args, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            r.rapid_lm_head_quant(*a, logits=out, want_stats=False)
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
        for a, stream in zip(args, streams):
            with torch.cuda.stream(stream):
                eager.append(r.rapid_lm_head_quant(*a)[0])
        torch.cuda.synchronize()
        assert all(torch.equal(a, w) for a, w in zip(outs + eager, want + want))


def test_draws_from_the_quantised_head():
    """The drafter's last two calls: head, then the draw at gamma = 0 on its statistics; the same token as from the logits alone."""
    rng = np.random.default_rng(9)
    head = Head(rng, 6, 1024, 32000)
    r = rapid()
    logits, stats = r.rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales, temperature=0.8)
    u = torch.rand((6, 1), device="cuda")
    empty = dict(draft_logits=torch.empty((6, 0, 32000), device="cuda"), draft_tokens=torch.empty((6, 0), dtype=torch.int32, device="cuda"))
    _, tokens, _ = r.rapid_accept(logits[:, None], empty["draft_logits"], empty["draft_tokens"], 0.0, u, temperature=0.8, target_stats=stats)
    p = torch.softmax(logits.double() / 0.8, -1).cpu().numpy()
    for b in range(6):
        c = np.cumsum(p[b])
        t = int(tokens[b, 0])
        lo, hi = (0 if t == 0 else c[t - 1]) / c[-1], c[t] / c[-1]
        assert lo - 1e-6 <= float(u[b, 0]) <= hi + 1e-6


# One shape for each of the kernels: codes by the product's own workgroups, the hidden dimension shared among the waves (slabs of 512 and of 256 bytes), a copy of h for each
# wave (likewise), one for the workgroup.
KERNELS = [(2, 1024, 12001), (5, 512, 5003), (20, 768, 1000), (9, 2304, 12001), (40, 1024, 17000), (72, 1024, 17000)]


@pytest.mark.parametrize("rows,hidden,vocab", KERNELS)
def test_a_chunk_with_a_nan_has_a_sum_that_is_none(rows, hidden, vocab):
    """Entries without a scale, at either end, beside one another, over a whole chunk; a row without one; a logit that is infinite: a chunk's sum is NaN where the formula's is,
    its maximum is that of the numbers, and the other chunks' statistics are what they are without."""
    head = Head(np.random.default_rng(rows + vocab), rows, hidden, vocab)
    r, chunk = rapid(), rapid().lm_head_chunk(vocab, rows)
    clean, clean_stats = r.rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales)
    scales = head.scales.clone()
    for v in (0, 3 * chunk + 7, 3 * chunk + 8, vocab - 1, *range(5 * chunk, 6 * chunk)):
        scales[v] = torch.nan
    scales[7 * chunk + 1] = 1e38                             # (times a scale of about 2^-6 and a sum of some thousands)
    logits, stats = r.rapid_lm_head_quant(head.h.cuda(), head.codes, scales)
    z = logits.double().cpu().numpy()
    assert np.array_equal(np.isnan(z), np.broadcast_to(torch.isnan(scales).cpu().numpy(), z.shape))
    s, was = (x.double().cpu().numpy() for x in (stats, clean_stats))
    for j, v0 in enumerate(range(0, vocab, chunk)):
        part = z[:, v0:v0 + chunk]
        bad = np.isnan(part).any(1) | (part == np.inf).any(1)
        numbers = np.where(np.isnan(part), -np.inf, part)
        assert np.array_equal(s[:, j, 0], numbers.max(1)), j
        assert np.array_equal(np.isnan(s[:, j, 1]), bad), j
        if j not in (0, 3, 5, 7, (vocab - 1) // chunk):
            assert np.array_equal(s[:, j], was[:, j]), j
    head.h[rows - 1, 0] = torch.nan
    z, stats = r.rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales)
    assert torch.isnan(z[rows - 1]).all() and (stats[rows - 1, :, 0] == -torch.inf).all() and torch.isnan(stats[rows - 1, :, 1]).all()
    assert torch.equal(z[:rows - 1], clean[:rows - 1]) and torch.equal(stats[:rows - 1], clean_stats[:rows - 1])


def test_a_draw_leaves_the_chunk_of_a_nan_out():
    """Of the row's sums: the token is one that there is, whatever the uniform."""
    vocab, T = 32000, 0.8
    head = Head(np.random.default_rng(10), 6, 1024, vocab)
    r, chunk = rapid(), rapid().lm_head_chunk(32000, 6)
    head.scales[3 * chunk + 5] = torch.nan
    logits, stats = r.rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales, temperature=T)
    none = dict(draft_logits=torch.empty((6, 0, vocab), device="cuda"), draft_tokens=torch.empty((6, 0), dtype=torch.int32, device="cuda"))
    for u in (0.0, 0.3, 0.999):
        _, tokens, _ = r.rapid_accept(logits[:, None], none["draft_logits"], none["draft_tokens"], 0.0, torch.full((6, 1), u, device="cuda"), temperature=T,
                                      target_stats=stats)
        assert ((tokens >= 0) & (tokens < vocab)).all()


def check_row_counts(counts, hidden, vocab, kind):
    """The first rows of one matrix; `kind` names the kernel that takes them, which goes by the entries a workgroup has and by the width."""
    head = Head(np.random.default_rng(hidden + vocab), max(counts), hidden, vocab)
    z, h = head.reference(), head.h
    assert rapid().lm_head_chunk(vocab) > 32 and {"narrow": hidden % 512 == 256, "wide": hidden % 512 == 0}[kind]
    for rows in counts:
        head.h, head.reference = h[:rows].contiguous(), lambda: z[:rows]
        head.check(*rapid().rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales, temperature=0.9), temperature=0.9)


@pytest.mark.parametrize("hidden,vocab", [(512, 17000), (1024, 12001), (1536, 17000), (4096, 12001)])
def test_row_counts_where_the_waves_share_a_copy(hidden, vocab):
    """From 49 rows on, with one slab and with several, and what is just below."""
    check_row_counts([17, 32, 33, 48, 49, 64, 65, 72, 80, 81, 95, 96], hidden, vocab, "wide")


@pytest.mark.parametrize("hidden,vocab", [(256, 12001), (768, 17000), (2304, 12001)])
def test_row_counts_of_narrow_slabs(hidden, vocab):
    """Rows that are no multiple of 512 bytes: slabs of 256, one and several, at which the workgroups begin in turn."""
    check_row_counts([1, 2, 16, 17, 33, 48, 49, 64, 65, 81, 96], hidden, vocab, "narrow")


@pytest.mark.parametrize("hidden,vocab", [(8192, 9000), (3584, 12001)])
def test_row_counts_of_wide_rows(hidden, vocab):
    check_row_counts([2, 16, 31, 47, 60, 96], hidden, vocab, "wide")


def test_borders_between_codes_of_all_maxima():
    """All quotients of two 8-bit significands, over twelve powers of two, a row for each maximum."""
    x = np.concatenate([np.arange(128, 256) * 2.0 ** -e for e in range(12)])
    rows = np.zeros((128, 2 * len(x) + 8))
    for i, top in enumerate(range(128, 256)):
        y = np.concatenate([[top], x[x <= top]])
        rows[i, :2 * len(y)] = np.concatenate([y, -y])
    for scale in (0, 63, 100, -63, -110, 119, -124):
        t = torch.from_numpy(np.ldexp(rows, scale)).to(torch.bfloat16)
        assert torch.isfinite(t).all()
        check_rows(t, *rapid().rapid_quant_rows(t.cuda()), t.shape[1])


@pytest.mark.parametrize("eta", [0.0, 5.0])
def test_the_accept_pass_leaves_a_sum_that_is_nan_out(eta):
    """Ratios, tokens and counts are those with a chunk of no weight, on either side and on both; a chunk that does not hold the row's maximum."""
    B, g, vocab = 2, 3, 32000
    head = Head(np.random.default_rng(11), B * (2 * g + 1), 1024, vocab)
    logits, stats = rapid().rapid_lm_head_quant(head.h.cuda(), head.codes, head.scales)
    zt, zd = logits[:B * (g + 1)].reshape(B, g + 1, vocab).contiguous(), logits[B * (g + 1):].reshape(B, g, vocab).contiguous()
    st, sd = stats[:B * (g + 1)].contiguous(), stats[B * (g + 1):].contiguous()
    tokens, u = zd.argmax(-1).int(), torch.full((B, g + 1), 0.6, device="cuda")
    for sides in ((st,), (sd,), (st, sd)):
        results = []
        for weight in (0.0, float("nan")):
            t, d = st.clone(), sd.clone()
            for x in (y for y, z in ((t, st), (d, sd)) if any(z is s for s in sides)):
                for row in range(len(x)):
                    chunk = int(x[row, :, 0].argmin())
                    x[row, chunk, 1] = weight
            results.append(rapid().rapid_accept(zt, zd, tokens, eta, u, target_stats=t, draft_stats=d))
        for a, b in zip(*results):
            assert torch.equal(a, b) and torch.isfinite(a.double()).all()
