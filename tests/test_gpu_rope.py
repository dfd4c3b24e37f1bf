"""rapid_kv_append_rope and rapid_kv_append_rope_quant: rotation on the way into the cache, against the rotation in 64 bits."""
import numpy as np
import pytest
import torch

import quant_util as qu
from gpu_util import rapid

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def frequencies(rot, base=500000.0):
    return torch.tensor(base ** (-2.0 * np.arange(rot // 2) / rot), dtype=torch.float32)


def rotation(x, pos, freq, interleaved, amplitude):
    """x [rows, heads, d] (float64), pos [rows] -> (rotated, the same with |cos| + |sin| = 1 and |x|: what errors of cos and sin act on)."""
    half = len(freq)
    y, size = x.copy(), np.zeros_like(x)
    c = np.arange(half)
    l, r = (2 * c, 2 * c + 1) if interleaved else (c, c + half)
    turns = pos.astype(np.float64)[:, None] * freq.double().numpy()
    cos, sin = np.cos(turns)[:, None], np.sin(turns)[:, None]
    a, b = x[..., l], x[..., r]
    y[..., l], y[..., r] = amplitude * (a * cos - b * sin), amplitude * (b * cos + a * sin)
    size[..., l] = size[..., r] = abs(amplitude) * (np.abs(a) + np.abs(b))
    return y, size


def tolerance(ref, size, pos):
    """The angle in half turns is rounded to 32 bits (2^-25 of a half turn, 2^-23 in radians), sin and cos are within 2 ulp, 2^-22 at most, and take
    the amplitude, a product and a sum round by 2^-24 each: under 2^-20 in all.  The angle's product in 64 bits rounds by 2.5 * 2^-53 of it, the
    reference's by 2^-53 (frequencies are at most 1): together less than 2^-51 of the position.  The result is rounded to bf16, half a step
    is 2^-8 of it."""
    return 2.0 ** -8 * np.abs(ref) + (2.0 ** -20 + np.abs(pos.astype(np.float64))[:, None, None] * 2.0 ** -51) * size + 1e-37


class Case:
    def __init__(self, rng, lens, gammas, Q, hq, hkv, d, rot=None, page=0, cap=None, fused=False, scale=1.0):
        self.lens, self.gammas, self.Q, self.hq, self.hkv, self.d, self.page = list(lens), list(gammas), Q, hq, hkv, d, page
        self.cap = cap or max(max(lens), Q)
        self.freq = frequencies(rot or d)
        B = len(lens)
        if fused:
            x = qu.bf16(rng, (B, Q, hq + 2 * hkv + 1, d), scale)         # (and a head that nobody asks for)
            self.q, self.k, self.v = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:hq + 2 * hkv]
        else:
            self.q, self.k, self.v = (qu.bf16(rng, (B, Q, h, d), scale) for h in (hq, hkv, hkv))
        self.fused = fused
        if page:
            self.table, n = qu.page_table(rng, [self.cap] * B, page)
            self.shape = (n, page, hkv, d)
        else:
            self.table, self.shape = None, (B, self.cap, hkv, d)

    def news(self):
        if not self.fused:
            return [t.cuda() for t in (self.q, self.k, self.v)]
        x = self.q._base.cuda()
        h = self.hq
        return [x[:, :, :h], x[:, :, h:h + self.hkv], x[:, :, h + self.hkv:h + 2 * self.hkv]]

    def place(self, b, j):
        return (np.full(len(j), b), j) if self.table is None else (self.table[b, j // self.page], j % self.page)

    def rows(self, b):
        """The rows that exist and have a token, and their tokens."""
        n = self.gammas[b] + 1
        i = np.arange(n)
        j = min(self.lens[b], self.cap) - n + i
        return i[j >= 0], j[j >= 0]

    def run(self, layout="token", quant=False, q_out=None, queries=True, positions=None, interleaved=False, amplitude=1.0):
        q, k, v = self.news()
        table = None if self.table is None else torch.from_numpy(self.table).cuda()
        kw = dict(gammas=i32(self.gammas), page_table=table, max_ctx=self.cap, interleaved=interleaved, amplitude=amplitude)
        if positions is not None:
            kw["positions"] = torch.from_numpy(positions).cuda()
        if queries:
            q_out = torch.full(q.shape, 3.0, dtype=torch.bfloat16, device="cuda") if q_out is None else q_out
            kw.update(q_new=q, q_out=q_out)
        if not quant:
            cache = [qu.laid_out(torch.full(self.shape, 5.0, dtype=torch.bfloat16, device="cuda"), layout) for _ in "kv"]
            got = rapid().rapid_kv_append_rope(*cache, k, v, self.freq.cuda(), i32(self.lens), **kw)
            return got, cache
        cache = [qu.laid_out(torch.full(self.shape, 9, dtype=torch.uint8, device="cuda"), layout) for _ in "kv"]
        slots = -(-self.shape[1] // 16) * 16
        cache += [torch.full((self.shape[0], self.hkv, slots), 77, dtype=torch.uint8, device="cuda") for _ in "kv"]
        got = rapid().rapid_kv_append_rope_quant(*cache, k, v, self.freq.cuda(), i32(self.lens), **kw)
        return got, cache

    def check(self, layout="token", queries=True, positions=None, interleaved=False, amplitude=1.0):
        q_out, cache = self.run(layout, False, None, queries, positions, interleaved, amplitude)
        k_cache, v_cache = (t.double().cpu().numpy() for t in cache)
        assert (q_out is None) == (not queries)
        want_v = np.full(self.shape, 5.0)
        for b in range(len(self.lens)):
            i, j = self.rows(b)
            pos = j if positions is None else positions[b, i]
            at = self.place(b, j)
            ref, size = rotation(self.k[b].double().numpy()[i], pos, self.freq, interleaved, amplitude)
            qu.close(k_cache[at], ref, tolerance(ref, size, pos), f"keys of {b}")
            k_cache[at] = 5.0
            want_v[at] = self.v[b].double().numpy()[i]
            if queries:
                ref, size = rotation(self.q[b].double().numpy()[i], pos, self.freq, interleaved, amplitude)
                got = q_out[b].double().cpu().numpy()
                qu.close(got[i], ref, tolerance(ref, size, pos), f"queries of {b}")
                assert (np.delete(got, i, 0) == 3.0).all()               # rows that do not exist
        assert (k_cache == 5.0).all() and np.array_equal(v_cache, want_v)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (128, 16), (64, 64), (64, 48), (64, 16)])
def test_both_pairings_and_every_part_of_a_head(d, rot, interleaved):
    rng = np.random.default_rng(d + rot)
    Case(rng, [300, 40, 7], [4, 2, 0], 5, 6, 2, d, rot).check(interleaved=interleaved)


@pytest.mark.parametrize("page,layout", [(0, "token"), (0, "head"), (0, "wide"), (16, "token"), (16, "head"), (64, "wide")])
@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("d,hq,hkv", [(128, 28, 4), (64, 4, 1), (128, 64, 8)])
def test_layouts_and_ragged_batches(page, layout, fused, d, hq, hkv):
    """Lengths from none on, sequences shorter than their rows, a length above the bound, a call without queries."""
    rng = np.random.default_rng(page + d + fused)
    case = Case(rng, [130, 0, 3, 16, 65, 900], [6, 2, 4, 0, 3, 6], 7, hq, hkv, d, page=page, cap=150, fused=fused)
    case.check(layout)
    case.check(layout, queries=False)


@pytest.mark.parametrize("B,Q,hq,hkv,d,page", [(1, 2048, 8, 2, 128, 0), (3, 1111, 4, 1, 64, 16), (2, 1025, 7, 7, 128, 64), (1, 2051, 14, 2, 64, 0)])
def test_prompts(B, Q, hq, hkv, d, page):
    """Enough rows for four to a workgroup; some sequences have fewer."""
    rng = np.random.default_rng(Q)
    lens = [Q + 100 - 60 * b for b in range(B)]
    case = Case(rng, lens, [Q - 1 - 301 * b for b in range(B)], Q, hq, hkv, d, page=page, fused=B > 1)
    case.check("head")
    case.check("token", interleaved=True, amplitude=0.7)


def test_positions_of_their_own():
    """Near and far ones, equal ones, and below zero."""
    rng = np.random.default_rng(3)
    case = Case(rng, [50, 60], [4, 4], 5, 4, 2, 128)
    pos = np.array([[0, 1, 131071, 131071, 1 << 24], [(1 << 31) - 1, -5, -(1 << 31), 7, 7]], np.int32)
    case.check(positions=pos, amplitude=1.25)


def test_angles_far_from_zero_keep_their_differences():
    """Scores of rotated rows depend on differences of positions alone: at 2^20 and at 0, to the rounding of the rows."""
    rng = np.random.default_rng(4)
    case = Case(rng, [8], [7], 8, 1, 1, 128)
    one = np.arange(8, dtype=np.int32)[None]
    near, far = (case.run(positions=p)[0][0, :, 0].double().cpu().numpy() for p in (one, one + (1 << 20)))
    size = np.linalg.norm(case.q[0, :, 0].double().numpy(), axis=1)
    # each row is off by half a bf16 step, 2^-8 of an element, on either side of two products
    assert np.abs(near @ near.T - far @ far.T).max() <= 4.1 * 2.0 ** -8 * size.max() ** 2


def test_queries_in_place():
    rng = np.random.default_rng(5)
    case = Case(rng, [40, 2500], [4, 2047], 2048, 4, 2, 64)
    want, _ = case.run()
    q, k, v = case.news()
    cache = [torch.zeros(case.shape, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    got = rapid().rapid_kv_append_rope(*cache, k, v, case.freq.cuda(), i32(case.lens), gammas=i32(case.gammas), q_new=q, q_out=q)
    assert got.data_ptr() == q.data_ptr()
    for b, g in enumerate(case.gammas):
        assert torch.equal(got[b, :g + 1], want[b, :g + 1])
        assert torch.equal(got[b, g + 1:].cpu(), case.q[b, g + 1:])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_pair(bad):
    rng = np.random.default_rng(6)
    case = Case(rng, [20], [2], 3, 2, 2, 64)
    case.k[0, 1, 0, 5] = bad
    case.v[0, 0, 1, 9] = bad
    _, (k, v) = case.run()
    j = 20 - 3
    assert not torch.isfinite(k[0, j + 1, 0, [5, 37]]).any()
    k[0, j + 1, 0, [5, 37]] = 0
    assert torch.isfinite(k).all() and (~torch.isfinite(v)).sum() == 1


@pytest.mark.parametrize("page,layout", [(0, "token"), (0, "head"), (16, "wide"), (64, "head")])
@pytest.mark.parametrize("d,rot,interleaved", [(128, 128, False), (64, 32, True), (64, 64, False), (128, 32, True)])
@pytest.mark.parametrize("Q", [6, 2048])
def test_eight_bit_cache_is_that_of_the_rotated_rows(page, layout, d, rot, interleaved, Q):
    """Byte for byte what rapid_kv_append_quant writes of the rows that rapid_kv_append_rope writes; queries are the same bits."""
    rng = np.random.default_rng(Q + d)
    lens, gammas = [Q + 40, 3, Q], [Q - 1, 4, Q // 2]
    case = Case(rng, lens, gammas, Q, 6, 2, d, rot, page=page, fused=True)
    case.k[0, 1, 0, 3] = float("nan")
    case.v[0, 2, 1, 4] = float("-inf")
    case.k[0, 0] = 0
    case.v[0, 0] *= 2.0 ** 120
    case.k[2, 0, 1] *= 2.0 ** -120
    q1, cache = case.run("token", interleaved=interleaved)
    q2, codes = case.run(layout, quant=True, interleaved=interleaved)
    assert torch.equal(q1, q2)
    # rows as appended, read back from the bf16 cache
    k, v = (torch.zeros((3, Q, 2, d), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    for b in range(3):
        i, j = case.rows(b)
        at = tuple(torch.from_numpy(x).cuda() for x in case.place(b, j))
        k[b, i], v[b, i] = cache[0][at], cache[1][at]
    want = [qu.laid_out(torch.full(case.shape, 9, dtype=torch.uint8, device="cuda"), layout) for _ in "kv"]
    want += [torch.full_like(codes[2], 77) for _ in "kv"]
    table = None if case.table is None else torch.from_numpy(case.table).cuda()
    rapid().rapid_kv_append_quant(*want, k, v, i32(lens), gammas=i32(gammas), page_table=table, max_ctx=case.cap)
    for a, b, name in zip(codes, want, ("k", "v", "k scales", "v scales")):
        assert torch.equal(a, b), name


def test_captured_calls_follow_their_lengths():
    """One graph, replayed as lengths and positions change, with eager calls between."""
    rng = np.random.default_rng(8)
    case = Case(rng, [100, 90], [3, 3], 4, 4, 2, 128, page=16, cap=128)
    q, k, v = case.news()
    lens, freq, table = i32(case.lens), case.freq.cuda(), torch.from_numpy(case.table).cuda()
    cache = [torch.zeros(case.shape, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    out = torch.zeros_like(q)
    call = lambda c, o: rapid().rapid_kv_append_rope(*c, k, v, freq, lens, page_table=table, max_ctx=128, q_new=q, q_out=o)
    call(cache, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(cache, out)
    for turn in range(4):
        lens.copy_(i32([100 + 4 * turn, 90 + turn]))
        q.normal_()
        graph.replay()
        torch.cuda.synchronize()
        eager = [torch.zeros_like(t) for t in cache], torch.zeros_like(q)
        call(*eager)
        for b in range(2):
            j = np.arange(int(lens[b]) - 4, int(lens[b]))
            at = case.place(b, j)
            at = tuple(torch.from_numpy(x).cuda() for x in at)
            assert torch.equal(cache[0][at], eager[0][0][at]) and torch.equal(cache[1][at], eager[0][1][at])
        assert torch.equal(out, eager[1])


def test_on_another_stream():
    rng = np.random.default_rng(9)
    case = Case(rng, [100, 90], [3, 2], 4, 4, 2, 128)
    want, cache = case.run()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got, other = case.run()
    side.synchronize()
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(cache, other))
