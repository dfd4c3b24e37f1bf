"""CPU checks of the drafter's entry points: what they refuse, before anything is launched, and the rounding rule of the 8-bit integers."""
import ctypes

import numpy as np
import pytest

from paper_2502_20330_amd import binding
from test_quant_prefix_abi import EALIGN, EINVAL, EUNSUPPORTED, EWORKSPACE, P, PAGED, ctx, shape


def rope_call(s, rope=None, quant=False, layout=None, **kw):
    lib = binding.load_library()
    rope = rope or binding.Rope(128, 0, 1.0, 8 * 128, 2 * 128, 2 * 128)
    p = dict(ctx=ctx(), q=P, k=P, v=P, freq=P, pos=None, lens=P, table=P if s.page_size else None, out=P, kc=P, vc=P, ks=P, vs=P)
    p.update(kw)
    new = (p["q"], p["k"], p["v"], p["freq"], p["pos"], p["lens"], None, p["table"], p["out"], p["kc"], p["vc"])
    if quant:
        return lib.rapid_kv_append_rope_quant(p["ctx"], s, layout or binding.QuantLayout(2 * 1008, 1008, 2 * 16), rope, *new, p["ks"], p["vs"],
                                              None)
    return lib.rapid_kv_append_rope(p["ctx"], s, rope, *new, None)


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("kw,want", [
    (dict(batch=0), EINVAL), (dict(q_max=0), EINVAL), (dict(n_q_heads=7), EINVAL), (dict(gamma=5), EINVAL), (dict(max_ctx=4), EINVAL),
    (dict(head_dim=96), EUNSUPPORTED), (dict(kv_token_stride=252), EALIGN), (dict(kv_head_stride=4), EALIGN), (dict(batch=70000), EUNSUPPORTED),
    (dict(PAGED, page_size=24), EUNSUPPORTED), (dict(PAGED, max_pages=62), EINVAL), (dict(n_pages=-1), EINVAL),
    (dict(kv_token_stride=1 << 62), EUNSUPPORTED), (dict(n_q_heads=1 << 17, n_kv_heads=1 << 15), None),
    (dict(PAGED, max_pages=1 << 26, max_ctx=1 << 30, q_max=(1 << 22) + 1, gamma=0), EUNSUPPORTED),
])
def test_shapes_that_the_append_refuses(quant, kw, want):
    s = shape(**kw)
    rope = binding.Rope(128, 0, 1.0, s.n_q_heads * 128, s.n_kv_heads * 128, s.n_kv_heads * 128)
    assert rope_call(s, rope, quant) == (EUNSUPPORTED if want is None else want)


@pytest.mark.parametrize("quant", [False, True])
def test_arguments_that_the_append_refuses(quant):
    R = binding.Rope
    for key in ("ctx", "k", "v", "freq", "lens", "kc", "vc", "q", "out") + (("ks", "vs") if quant else ()):
        assert rope_call(shape(), quant=quant, **{key: None}) == EINVAL, key          # (q and q_out go together)
    for key in ("q", "k", "v", "out", "kc", "vc") + (("ks", "vs") if quant else ()):
        assert rope_call(shape(), quant=quant, **{key: P + 8}) == EALIGN, key
    for key in ("freq", "pos"):
        assert rope_call(shape(), quant=quant, **{key: P + 2}) == EALIGN, key
    assert rope_call(shape(**PAGED), quant=quant, table=None) == EINVAL
    for rot in (0, 8, 24, 144, -16):
        assert rope_call(shape(), R(rot, 0, 1.0, 1024, 256, 256), quant) == EUNSUPPORTED, rot
    for strides in ((1016, 256, 256), (1024, 248, 256), (1024, 256, 248), (1028, 256, 256), (1024, 260, 256), (1024, 256, 1 << 30 | 4)):
        assert rope_call(shape(), R(128, 0, 1.0, *strides), quant) == EALIGN, strides
    for amplitude in (float("nan"), float("inf"), -float("inf")):
        assert rope_call(shape(), R(128, 0, amplitude, 1024, 256, 256), quant) == EINVAL
    assert rope_call(shape(), R(128, 2, 1.0, 1024, 256, 256), quant) == EINVAL
    if quant:
        assert rope_call(shape(), quant=True, layout=binding.QuantLayout(2016, 1000, 0)) == EALIGN


def rows_call(**kw):
    p = dict(ctx=ctx(), rows=5, cols=64, x=P, stride=64, codes=P, scales=P)
    p.update(kw)
    return binding.load_library().rapid_quant_rows(p["ctx"], p["rows"], p["cols"], p["x"], p["stride"], p["codes"], p["scales"], None)


def test_what_the_row_quantisation_refuses():
    for key in ("ctx", "x", "codes", "scales"):
        assert rows_call(**{key: None}) == EINVAL, key
    for kw in (dict(rows=0), dict(cols=0), dict(rows=-1), dict(stride=56)):
        assert rows_call(**kw) == EINVAL, kw
    for kw in (dict(rows=1 << 24), dict(cols=60), dict(cols=(1 << 17) + 8, stride=1 << 18)):
        assert rows_call(**kw) == EUNSUPPORTED, kw
    for kw in (dict(x=P + 8), dict(codes=P + 8), dict(scales=P + 2), dict(stride=68)):
        assert rows_call(**kw) == EALIGN, kw


def head_call(**kw):
    p = dict(ctx=ctx(), rows=9, hidden=512, vocab=1000, h=P, w=P, s=P, t=1.0, z=P, ldz=1000, stats=P, ws=P, nbytes=1 << 30)
    p.update(kw)
    return binding.load_library().rapid_lm_head_quant(p["ctx"], p["rows"], p["hidden"], p["vocab"], p["h"], p["w"], p["s"], p["t"], p["z"],
                                                      p["ldz"], p["stats"], p["ws"], p["nbytes"], None)


def test_what_the_head_refuses():
    lib = binding.load_library()
    for key in ("ctx", "h", "w", "s", "z"):
        assert head_call(**{key: None}) == EINVAL, key
    for kw in (dict(rows=0), dict(hidden=0), dict(vocab=0), dict(ldz=999), dict(t=0.0), dict(t=float("nan"))):
        assert head_call(**kw) == EINVAL, kw
    for kw in (dict(rows=97), dict(hidden=500), dict(hidden=(1 << 17) + 8), dict(vocab=15)):
        assert head_call(**kw) == EUNSUPPORTED, kw
    for kw in (dict(h=P + 8), dict(w=P + 8), dict(s=P + 2), dict(z=P + 2), dict(stats=P + 4)):
        assert head_call(**kw) == EALIGN, kw
    need = lib.rapid_lm_head_quant_workspace_bytes(None, 9, 512)
    assert need >= 9 * (512 + 4)
    for kw in (dict(ws=None), dict(ws=P + 16), dict(nbytes=need - 1)):
        assert head_call(**kw) == EWORKSPACE, kw
    for bad in ((0, 512), (97, 512), (9, 0), (9, 500), (9, (1 << 17) + 8)):
        assert lib.rapid_lm_head_quant_workspace_bytes(None, *bad) == 0


def test_the_structure_is_that_of_the_header():
    assert ctypes.sizeof(binding.Rope) == 40 and binding.Rope.q_stride.offset == 16


def test_quotients_of_32_bits_fall_on_the_right_side():
    """127 x / m, rounded to 32 bits and then to a whole number, is the rounding of the exact quotient, for every two significands of 8 bits and
    every power of two between them that matters; x = m is 127, and the borders go to the even code."""
    m = np.arange(128, 256)[:, None, None]
    x = np.arange(128, 256)[None, :, None]
    e = np.arange(0, 12)[None, None, :]
    keep = (x <= m) | (e > 0)
    got = np.rint((np.float32(127) * x.astype(np.float32) * np.float32(2.0) ** -e.astype(np.float32)) / m.astype(np.float32)).astype(np.int64)
    num, den = 127 * x, m << e                              # the exact quotient
    twice = 2 * num - (num // den) * 2 * den                # twice the rest, against den
    floor = num // den
    want = np.where(twice > den, floor + 1, np.where(twice < den, floor, floor + floor % 2))
    assert np.array_equal(np.where(keep, got, 0), np.where(keep, want, 0))
    assert (np.where(keep, got, 0) <= 127).all() and (got[np.arange(128), np.arange(128), 0] == 127).all()
    gap = np.where(twice == den, 1.0, np.abs(twice - den) / (2.0 * den))
    assert np.where(keep & (got > 0), gap, 1.0).min() >= 2.0 ** -17


@pytest.mark.parametrize("off", [0, 1, -1])
def test_quotients_by_the_reciprocal_fall_on_the_right_side(off):
    """The kernels' sequence for 127 x / m: r = t (1/m), then r + (t - r m) (1/m), each fused operation rounded once to 32 bits, and the whole number from the last bits of a
    sum with 1.5 * 2^23; for every two significands of 8 bits and every power of two between them that matters, also with a reciprocal that is one last place off."""
    f = np.float32
    wide = np.longdouble                                     # both fused operations are exact in 64 bits before they are rounded
    assert np.finfo(wide).nmant >= 63
    m = np.arange(128, 256)[:, None, None]
    x = np.arange(128, 256)[None, :, None]
    e = np.arange(0, 12)[None, None, :]
    keep = (x <= m) | (e > 0)
    inv = f(1) / m.astype(f)
    inv = inv if off == 0 else np.nextafter(inv, f(off) * f(np.inf))
    t = f(127) * x.astype(f) * f(2.0) ** -e.astype(f)
    r = t * inv
    rest = (t.astype(wide) - r.astype(wide) * m).astype(f)
    q = (r.astype(wide) + rest.astype(wide) * inv.astype(wide)).astype(f)
    assert inv.dtype == t.dtype == r.dtype == q.dtype == f
    got = (q + f(1.5 * 2 ** 23)).view(np.int32) & 0xff
    num, den = 127 * x, m << e
    floor, twice = num // den, 2 * (num % den)
    want = np.where(twice > den, floor + 1, np.where(twice < den, floor, floor + floor % 2))
    assert np.array_equal(np.where(keep, got, 0), np.where(keep, want, 0))
    # of the product with the reciprocal alone this is not so
    alone = np.rint(t * inv).astype(np.int64)
    assert off or not np.array_equal(np.where(keep, alone, 0), np.where(keep, want, 0))


def window_call(s, window=100, sinks=4, **kw):
    lib = binding.load_library()
    p = dict(ctx=ctx(), q=P, k=P, v=P, lens=P, table=P if s.page_size else None, out=P, ws=P, nbytes=1 << 40)
    p.update(kw)
    return lib.rapid_verify_attn_window(p["ctx"], s, window, sinks, p["q"], p["k"], p["v"], p["lens"], None, p["table"], p["out"], None,
                                        p["ws"], p["nbytes"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(batch=0), EINVAL), (dict(q_max=0), EINVAL), (dict(n_q_heads=7), EINVAL), (dict(gamma=5), EINVAL), (dict(max_ctx=4), EINVAL),
    (dict(softmax_scale=0.0), EINVAL), (dict(softmax_scale=float("nan")), EINVAL), (dict(chunk_tokens=-1), EINVAL), (dict(n_pages=-1), EINVAL),
    (dict(head_dim=96), EUNSUPPORTED), (dict(kv_token_stride=252), EALIGN), (dict(kv_head_stride=4), EALIGN), (dict(batch=70000), EUNSUPPORTED),
    (dict(PAGED, page_size=24), EUNSUPPORTED), (dict(PAGED, max_pages=62), EINVAL), (dict(kv_token_stride=1 << 62), EUNSUPPORTED),
    (dict(PAGED, max_pages=1 << 27, max_ctx=(1 << 30) + 1), EUNSUPPORTED), (dict(PAGED, max_pages=1 << 27, max_ctx=1 << 30, batch=64), EUNSUPPORTED),
    (dict(PAGED, max_pages=1 << 26, max_ctx=1 << 30, q_max=1 << 29, gamma=0), EUNSUPPORTED),
    (dict(PAGED, max_pages=1 << 26, max_ctx=1 << 30, q_max=1 << 24, gamma=0, batch=8, n_kv_heads=8), EUNSUPPORTED),
    (dict(PAGED, max_pages=1 << 26, max_ctx=1 << 30, q_max=1 << 22, gamma=0, batch=8, n_kv_heads=8), None),
])
def test_shapes_that_the_window_refuses(kw, want):
    s = shape(**kw)
    lib = binding.load_library()
    if want is None:
        assert window_call(s, ws=None) == EWORKSPACE and lib.rapid_verify_attn_window_workspace_bytes(None, s, 100, 4) > 0
        return
    assert window_call(s) == want
    assert lib.rapid_verify_attn_window_workspace_bytes(None, s, 100, 4) == 0


@pytest.mark.parametrize("Q", [5, 200])
def test_arguments_that_the_window_refuses(Q):
    s, lib = shape(q_max=Q, gamma=Q - 1), binding.load_library()
    for key in ("ctx", "q", "k", "v", "lens", "out"):
        assert window_call(s, **{key: None}) == EINVAL, key
    for key in ("q", "k", "v", "out"):
        assert window_call(s, **{key: P + 8}) == EALIGN, key
    assert window_call(shape(q_max=Q, gamma=Q - 1, **PAGED), table=None) == EINVAL
    for window, sinks in ((0, 4), (-1, 4), (100, -1)):
        assert window_call(s, window, sinks) == EINVAL
        assert lib.rapid_verify_attn_window_workspace_bytes(None, s, window, sinks) == 0
    need = lib.rapid_verify_attn_window_workspace_bytes(None, s, 100, 4)
    assert need > 0
    for kw in (dict(ws=None), dict(ws=P + 16), dict(nbytes=need - 1)):
        assert window_call(s, **kw) == EWORKSPACE, kw


def test_workspaces_of_the_window_are_bounded_whatever_the_sizes():
    """Partials are kept only where the row tiles do not fill the chip: never more than three rounds of workgroups of the largest tile."""
    lib = binding.load_library()
    rng = np.random.default_rng(1)
    for _ in range(300):
        d, hkv, group = int(rng.choice([64, 128])), int(rng.choice([1, 2, 4, 8])), int(rng.choice([1, 4, 7, 8]))
        ctx_max = int(2 ** rng.uniform(0, 20))
        q = int(max(1, min(ctx_max, 2 ** rng.uniform(0, 15))))
        s = binding.AttnShape(int(rng.integers(1, 20)), q, hkv * group, hkv, d, ctx_max, q - 1, 0.1, ctx_max * d * hkv, d, ctx_max * d, 0, 0, 0, 0, 0,
                              0)
        window, sinks = int(2 ** rng.uniform(0, 31)) - 1 or 1, int(2 ** rng.uniform(0, 31)) - 1
        need = lib.rapid_verify_attn_window_workspace_bytes(None, s, window, sinks)
        assert 256 <= need <= 3 * 256 * 384 * (d + 2) * 4 + 512
