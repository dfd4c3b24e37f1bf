"""CPU checks of the entry points for a cache in 8 bits and for a shared prefix: what they refuse, before anything is launched, and the
format that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

import quant_util as qu
from paper_2502_20330_amd import binding

P = 0x10000                                              # an address that is never followed: every call here is refused first
EINVAL, EALIGN, EUNSUPPORTED, EWORKSPACE = -1, -2, -3, -4


def shape(**kw):
    s = binding.AttnShape(2, 5, 8, 2, 128, 1000, 4, 0.1, 1000 * 256, 256, 128, 0, 0, 0, 0, 0, 0)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


PAGED = dict(page_size=16, max_pages=63, kv_page_stride=16 * 256, kv_batch_stride=0)


def ctx():
    return ctypes.create_string_buffer(4096)             # stands for a context: nothing is read from it before a call is accepted


def quant_call(name, s, layout=None, **kw):
    lib = binding.load_library()
    layout = layout or binding.QuantLayout(2 * 1008, 1008, 2 * 16)
    p = dict(q=P, k=P, v=P, ks=P, vs=P, lens=P, table=P if s.page_size else None, out=P, ws=P, nbytes=1 << 40, ctx=ctx(), rows=P)
    p.update(kw)
    if name == "attn":
        return lib.rapid_verify_attn_quant(p["ctx"], s, layout, p["q"], p["k"], p["v"], p["ks"], p["vs"], p["lens"], None, p["table"],
                                           p["out"], None, p["ws"], p["nbytes"], None)
    if name == "append":
        return lib.rapid_kv_append_quant(p["ctx"], s, layout, p["rows"], p["rows"], p["lens"], None, p["table"], p["k"], p["v"], p["ks"],
                                         p["vs"], None)
    return lib.rapid_kv_read_quant(p["ctx"], s, layout, p["k"], p["v"], p["ks"], p["vs"], p["lens"], None, p["table"], p["rows"],
                                   p["rows"], None)


@pytest.mark.parametrize("name", ["attn", "append", "read"])
@pytest.mark.parametrize("kw,want", [
    (dict(batch=0), EINVAL), (dict(q_max=0), EINVAL), (dict(n_kv_heads=0), EINVAL), (dict(n_q_heads=7), EINVAL), (dict(gamma=5), EINVAL),
    (dict(gamma=-1), EINVAL), (dict(max_ctx=0), EINVAL), (dict(max_ctx=4), EINVAL), (dict(n_pages=-1), EINVAL),
    (dict(chunk_tokens=-1), EINVAL), (dict(ctx_sum_hint=-1), EINVAL), (dict(batch=40000), EUNSUPPORTED),
    (dict(head_dim=96), EUNSUPPORTED), (dict(kv_token_stride=264), EALIGN), (dict(kv_token_stride=112), EALIGN),
    (dict(kv_head_stride=72), EALIGN), (dict(kv_batch_stride=8), EALIGN), (dict(PAGED, page_size=24), EUNSUPPORTED),
    (dict(PAGED, page_size=8), EUNSUPPORTED), (dict(PAGED, max_pages=62), EINVAL), (dict(PAGED, kv_page_stride=8), EALIGN),
    (dict(max_ctx=1 << 24, kv_token_stride=256), EUNSUPPORTED),
])
def test_shapes_that_are_refused(name, kw, want):
    assert quant_call(name, shape(**kw)) == want
    if name == "attn":
        assert binding.load_library().rapid_verify_attn_quant_workspace_bytes(None, shape(**kw)) == 0


@pytest.mark.parametrize("name", ["attn", "append", "read"])
def test_pointers_and_layouts_that_are_refused(name):
    s = shape()
    for key in ("ctx", "k", "v", "ks", "vs", "lens") + (("q", "out") if name == "attn" else ("rows",)):
        assert quant_call(name, s, **{key: None}) == EINVAL, key
    for key in ("k", "v", "ks", "vs") + (("q", "out") if name == "attn" else ("rows",)):
        assert quant_call(name, s, **{key: P + 8}) == EALIGN, key
    assert quant_call(name, shape(**PAGED), table=None) == EINVAL
    assert quant_call(name, s, binding.QuantLayout(2016, 1000, 0)) == EALIGN
    assert quant_call(name, s, binding.QuantLayout(2008, 1008, 0)) == EALIGN
    assert quant_call(name, shape(**PAGED), binding.QuantLayout(1, 16, 24)) == EALIGN


def test_attention_alone_is_held_to_rows_scale_and_workspace():
    need = binding.load_library().rapid_verify_attn_quant_workspace_bytes(None, shape())
    assert need > 0
    assert quant_call("attn", shape(q_max=25, gamma=24)) == EUNSUPPORTED          # 100 rows a kv head
    assert quant_call("attn", shape(softmax_scale=0.0)) == EINVAL
    assert quant_call("attn", shape(softmax_scale=float("nan"))) == EINVAL
    assert quant_call("attn", shape(), ws=None) == EWORKSPACE
    assert quant_call("attn", shape(), ws=P + 16) == EWORKSPACE
    assert quant_call("attn", shape(), nbytes=need - 1) == EWORKSPACE


def prefix_call(s, prefix=None, **kw):
    lib = binding.load_library()
    prefix = prefix or binding.PrefixLayout(500, 0, 256, 128)
    p = dict(q=P, kp=P, vp=P, n=P, pt=None, k=P, v=P, lens=P, table=P if s.page_size else None, out=P, ws=P, nbytes=1 << 40, ctx=ctx())
    p.update(kw)
    return lib.rapid_verify_attn_prefix(p["ctx"], s, prefix, p["q"], p["kp"], p["vp"], p["n"], p["pt"], p["k"], p["v"], p["lens"], None,
                                        p["table"], p["out"], None, p["ws"], p["nbytes"], None)


def test_what_the_prefix_call_refuses():
    lay = binding.PrefixLayout
    for key in ("ctx", "q", "kp", "vp", "n", "k", "v", "lens", "out"):
        assert prefix_call(shape(), **{key: None}) == EINVAL, key
    for key in ("q", "kp", "vp", "k", "v", "out"):
        assert prefix_call(shape(), **{key: P + 8}) == EALIGN, key
    assert prefix_call(shape(head_dim=96)) == EUNSUPPORTED
    assert prefix_call(shape(q_max=25, gamma=24)) == EUNSUPPORTED
    assert prefix_call(shape(), lay(-1, 0, 256, 128)) == EINVAL
    assert prefix_call(shape(), lay(500, 0, 252, 128)) == EALIGN
    assert prefix_call(shape(), lay(500, 0, 256, 4)) == EALIGN
    assert prefix_call(shape(), lay(500, 0, 64, 128)) == EALIGN
    assert prefix_call(shape(), lay(1 << 24, 0, 256, 128)) == EUNSUPPORTED
    assert prefix_call(shape(), pt=P, kp=None, vp=None) == EINVAL                 # no pages to name
    assert prefix_call(shape(**PAGED), lay(500, 40, 0, 0), pt=P) == EINVAL        # both
    assert prefix_call(shape(**PAGED), lay(500, 31, 0, 0), pt=P, kp=None, vp=None) == EINVAL
    assert prefix_call(shape(), ws=None) == EWORKSPACE
    need = binding.load_library().rapid_verify_attn_prefix_workspace_bytes(None, shape(), lay(500, 0, 256, 128))
    assert need > 0 and prefix_call(shape(), nbytes=need - 1) == EWORKSPACE
    assert prefix_call(shape(), ws=P + 16) == EWORKSPACE
    assert binding.load_library().rapid_verify_attn_prefix_workspace_bytes(None, shape(), lay(-1, 0, 256, 128)) == 0
    assert binding.load_library().rapid_verify_attn_prefix_workspace_bytes(None, shape(head_dim=32), lay(1, 0, 256, 128)) == 0


def test_bounds_of_the_positions():
    lib, lay = binding.load_library(), binding.PrefixLayout
    wide = dict(PAGED, max_pages=1 << 27)
    for kw in (dict(wide, max_ctx=(1 << 30) + 1), dict(wide, max_ctx=1 << 30, batch=64), dict(kv_token_stride=1 << 62)):
        assert quant_call("attn", shape(**kw)) == EUNSUPPORTED
    assert quant_call("attn", shape(**dict(wide, max_ctx=1 << 30)), ws=None) == EWORKSPACE
    assert quant_call("append", shape(kv_token_stride=1 << 62)) == EUNSUPPORTED
    for kw in (dict(wide, max_ctx=(1 << 30) + 1), dict(wide, max_ctx=1 << 30, batch=64)):
        assert prefix_call(shape(**kw)) == EUNSUPPORTED
    assert prefix_call(shape(**PAGED), lay((1 << 30) + 1, 1 << 27, 0, 0), kp=None, vp=None, pt=P) == EUNSUPPORTED
    assert prefix_call(shape(), lay(500, 0, 1 << 62, 128)) == EUNSUPPORTED


def test_no_prefix_needs_no_layout():
    assert prefix_call(shape(), binding.PrefixLayout(0, 0, 0, 0), kp=None, vp=None, ws=None) == EWORKSPACE


def test_the_format_of_the_tests_is_torch_s_e4m3():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(qu.e4m3_values(codes), want, equal_nan=True)
    y = np.concatenate([np.linspace(-448, 448, 100001), qu.POSITIVE[:-1] + np.diff(qu.POSITIVE) / 2, [-0.0, 0.0]]).astype(np.float32)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(qu.e4m3_codes(y.astype(np.float64)), want)


def test_scales_of_the_format():
    """The smallest power of two that keeps the largest value within 448, on both sides of its borders."""
    for top, k in ((448.0, 0), (450.0, 1), (224.0, -1), (1.75, -8), (1.7578125, -7), (2.0 ** -133, -100), (3.3895e38, 119), (0.0, -100)):
        x = torch.tensor([[0.0, -top, top / 4]], dtype=torch.bfloat16).double().numpy()
        codes, scales = qu.quantise(x)
        assert int(scales[0]) - 127 == k, top
        assert np.abs(qu.e4m3_values(codes)).max() <= 448
