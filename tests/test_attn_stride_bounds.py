"""CPU checks: token strides whose products pass 64 bits are refused by every call that takes an rapid_attn_shape."""
import ctypes

import pytest

from paper_2502_20330_amd import binding
from test_quant_prefix_abi import PAGED, prefix_call, quant_call, shape


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("stride", [1 << 28, 1 << 40, 1 << 61, 1 << 62, (1 << 63) - 16])
def test_huge_token_strides_are_refused(stride, paged):
    s = shape(kv_token_stride=stride, **(PAGED if paged else {}))
    lib = binding.load_library()
    no_prefix = binding.PrefixLayout(0, 0, 0, 0)
    assert prefix_call(s, no_prefix, kp=None, vp=None, ws=None) == binding.RAPID_EUNSUPPORTED
    assert lib.rapid_verify_attn_prefix_workspace_bytes(None, s, no_prefix) == 0
    assert lib.rapid_verify_attn_workspace_bytes(None, ctypes.byref(s)) == 0
    assert lib.rapid_verify_attn_chunk(None, ctypes.byref(s)) == binding.RAPID_EUNSUPPORTED
    assert quant_call("attn", s, ws=None) == binding.RAPID_EUNSUPPORTED


@pytest.mark.parametrize("span,stride,taken", [(1000, 2147480, True), (1000, 2147488, False), (1024, (1 << 21) - 8, True), (1024, 1 << 21, False)])
def test_the_bound_is_4_gib_of_a_sequence(span, stride, taken):
    """2 bytes an element: stride * 2 * tokens stays below 2^32."""
    need = binding.load_library().rapid_verify_attn_workspace_bytes(None, ctypes.byref(shape(max_ctx=span, kv_token_stride=stride)))
    assert (need > 0) == taken == (stride * 2 * span < 1 << 32)
