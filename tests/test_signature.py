"""The key of a call's tensors: equal for tensors that the checks cannot tell apart, different for any others."""
import itertools

import pytest
import torch

from paper_2502_20330_amd import binding


def test_every_property_counts():
    x = torch.zeros((4, 6, 8))
    some = [x, x.bfloat16(), x.half(), x.int(), x[:, :, :4], x[:, :4], x[:2], x.transpose(0, 1), x.transpose(0, 1).contiguous(), x.reshape(24, 8),
            x.reshape(24, 8)[:, None], x.to("meta"), torch.zeros(()), torch.zeros(1), torch.zeros(0), torch.zeros((0, 5)), x.view(torch.uint8),
            x.view(torch.float8_e4m3fn), x.view(torch.float8_e8m0fnu), None]
    keys = [binding._sizes(t) for t in some]
    assert len(set(keys)) == len(keys)
    assert binding._sizes(x) == binding._sizes(torch.ones((4, 6, 8)))
    pairs = [binding._sizes(a, b) for a, b in itertools.product(some, some)]
    assert len(set(pairs)) == len(pairs) and not set(pairs) & set(keys)
    assert binding._sizes() == b""


def test_what_is_no_tensor():
    for bad in (1, "a", [torch.zeros(1)], torch.zeros((1,) * 9), torch.zeros((2, 2)).to_sparse()):
        with pytest.raises(TypeError):
            binding._sizes(bad)
    with pytest.raises(ValueError):
        binding._sizes(*[None] * 33)
