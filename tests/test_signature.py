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


class NoSizes(torch.Tensor):
    """A subclass whose sizes are asked for in Python, where there is an error."""
    @staticmethod
    def __new__(cls):
        return torch.Tensor._make_wrapper_subclass(cls, (2, 3), dispatch_sizes_strides_policy="sizes")

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise ValueError("no sizes")


def test_what_torch_throws_is_an_exception():
    """Tensors whose sizes or strides torch refuses to give: an error like any other, and the process lives."""
    rows = [torch.zeros((2, 3)), torch.zeros((4, 3))]
    for layout in (torch.strided, torch.jagged):
        with pytest.raises(TypeError):
            binding._sizes(torch.zeros(2), torch.nested.nested_tensor(rows, layout=layout))
    with pytest.raises(ValueError, match="no sizes"):
        binding._sizes(torch.zeros(2), NoSizes())
    assert binding._sizes(torch.zeros(2), None) == binding._sizes(torch.ones(2), None)
