"""What the binding keeps from one call for the next, by sizes: nothing that a tensor's content decides."""
import numpy as np
import pytest
import torch

import quant_util as qu
from gpu_util import rapid
from test_gpu_prefix import Batch, i32

pytestmark = pytest.mark.gpu


def test_sizes_and_scales_are_numbers_of_the_host():
    """A tensor in the place of a number could change its value between two calls without a trace in its sizes: refused, on either device."""
    from paper_2502_20330_amd import binding
    rng = np.random.default_rng(1)
    r = rapid()
    kc, vc, ks, vs, _ = qu.QuantCache(rng, [64], 2, 64).dev()
    n, q, new = i32([64]), qu.bf16(rng, (1, 3, 4, 64)).cuda(), qu.bf16(rng, (1, 3, 2, 64)).cuda()
    args, kw = Batch(rng, 70, [20], 2, 64).args("token")
    for device in ("cpu", "cuda"):
        two, scale = torch.tensor(2, device=device), torch.tensor(0.1, device=device)
        bad = [lambda: r.rapid_verify_attn_quant(q, kc, vc, ks, vs, n, two),
               lambda: r.rapid_verify_attn_quant(q, kc, vc, ks, vs, n, max_ctx=two + 62),
               lambda: r.rapid_verify_attn_quant(q, kc, vc, ks, vs, n, softmax_scale=scale),
               lambda: r.rapid_kv_append_quant(kc, vc, ks, vs, new, new, n, two),
               lambda: r.rapid_kv_read_quant(kc, vc, ks, vs, n, 3, two),
               lambda: r.rapid_verify_attn_prefix(q, *args, two, **kw),
               lambda: r.rapid_verify_attn_prefix(q, *args, softmax_scale=scale, **kw),
               lambda: r.rapid_verify_attn_prefix(q, *args, **dict(kw, max_prefix=two + 68))]
        for i, call in enumerate(bad):
            with pytest.raises(binding.RapidError):
                call()
                pytest.fail(f"call {i} was taken")


def test_calls_of_the_same_sizes_differ_by_their_numbers():
    """Every number of a call is part of what is kept: calls that differ in one of them alone give what a fresh object gives."""
    from paper_2502_20330_amd import binding
    rng = np.random.default_rng(2)
    kc, vc, ks, vs, _ = qu.QuantCache(rng, [64, 64], 2, 64).dev()
    n, q = i32([64, 50]), qu.bf16(rng, (2, 3, 4, 64)).cuda()
    args, kw = Batch(rng, 70, [20, 9], 2, 64).args("token")
    some = [lambda r, x=x: r.rapid_verify_attn_quant(q, kc, vc, ks, vs, n, **x)
            for x in ({}, dict(gamma=1), dict(max_ctx=40), dict(softmax_scale=0.5), dict(gammas=i32([0, 2])))]
    some += [lambda r, x=x: r.rapid_verify_attn_prefix(q, *args, **dict(kw, **x))
             for x in ({}, dict(gamma=1), dict(max_ctx=12), dict(softmax_scale=0.5), dict(max_prefix=33), dict(gammas=i32([0, 2])))]
    some += [lambda r, x=x: torch.cat(r.rapid_kv_read_quant(kc, vc, ks, vs, n, 3, **x)) for x in ({}, dict(gamma=1), dict(max_ctx=48))]
    want = [call(binding.Rapid(0)) for call in some]
    assert all(not torch.equal(a, b) for i, a in enumerate(want) for b in want[:i] if a.shape == b.shape)
    one = rapid()
    for _ in range(2):
        for call, w in zip(some, want):
            assert torch.equal(call(one), w)
