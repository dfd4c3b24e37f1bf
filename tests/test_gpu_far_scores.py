"""Scores far from zero, in the attention over a cache in 8 bits and behind a shared prefix: products with the scale that have more bits than
a 32-bit number holds, of either sign, beside ordinary rows."""
import numpy as np
import pytest
import torch

import quant_util as qu
from gpu_util import rapid
from test_gpu_prefix import Batch, i32

pytestmark = pytest.mark.gpu

# factors of K and q that no power of two divides into 1, so that score * scale is rounded: scores near 2^45, 2^62 and 2^111
FACTORS = [(1.5 * 2.0 ** 20, 1.25 * 2.0 ** 18), (1.375 * 2.0 ** 30, 1.125 * 2.0 ** 25), (1.5 * 2.0 ** 50, 1.25 * 2.0 ** 54)]


def equal_weights(out, lse, vals, score, d, what):
    """Rows whose scores are all the same number: the mean of the values.  Weights of 1 are exact; 32-bit sums of them, and the rounding of the result."""
    n = len(vals)
    tol = 2 * n * 2.0 ** -24 * np.abs(vals).mean(0) + 2.0 ** -8 * np.abs(vals.mean(0))
    qu.close(out, vals.mean(0), tol, what)
    want = np.array([score + np.log(n)])
    qu.close(lse.reshape(1), want, qu.lse_tolerance(want, np.abs(want), d, n), what + " lse")


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("k,q", FACTORS)
@pytest.mark.parametrize("n", [1, 100, 3000])
@pytest.mark.parametrize("d", [64, 128])
def test_equal_scores_over_a_cache_in_8_bits(d, n, k, q, sign):
    rng = np.random.default_rng(n)
    cache = qu.QuantCache(rng, [n], 1, d)
    cache.put("k", 0, np.arange(n), *qu.quantise(np.full((n, 1, d), sign * k)))
    kc, vc, ks, vs, _ = cache.dev()
    lse = torch.empty((1, 4, 1), device="cuda")
    out = rapid().rapid_verify_attn_quant(torch.full((1, 1, 4, d), q, dtype=torch.bfloat16, device="cuda"), kc, vc, ks, vs, i32([n]), lse_out=lse)
    equal_weights(out[0, 0, 3], lse[0, 3].double().cpu().numpy(), cache.tokens("v", 0)[:, 0], sign * k * q * d ** 0.5, d, f"{n} keys")


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("k,q", FACTORS)
@pytest.mark.parametrize("B,Q,P,bound", [(2, 1, 200, 200), (5, 6, 33, 900), (8, 9, 300, 26000)])
def test_equal_scores_behind_a_prefix(B, Q, P, bound, k, q, sign):
    """The last with more rows than the streaming kernel takes at a time, and enough of them for the kernel of many rows."""
    rng = np.random.default_rng(B)
    d, n = 128, 20
    batch = Batch(rng, P, [n] * B, 4, d, prefix_cap=bound)
    for x in [batch.shared["k"], *batch.own["k"]]:
        x.fill_(sign * k)
    batch.store()
    args, kw = batch.args("token")
    lse = torch.empty((B, 16, Q), device="cuda")
    out = rapid().rapid_verify_attn_prefix(torch.full((B, Q, 16, d), q, dtype=torch.bfloat16, device="cuda"), *args, lse_out=lse, **kw)
    for b in (0, B - 1):
        for h in (0, 3, 15):
            vals = torch.cat([batch.shared["v"], batch.own["v"][b][:n]])[:, h // 4].double().numpy()
            equal_weights(out[b, Q - 1, h], lse[b, h, Q - 1].double().cpu().numpy(), vals, sign * k * q * d ** 0.5, d, f"sequence {b} head {h}")


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("n", [40, 700])
def test_one_key_above_the_others(n, sign):
    """Its score is the largest by an eighth: it has all the weight."""
    rng = np.random.default_rng(n)
    d = 64
    x = np.full((n, 1, d), sign * 1.5 * 2.0 ** 20)
    x[7] = sign * 1.5 * 2.0 ** 20 * (1 + sign / 8)
    x = torch.from_numpy(x).to(torch.bfloat16).double().numpy()
    cache = qu.QuantCache(rng, [n], 1, d)
    cache.put("k", 0, np.arange(n), *qu.quantise(x))
    kc, vc, ks, vs, _ = cache.dev()
    q = torch.full((1, 1, 4, d), 1.25 * 2.0 ** 18, dtype=torch.bfloat16, device="cuda")
    out = rapid().rapid_verify_attn_quant(q, kc, vc, ks, vs, i32([n]))
    assert np.array_equal(out[0, 0, 1].double().cpu().numpy(), cache.tokens("v", 0)[7, 0])


def test_ordinary_rows_beside_far_ones_keep_their_bits():
    """A row's result does not depend on what the others hold: some rows' q is 2^40 times as large, and those rows are finite too."""
    rng = np.random.default_rng(5)
    cache = qu.QuantCache(rng, [1500], 2, 128)
    dev = cache.dev()
    q = qu.bf16(rng, (1, 5, 8, 128))
    far = q.clone()
    far[0, 1::2] *= 2.0 ** 40
    outs, lses = [], []
    for x in (q, far):
        lses.append(torch.empty((1, 8, 5), device="cuda"))
        outs.append(rapid().rapid_verify_attn_quant(x.cuda(), *dev[:4], i32([1500]), lse_out=lses[-1]))
    assert torch.equal(outs[0][:, ::2], outs[1][:, ::2]) and torch.equal(lses[0][..., ::2], lses[1][..., ::2])
    assert torch.isfinite(outs[1]).all() and torch.isfinite(lses[1]).all()
    batch = Batch(rng, 700, [30, 5], 2, 128)
    args, kw = batch.args("token")
    q = qu.bf16(rng, (2, 5, 8, 128))
    far = q.clone()
    far[:, 1::2] *= 2.0 ** 40
    outs = [rapid().rapid_verify_attn_prefix(x.cuda(), *args, **kw) for x in (q, far)]
    assert torch.equal(outs[0][:, ::2], outs[1][:, ::2]) and torch.isfinite(outs[1]).all()
