"""rapid_verify_attn_prefix under bounds far above the lengths: a capacity in the place of a length (the binding's default) divides the chip no
differently, which shows in results of the same bits.  (Beyond 96 rows a kv head the bound of the prefix also chooses the kernel.)"""
import numpy as np
import pytest
import torch

import quant_util as qu
from gpu_util import rapid
from test_gpu_prefix import Batch, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,Q,P", [([300, 17, 0, 250], 5, 9000), ([40, 9], 3, 0), ([2500, 1000, 700], 4, 65), ([9] * 70, 1, 2000)])
def test_a_capacity_as_the_bound_changes_no_bit(lens, Q, P, d):
    rng = np.random.default_rng(P + d)
    B, hq, hkv, page = len(lens), 8, 2, 16
    batch = Batch(rng, P, lens, hkv, d, page, cap=max(lens), prefix_cap=max(P, 1))
    q = qu.bf16(rng, (B, Q, hq, d))
    gammas = [int(x) for x in rng.integers(0, Q, B)]
    (k, v, n, length), kw = batch.args("token")
    wide = lambda t, pages: torch.cat([t, torch.full((*t.shape[:-1], pages - t.shape[-1]), -1, dtype=torch.int32, device="cuda")], -1)
    lses = [torch.empty((B, hq, Q), device="cuda") for _ in range(4)]
    call = lambda i, **more: rapid().rapid_verify_attn_prefix(q.cuda(), k, v, n, length, gammas=i32(gammas), lse_out=lses[i], **dict(kw, **more))
    tight = call(0)
    batch.compare(q, tight, lses[0], gammas)
    table = wide(kw["page_table"], 8192)                      # 128K tokens a sequence
    prefix = wide(kw["prefix_table"], 4096)
    loose = [call(1, page_table=table, max_ctx=None), call(2, prefix_table=prefix, max_prefix=None),
             call(3, page_table=table, max_ctx=None, prefix_table=prefix, max_prefix=None)]
    for out, lse in zip(loose, lses[1:]):
        batch.compare(q, out, lse, gammas)
    same = (1, 2, 3) if B * Q * hq // hkv <= 96 else (1,)
    assert all(torch.equal(loose[i - 1], tight) and torch.equal(lses[i], lses[0]) for i in same)
    assert torch.equal(loose[1], loose[2]) and torch.equal(lses[2], lses[3])


@pytest.mark.parametrize("B,Q,hq,hkv,d,P", [(200, 2, 32, 8, 64, 300), (100, 2, 32, 8, 128, 900), (3, 2, 300, 300, 64, 500), (40, 2, 64, 16, 128, 65),
                                            (130, 1, 8, 1, 64, 1500), (2, 24, 128, 32, 64, 1)])
def test_more_row_tiles_or_heads_than_there_is_room_for(B, Q, hq, hkv, d, P):
    """From one row tile a head on one compute unit for each to 34 row tiles on 32 units a head, sequences without tokens among them."""
    rng = np.random.default_rng(B)
    lens, gammas = [int(x) for x in rng.integers(0, 300, B)], [int(x) for x in rng.integers(0, Q, B)]
    lens[0], lens[-1], some = 299, 0, sorted({0, 1, B // 2, B - 1})
    batch = Batch(rng, P, lens, hkv, d, 16)
    q, lses = qu.bf16(rng, (B, Q, hq, d)), [torch.empty((B, hq, Q), device="cuda") for _ in range(2)]
    (k, v, n, length), kw = batch.args("head")
    kw.pop("max_prefix")
    out = rapid().rapid_verify_attn_prefix(q.cuda(), k, v, n, length, gammas=i32(gammas), lse_out=lses[0], **kw)
    whole = {x: [torch.cat([batch.shared[x], batch.own[x][b]]).double().numpy() for b in some] for x in "kv"}
    qu.check_attention(q[some], out[some], lses[0][some], lambda b, h: (whole["k"][b][:, h * hkv // hq], whole["v"][b][:, h * hkv // hq], P),
                       [gammas[b] for b in some], d ** -0.5, [lens[b] for b in some])
    kw["max_ctx"] = None
    kw["page_table"] = torch.cat([kw["page_table"], torch.full((B, 500), -1, dtype=torch.int32, device="cuda")], -1)
    again = rapid().rapid_verify_attn_prefix(q.cuda(), k, v, n, length, gammas=i32(gammas), lse_out=lses[1], **kw)
    assert torch.equal(out, again) and torch.equal(lses[0], lses[1])
