"""Append with rotary positions and windowed attention at the ends of their ranges: device data outside of theirs, and the most sequences a call may have."""
import pytest
import torch

import quant_util as qu
from gpu_util import rapid
from test_gpu_window import i32

pytestmark = pytest.mark.gpu

MOST = 65535


def randn(shape, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("Q,hq,hkv", [(6, 8, 2), (300, 32, 8)])
def test_lengths_and_row_counts_are_brought_into_range(Q, hq, hkv, page):
    """Lengths below zero and beyond max_ctx, row counts below one and beyond Qmax, page ids that there are none of: the bits of the call with the nearest that there are."""
    cap, d, B = 704, 64, 4
    wild = [-5, cap + 1000, 333, (1 << 31) - 1], [Q - 1, 1 << 30, -7, Q]
    tame = [0, cap, 333, cap], [Q - 1, Q - 1, 0, Q - 1]
    table = None
    if page:
        table = torch.randperm(B * cap // page).reshape(B, -1).int()
        bad = table.clone()
        bad[table == table.max()], bad[table == 0] = 1 << 30, -9
        table, bad = table.cuda(), bad.cuda()
    shape = (B * cap // page, page, hkv, d) if page else (B, cap, hkv, d)
    q, k_new, v_new = randn((B, Q, hq, d), 1), randn((B, Q, hkv, d), 2), randn((B, Q, hkv, d), 3)
    freq = torch.arange(1, d // 2 + 1, device="cuda").float() ** -1.5
    codes = torch.zeros(shape, dtype=torch.uint8, device="cuda")
    scales = torch.zeros((shape[0], hkv, shape[1]), dtype=torch.uint8, device="cuda")
    r, results = rapid(), []
    for (lens, gammas), t in ((wild, bad if page else None), (tame, table)):
        kw = dict(gammas=i32(gammas), page_table=t, max_ctx=cap)
        k, v = randn(shape, 4), randn(shape, 5)
        q_out = torch.full_like(q, 7.0)
        r.rapid_kv_append_rope(k, v, k_new, v_new, freq, i32(lens), q_new=q, q_out=q_out, **kw)
        out = r.rapid_verify_attn_window(q_out, k, v, i32(lens), 100, sinks=3, **kw)
        small = [x.clone() for x in (codes, codes, scales, scales)]
        r.rapid_kv_append_rope_quant(*small, k_new, v_new, freq, i32(lens), **kw)
        results.append([q_out, k, v, out, *small])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert results[0][4].any() and torch.isfinite(results[0][3]).all()


@pytest.mark.parametrize("Q,hq", [(1, 1), (2, 3)])
def test_the_most_sequences(Q, hq):
    """65535 short ones: every result of the attention, and the appended rows of the last ones."""
    d, cap, window = 64, 16, 5
    q, k, v = randn((MOST, Q, hq, d), 1), randn((MOST, cap, 1, d), 2), randn((MOST, cap, 1, d), 3)
    lens = torch.randint(0, cap + 1, (MOST,), generator=torch.Generator().manual_seed(4)).int().cuda()
    out = rapid().rapid_verify_attn_window(q, k, v, lens, window, sinks=2)
    pos = lens[:, None, None] - Q + torch.arange(Q, device="cuda")[None, :, None]
    j = torch.arange(cap, device="cuda")[None, None]
    seen = ((j <= pos) & ((j > pos - window) | (j < 2)))[:, None]              # [B, 1, Q, tokens]
    qd, kd, vd = q.double().transpose(1, 2), k[:, None, :, 0].double(), v[:, None, :, 0].double()
    # (products of 64 bits as sums, three dimensions at a time)
    s = torch.stack([(qd * kd[:, :, t, None]).sum(-1) for t in range(cap)], -1) * d ** -0.5
    reach = torch.stack([(qd.abs() * kd[:, :, t, None].abs()).sum(-1) for t in range(cap)], -1).masked_fill(~seen, 0).amax(-1) * d ** -0.5
    s = s.masked_fill(~seen, -torch.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-1e300))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-300)
    ref = sum(p[..., t, None] * vd[:, :, t, None] for t in range(cap))
    weight = sum(p[..., t, None] * vd[:, :, t, None].abs() for t in range(cap))
    flat = lambda x: x.transpose(1, 2).reshape(MOST * Q * hq, -1).cpu().numpy()
    ref, weight, reach = flat(ref), flat(weight), flat(reach[..., None])[:, 0]
    qu.close(out.reshape(MOST * Q * hq, d), ref, qu.tolerance(ref, weight, reach, d, cap))

    freq = torch.arange(1, d // 2 + 1, device="cuda").float() ** -1.0
    k_new, v_new, last = randn((MOST, Q, 1, d), 5), randn((MOST, Q, 1, d), 6), slice(MOST - 100, MOST)
    all_q = torch.zeros_like(q)
    before = k[last].clone(), v[last].clone(), torch.zeros_like(q[last])
    rapid().rapid_kv_append_rope(k, v, k_new, v_new, freq, lens, q_new=q, q_out=all_q)
    rapid().rapid_kv_append_rope(*before[:2], k_new[last], v_new[last], freq, lens[last].clone(), q_new=q[last], q_out=before[2])
    assert torch.equal(k[last], before[0]) and torch.equal(v[last], before[1]) and torch.equal(all_q[last], before[2])
