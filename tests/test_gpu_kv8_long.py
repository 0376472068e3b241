"""Attention over the 8-bit cache where sequences are cut into long ranges or many: the ranges that the device chose, and rows of every head against 64 bits."""
import numpy as np
import pytest
import torch

import kv8_model as m
import kv8_plan_model as pm
from paper_2511_16665_amd import binding as tlt

pytestmark = pytest.mark.gpu
GUARD = 4096


@pytest.mark.parametrize("kernel,Hq,Hkv,n,lens,longest_range,most_ranges", [
    ("few", 28, 4, 1, [8192] * 16, 17, 8),                                # a batch that fills the chip: the search, ranges of 16 and 17 tiles
    ("few", 28, 4, 4, [9000, 12001, 7000, 64, 8000, 20000, 4095, 4096], 9, 35),
    ("few", 28, 4, 1, [45000], 10, 71),                                   # more than 64 ranges: a second turn of the join
    ("few", 8, 1, 1, [200000], 21, 149),                                  # and a third
    ("mid", 28, 4, 16, [8192] * 16, 17, 8),
    ("mid", 40, 20, 40, [20000, 9000, 3], 20, 16),
    ("many", 28, 4, 48, [19000, 12000, 700, 4100, 30, 9000], 12, 25),     # three tiles of rows a wave
    ("many", 96, 32, 64, [20001, 5000], 53, 6),                           # two, and ranges that wrap the stages many times
    ("many", 64, 8, 64, [30000, 11000], 43, 11),                          # two groups of row tiles
    ("many", 160, 32, 64, [20001, 5000], 53, 6),                          # three, long ranges
])
def test_long_ranges(kernel, Hq, Hkv, n, lens, longest_range, most_ranges):
    B, d, total = len(lens), 128, max(lens) + n
    rng = np.random.default_rng(n)
    c = pm.long_cache(lens, n, Hkv, seed=n)
    c.upload()
    plan = pm.plan(B, n, Hq, Hkv, total)
    first, k = pm.segments(lens, n, plan)
    tiles = -(-(np.array(lens) + n) // 64)
    assert plan.kernel == kernel and plan.planned and int((-(-tiles // k)).max()) == longest_range and int(k.max()) == most_ranges
    q = torch.from_numpy(rng.standard_normal((B, n, Hq, d)).astype(np.float32) * 0.7).bfloat16()
    mask = m.random_trees(rng, B, n)[1]
    # workspace and output inside larger buffers, of exactly the size that is asked for
    need = tlt.load().tlt_kv8_attention_workspace_bytes(B, n, Hq, Hkv, d, total)
    store = torch.full((need + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    outs = torch.full((B * n * Hq * d + 2 * GUARD,), 7.0, dtype=torch.bfloat16, device="cuda")
    ws, out = store[GUARD:GUARD + need], outs[GUARD:-GUARD].view(B, n, Hq * d)
    pools = [t.clone() for t in (c.kv.k_exp, c.kv.v_exp)]
    print("long ranges", kernel, Hq, Hkv, n, lens[:3], flush=True)
    x, mk = q.view(B, n, Hq * d).cuda(), torch.from_numpy(mask.view(np.int64)).cuda()
    tlt.kv8_attention(tlt.TLT_BF16, Hq, x, mk, c.kv, 0, out, ws)
    torch.cuda.synchronize()
    seg = ws[:8 * B].view(torch.int32).view(B, 2).cpu().numpy()
    np.testing.assert_array_equal(seg[:, 1], k)
    np.testing.assert_array_equal(seg[:, 0], first)
    for t in (store[:GUARD], store[-GUARD:]):
        assert (t == 0xA5).all()
    for t in (outs[:GUARD], outs[-GUARD:]):
        assert (t == 7.0).all()
    assert all(torch.equal(a, b) for a, b in zip(pools, (c.kv.k_exp, c.kv.v_exp)))
    got, q64 = out.view(B, n, Hq, d).double().cpu().numpy(), q.double().numpy()
    worst = 0.0
    for b in sorted({0, B // 2, B - 1}):
        for h in sorted({0, Hq // 2 + 1, Hq - 1}):
            nodes = sorted({0, n // 2, n - 1})
            want, tol = pm.attention_rows(c, b, q64[b, nodes, h], mask[b], nodes, h, Hq // Hkv)
            err = np.abs(got[b, nodes, h] - want)
            assert (err <= tol).all(), (b, h, float((err / tol).max()))
            worst = max(worst, float((err / tol).max()))
    print(f"  worst share of what is allowed: {worst:.3f}", flush=True)
    # every row against the kernel that cuts nothing: with values up to 3.5 they are within 3 * 2^-8 * 3.5 and 2^-8 * 3.5 of the definition, and what scores add,
    # 2 ds * 3.5, is below 2^-8 (136 * 2^-24 of a score's magnitudes, some 10)
    whole = torch.empty_like(out)
    tlt.kv8_attention(tlt.TLT_BF16, Hq, x, mk, c.kv, 0, whole, ws, 0)
    assert float((whole.float() - out.float()).abs().max()) < 2.0 ** -6 * 3.75
    again = torch.empty_like(out)
    tlt.kv8_attention(tlt.TLT_BF16, Hq, x, mk, c.kv, 0, again, ws)
    assert torch.equal(again, out)
