"""The 8-bit cache at the ends of what its rows can hold: the largest finite rows, the smallest values, scores that are not finite."""
import numpy as np
import pytest
import torch

import kv8_model as m
from paper_2511_16665_amd import binding as tlt
from test_gpu_kv8 import DTYPE, check_attention, cuda, run_attention, run_write

pytestmark = pytest.mark.gpu
TOP = 3.3895313892515355e38      # bf16's largest number, 255 * 2^120


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64), ("fp32", 256)])
def test_the_largest_rows_are_read_as_finite(dtype, d):
    """Rows from 448 * 2^119 on have the largest exponent.  Their values come back within 2^-4 of what was written: half a step of e4m3, or, from 248 * 2^120 on,
    where the nearest code would be 2^128, the code below it, 240 * 2^120 (at most 16 / 256 off)."""
    Hkv = 3
    rows = np.array([np.where(np.arange(d) % 2, TOP, -TOP), np.where(np.arange(d) == 5, -248 * 2.0 ** 120, np.arange(d) * 2.0 ** 119 / d),
                     np.where(np.arange(d) == d - 1, 247 * 2.0 ** 120, 1.0)])
    x = np.zeros((1, 1, 3 * Hkv, d), np.float32)
    x[0, 0, Hkv:2 * Hkv] = x[0, 0, 2 * Hkv:] = rows
    code, dt, _ = DTYPE[dtype]
    c = m.Cache([0], 1, Hkv, d, 16)
    print("the largest rows", dtype, d, flush=True)
    run_write(c, dtype, Hkv, x.reshape(1, 1, -1), None, None, 1e4)
    held = torch.from_numpy(x[0, 0, Hkv:2 * Hkv]).to(dt).double().numpy()
    for out_type in ("bf16", "fp32"):
        out = [torch.full((1, 1, 1, Hkv, d), 5.0, dtype=DTYPE[out_type][1], device="cuda") for _ in range(2)]
        tlt.kv8_read(DTYPE[out_type][0], c.kv, cuda(np.zeros(1, np.int32)), None, *out)
        for o in out:
            got = o[0, 0, 0].double().cpu().numpy()
            assert np.isfinite(got).all()
            # (a subnormal code is off by half of its step, 2^-10 * 2^120, at most)
            assert (np.abs(got - held) <= np.maximum(2.0 ** -4 * np.abs(held), 2.0 ** 110)).all()
            assert (np.abs(got[0]) == 240 * 2.0 ** 120).all() and got[1, 5] == -240 * 2.0 ** 120 and got[2, d - 1] == 240 * 2.0 ** 120


@pytest.mark.parametrize("dtype,Hq,Hkv,d,n,impl", [("bf16", 28, 4, 128, 2, -1), ("bf16", 28, 4, 128, 4, -1), ("bf16", 28, 4, 128, 16, -1), ("bf16", 28, 4, 128, 24, -1),
                                                   ("bf16", 28, 4, 128, 48, -1), ("bf16", 28, 4, 128, 4, 0), ("fp32", 4, 2, 64, 6, -1)])
@pytest.mark.parametrize("ctx", [0, 150])
def test_the_largest_rows_reach_only_the_rows_that_see_them(dtype, Hq, Hkv, d, n, ctx, impl):
    """Nodes whose key or value is of the largest: a row that does not see them is finite and right, and keeps its bits where only values are (a score moves
    the reference that a row's exponentials are taken from for all 16 rows of a tile: their weights are rounded anew, within the model's bound).  Seen
    with a weight of one, or with a score of zero, they count as finite."""
    rng = np.random.default_rng(n + ctx)
    c = m.Cache([ctx, 70], n, Hkv, d, 16, seed=9)
    q = rng.standard_normal((2, n, Hq, d)).astype(np.float32)
    q64 = torch.from_numpy(q).to(DTYPE[dtype][1]).double().numpy()
    own = np.tile(np.uint64(1) << np.arange(n, dtype=np.uint64), (2, 1))             # every row sees itself
    print("rows that do not see the largest", dtype, Hq, Hkv, n, ctx, impl, flush=True)
    clean = run_attention(c, dtype, q, own, impl=impl)
    top = [np.where(np.arange(d) % 2, TOP, -TOP), np.where(np.arange(d) == 7, TOP, 1.0)]
    slots = [(0, "v", ctx + n - 1, 0, top[0]), (0, "k", ctx, 1, top[1]), (1, "v", 70 + n // 2, Hkv - 1, top[1]), (1, "k", 70 + n - 1, 0, top[0])]
    G = Hq // Hkv
    seen = torch.zeros((2, n, Hkv), dtype=torch.bool)
    for what in ("v", "k"):
        for b, x, slot, h, row in slots:
            if x == what:
                codes, e = m.encode(row[None])
                assert e[0] == 247 and 0x78 in codes[0] & 0x7f
                pg = c.table[b, slot // 16]
                c.codes[x][0, pg, h, slot % 16], c.exps[x][0, pg, h, slot % 16] = codes[0], e[0]
                seen[b, slot - int(c.ctx[b]), h] = True
        c.upload()
        got = run_attention(c, dtype, q, own, impl=impl)
        unseen = (~seen).repeat_interleave(G, 2)
        assert torch.isfinite(got.cpu()[unseen]).all()
        assert what == "k" or torch.equal(got.cpu()[unseen], clean.cpu()[unseen])
        for b in range(2):
            want, tol = m.attention(c, b, q64[b], own[b], rounded=dtype == "bf16")
            on = unseen[b].numpy()
            assert (np.abs(got[b].double().cpu().numpy() - want)[on] <= tol[on]).all(), b
    if ctx == 0:        # row n - 1 sees its own value alone
        want = np.where(np.arange(d) % 2, 1.0, -1.0) * 240 * 2.0 ** 120
        np.testing.assert_array_equal(got[0, n - 1, :G].double().cpu().numpy(), np.tile(want, (G, 1)))
    # queries of zero: every key has a score of zero, whatever it holds
    for b, x, slot, h, row in slots:
        if x == "v":
            pg = c.table[b, slot // 16]
            c.exps[x][0, pg, h, slot % 16] = 120
    c.exps["k"][0, :, :, ::3], c.codes["k"][0, :, :, ::3] = 247, m.encode(top[0][None])[0][0]
    c.upload()
    check_attention(c, dtype, q * 0, own, run_attention(c, dtype, q * 0, own, impl=impl))


@pytest.mark.parametrize("dtype,Hq,Hkv,d,n,impl", [("bf16", 28, 4, 128, 1, -1), ("bf16", 28, 4, 128, 4, -1), ("bf16", 28, 4, 128, 16, -1), ("bf16", 28, 4, 128, 24, -1),
                                                   ("bf16", 28, 4, 128, 48, -1), ("bf16", 28, 4, 128, 4, 0), ("fp32", 4, 2, 64, 6, -1)])
def test_scores_of_minus_infinity_alone_are_not_nothing(dtype, Hq, Hkv, d, n, impl):
    """A row whose visible scores are all -infinity has no softmax: NaN, as the definition gives, in one range or several, in the context or among the new rows.
    A row that sees nothing is zeros whatever its query; the others are right (they need not keep their bits: scores move the references of a tile's 16 rows)."""
    ctxs = [90, 0, 3000]
    c = m.Cache(ctxs, n, Hkv, d, 16, seed=9)
    c.codes["k"][..., 0] = 0x38                          # 1.0: times -infinity, and the other products finite
    c.upload()
    q = np.random.default_rng(n).standard_normal((3, n, Hq, d)).astype(np.float32)
    mask = np.tile(np.uint64(1) << np.arange(n, dtype=np.uint64), (3, 1))
    mask[1, n // 2:] = 0
    print("scores of -infinity", dtype, Hq, Hkv, n, impl, flush=True)
    q64 = torch.from_numpy(q).to(DTYPE[dtype][1]).double().numpy()
    q[:, :, 1, 0], q[:, n - 1, Hq - 1, 0] = -np.inf, -np.inf
    got = run_attention(c, dtype, q, mask, impl=impl).cpu()
    bad = torch.zeros((3, n, Hq), dtype=torch.bool)
    bad[:, :, 1], bad[:, n - 1, Hq - 1] = True, True
    blind = torch.from_numpy((mask == 0) & (np.array(ctxs) == 0)[:, None])[..., None].expand(-1, -1, Hq)
    assert not got[blind].any() and blind.any()
    assert torch.isnan(got[bad & ~blind]).all()
    for b in range(3):
        want, tol = m.attention(c, b, q64[b], mask[b], rounded=dtype == "bf16")
        ok = ~bad[b].numpy()
        assert (np.abs(got[b].double().numpy() - want)[ok] <= tol[ok]).all(), b


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_the_smallest_values(dtype):
    """Exponents 1 to 9: exact in fp32, whose smallest number is 2^-149; in bf16 rounded to its smallest number, 2^-133, below 2^-125."""
    c = m.Cache([140], 1, 2, 128, 16, seed=4)
    rng = np.random.default_rng(0)
    for x in ("k", "v"):
        c.exps[x][:] = rng.integers(1, 10, c.exps[x].shape)
        c.codes[x][..., :32] = np.concatenate([np.arange(16), 128 + np.arange(16)])
    c.upload()
    code, dt, _ = DTYPE[dtype]
    out = [torch.full((1, 1, 140, 2, 128), 5.0, dtype=dt, device="cuda") for _ in range(2)]
    print("the smallest values", dtype, flush=True)
    tlt.kv8_read(code, c.kv, cuda(np.zeros(1, np.int32)), None, *out)
    for x, o in zip(("k", "v"), out):
        want = c.rows(x, 0, 0, 0, 140)
        if dtype == "bf16":
            want = np.where(np.abs(want) < 2.0 ** -125, np.rint(want * 2.0 ** 133) * 2.0 ** -133, want)
            assert (want != c.rows(x, 0, 0, 0, 140)).any()
        np.testing.assert_array_equal(o[0, 0].double().cpu().numpy(), want)
