"""The 8-bit cache's operators (tlt_kv8_*) against float64 on the host: writing, attention, commit and read, each by itself and as a step."""
import numpy as np
import pytest
import torch

import kv8_model as m
from paper_2511_16665_amd import binding as tlt

pytestmark = pytest.mark.gpu
DTYPE = {"fp32": (tlt.TLT_F32, torch.float32, 2.0 ** -24), "bf16": (tlt.TLT_BF16, torch.bfloat16, 2.0 ** -8)}
cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()


def download(c):
    """The cache's device contents into a copy of its host model."""
    torch.cuda.synchronize()
    for x, pool, exp in (("k", c.kv.k_pool, c.kv.k_exp), ("v", c.kv.v_pool, c.kv.v_exp)):
        c.codes[x], c.exps[x] = pool.cpu().numpy(), exp.cpu().numpy()
    return c


# ---- write

def run_write(c, dtype, Hq, qkv, bias, depth, theta, layer=0, in_place=False):
    code, dt, _ = DTYPE[dtype]
    d = c.kv.k_pool.shape[-1]
    x = cuda(qkv).to(dt)
    q = x[..., :Hq * d] if in_place else torch.full((*x.shape[:2], Hq * d), 9.0, dtype=dt, device="cuda")
    tlt.kv8_write(code, Hq, theta, x, None if bias is None else cuda(bias).to(dt), None if depth is None else cuda(depth), c.kv, layer, q)
    return q.float().cpu().numpy().astype(np.float64), x


@pytest.mark.parametrize("dtype,Hq,Hkv,d,n,ctxs,page,with_bias,with_depth", [
    ("bf16", 28, 4, 128, 1, [8191], 16, True, True),
    ("bf16", 40, 8, 128, 13, [0, 1, 15, 16, 300], 16, True, True),
    ("bf16", 7, 1, 64, 5, [31, 100000], 16, False, False),
    ("bf16", 6, 2, 192, 3, [7, 40], 5, True, True),
    ("bf16", 2, 2, 256, 2, [0, 2000000], 64, True, False),
    ("bf16", 64, 8, 128, 70, [3, 500], 16, False, False),     # more rows than a tree has
    ("fp32", 4, 2, 64, 5, [128, 0], 16, True, True),
    ("fp32", 3, 3, 128, 4, [30000], 16, False, True),
    ("fp32", 5, 1, 256, 1, [77, 78, 79], 1, True, False),
])
def test_write(dtype, Hq, Hkv, d, n, ctxs, page, with_bias, with_depth):
    """Queries and cached values against the rotation in 64 bits.  fp32 rotates with errors of 4 * 2^-24 of |lo| + |hi| at most (two products, a sum, cosine and
    sine, the bias); a query is then off by half a step of its type, a value by half a step of e4m3."""
    print("write", dtype, Hq, Hkv, d, n, ctxs, flush=True)
    B, theta = len(ctxs), 1e6
    rng = np.random.default_rng(d + n)
    pages_for = [min(x, 4000) for x in ctxs]
    c = m.Cache(pages_for, n, Hkv, d, page, layers=2, seed=n)
    if pages_for != list(ctxs):      # far positions by way of the tree's depths: the slots stay near
        far = np.array([x - y for x, y in zip(ctxs, pages_for)], np.int32)
    else:
        far = np.zeros(B, np.int32)
    depth = (m.random_trees(rng, B, n)[0] if n <= 64 else np.tile(np.arange(n, dtype=np.int32), (B, 1))) if with_depth or far.any() else None
    if depth is not None:
        depth = depth + far[:, None]
    before = {x: (c.codes[x].copy(), c.exps[x].copy()) for x in ("k", "v")}
    half_of = lambda a: torch.from_numpy(a.astype(np.float32)).to(DTYPE[dtype][1]).double().numpy()
    qkv = half_of(rng.standard_normal((B, n, (Hq + 2 * Hkv) * d)) * 2)
    bias = half_of(rng.standard_normal((Hq + 2 * Hkv) * d)) if with_bias else None
    q, _ = run_write(c, dtype, Hq, qkv.astype(np.float32), None if bias is None else bias.astype(np.float32), depth, theta, layer=1)
    download(c)
    x = (qkv + (0 if bias is None else bias)).reshape(B, n, Hq + 2 * Hkv, d)
    pos = c.ctx[:, None] + (np.arange(n)[None] if depth is None else depth)
    ang = pos[..., None].astype(np.float64) * theta ** (-np.arange(0, d, 2) / d)
    cos, sin = np.cos(ang)[:, :, None], np.sin(ang)[:, :, None]
    lo, hi = x[..., : d // 2], x[..., d // 2:]
    rot = np.concatenate([lo * cos - hi * sin, hi * cos + lo * sin], -1)
    slack = 4 * 2.0 ** -24 * np.tile(np.abs(lo) + np.abs(hi), 2)
    want_q = rot[:, :, :Hq].reshape(B, n, -1)
    assert (np.abs(q - want_q) <= DTYPE[dtype][2] * np.abs(want_q) + 2 * slack[:, :, :Hq].reshape(B, n, -1)).all()
    touched = {"k": np.zeros(c.exps["k"].shape[1:], bool), "v": np.zeros(c.exps["v"].shape[1:], bool)}
    for name, want, sl in (("k", rot[:, :, Hq:Hq + Hkv], slack[:, :, Hq:Hq + Hkv]), ("v", x[:, :, Hq + Hkv:], 2.0 ** -24 * np.abs(x[:, :, Hq + Hkv:]))):
        for b in range(B):
            for i in range(n):
                slot = int(c.ctx[b]) + i
                pg, r = c.table[b, slot // page], slot % page
                touched[name][pg, :, r] = True
                codes, e = c.codes[name][1, pg, :, r], c.exps[name][1, pg, :, r].astype(np.float64) - 127
                w, s = want[b, i], sl[b, i]
                amax, am_s = np.abs(w).max(-1), s.max(-1)
                assert (448 * np.exp2(e) >= amax - am_s).all() and (448 * np.exp2(e - 1) <= amax + am_s).all()
                got = m.decode(codes, c.exps[name][1, pg, :, r])
                step = np.exp2(np.floor(np.log2(np.maximum(np.abs(w) / np.exp2(e)[:, None], 2.0 ** -6))) - 3 + e[:, None])
                assert (np.abs(got - w) <= step / 2 + s).all(), (name, b, i)
        # every other row, and the other layer, are as they were
        np.testing.assert_array_equal(c.codes[name][1][~touched[name]], before[name][0][1][~touched[name]])
        np.testing.assert_array_equal(c.exps[name][1][~touched[name]], before[name][1][1][~touched[name]])
        np.testing.assert_array_equal(c.codes[name][0], before[name][0][0])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_write_is_the_format_to_the_bit(dtype):
    """At position zero nothing turns: codes and exponents are the definition's, for values on ties and borders, subnormals, zeros, rows that are not finite."""
    d, Hq, Hkv = 128, 4, 4
    rng = np.random.default_rng(5)
    rows = [np.concatenate([(m.POSITIVE[:-1] + m.POSITIVE[1:])[:127] / 2, [448.0, -448.0]])[:d],       # ties
            rng.standard_normal(d) * 2.0 ** -100, rng.standard_normal(d) * 2.0 ** 100, np.zeros(d), np.full(d, -0.0),
            np.where(np.arange(d) == 3, 448.0, 1e-3 * rng.standard_normal(d)), np.where(np.arange(d) == 3, 456.0, 2.0 ** -9 * rng.standard_normal(d)),
            np.where(np.arange(d) == 100, np.inf, 1.0), np.where(np.arange(d) == 64, np.nan, 1.0), np.where(np.arange(d) == 0, -np.inf, np.nan),
            np.full(d, 3.3895313892515355e38), np.full(d, 2.0 ** -126), np.full(d, 2.0 ** -133), rng.standard_normal(d), rng.standard_cauchy(d), np.full(d, 1.0)]
    vals = torch.from_numpy(np.array(rows)).to(DTYPE[dtype][1])
    B = len(rows) // Hkv
    x = torch.zeros((B, 1, Hq + 2 * Hkv, d), dtype=DTYPE[dtype][1])
    x[:, 0, Hq:Hq + Hkv] = vals.view(B, Hkv, d)
    x[:, 0, Hq + Hkv:] = vals.flip(0).view(B, Hkv, d)
    c = m.Cache([0] * B, 1, Hkv, d, 16)
    print("write to the bit", dtype, flush=True)
    run_write(c, dtype, Hq, x.view(B, 1, -1).float().numpy(), None, None, 1e4)
    download(c)
    for name, want in (("k", vals), ("v", vals.flip(0))):
        codes, exps = m.encode(want.double().numpy().reshape(B, Hkv, d))
        for b in range(B):
            np.testing.assert_array_equal(c.exps[name][0, c.table[b, 0], :, 0], exps[b])
            got = c.codes[name][0, c.table[b, 0], :, 0]
            if name == "k":                                       # (x * 1 - y * 0: a zero's sign may turn)
                got, codes[b] = np.where(got == 128, 0, got), np.where(codes[b] == 128, 0, codes[b])
            np.testing.assert_array_equal(got, codes[b])


def test_write_in_place_and_without_pages():
    """q_out inside qkv; rows whose page is missing are rotated and not written."""
    d, Hq, Hkv, n = 128, 8, 2, 5
    c = m.Cache([30, 30], n, Hkv, d, 16, seed=2)
    rng = np.random.default_rng(0)
    qkv = rng.standard_normal((2, n, (Hq + 2 * Hkv) * d)).astype(np.float32)
    q, _ = run_write(c, "bf16", Hq, qkv, None, None, 1e6)
    kept = {x: c.kv.__dict__[x].clone() for x in ("k_pool", "v_pool", "k_exp", "v_exp")}
    q2, whole = run_write(c, "bf16", Hq, qkv, None, None, 1e6, in_place=True)
    np.testing.assert_array_equal(q, q2)
    assert torch.equal(whole[..., Hq * d:].float().cpu(), torch.from_numpy(qkv[..., Hq * d:]).bfloat16().float())
    c.kv.block_table[0, 2], c.kv.block_table[1, 2] = -1, c.kv.k_pool.shape[1]     # rows 2 .. 4 of both: slots 32 .. 34
    q3, _ = run_write(c, "bf16", Hq, qkv * 2, None, None, 1e6)
    np.testing.assert_array_equal(q3, 2 * q)
    for b in range(2):
        pg = int(c.table[b, 2])
        assert all(torch.equal(c.kv.__dict__[x][0, pg], kept[x][0, pg]) for x in kept)


def test_one_row_of_queries_inside_their_projection():
    """With one node the queries' rows are as far apart as the sequences are."""
    d, Hq, Hkv = 128, 4, 2
    for B in (1, 3):
        c = m.Cache([20 + b for b in range(B)], 1, Hkv, d, 16, seed=2)
        qkv = np.random.default_rng(0).standard_normal((B, 1, (Hq + 2 * Hkv) * d)).astype(np.float32)
        print("one row each,", B, flush=True)
        q, _ = run_write(c, "bf16", Hq, qkv, None, None, 1e6)
        q2, whole = run_write(c, "bf16", Hq, qkv, None, None, 1e6, in_place=True)
        np.testing.assert_array_equal(q, q2)
        out = [torch.zeros((B, 1, Hq * d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        ws = tlt.kv8_attention_workspace(B, 1, Hq, Hkv, d, 30)
        tlt.kv8_attention(tlt.TLT_BF16, Hq, whole[..., :Hq * d], None, c.kv, 0, out[0], ws)
        tlt.kv8_attention(tlt.TLT_BF16, Hq, whole[..., :Hq * d].clone(memory_format=torch.contiguous_format), None, c.kv, 0, out[1], ws)
        assert torch.equal(*out) and out[0].any()


# ---- read

@pytest.mark.parametrize("dtype,Hkv,d,page,n,L", [("bf16", 4, 128, 16, 37, 3), ("fp32", 2, 64, 16, 1, 2), ("fp32", 1, 192, 5, 20, 1), ("bf16", 3, 256, 7, 16, 2)])
def test_read(dtype, Hkv, d, page, n, L):
    """Exact values, rows at and behind `count` untouched, slots without a page zero, NaN rows NaN."""
    ctxs = [n + 9, n, 3 * n + 50]
    c = m.Cache(ctxs, 1, Hkv, d, page, layers=L, seed=4)
    c.exps["k"][:, c.table[0, 0], 0, 0] = 255
    c.codes["k"][:, c.table[0, 0], 0, 0] = 0
    c.upload()
    c.kv.block_table[2, 1] = -1
    c.table[2, 1] = -1
    first, count = np.array([3 if n > 3 else 0, 0, 2 * page - 1], np.int32), np.array([n, n // 2, n + 7], np.int32)
    code, dt, _ = DTYPE[dtype]
    out = [torch.full((L, 3, n, Hkv, d), 5.0, dtype=dt, device="cuda") for _ in range(2)]
    print("read", dtype, Hkv, d, page, n, flush=True)
    tlt.kv8_read(code, c.kv, cuda(first), cuda(count), *out)
    for x, o in zip(("k", "v"), out):
        got = o.double().cpu().numpy()
        for l in range(L):
            for b in range(3):
                want = np.full((n, Hkv, d), 5.0)
                k = min(count[b], n)
                want[:k] = c.rows(x, l, b, first[b], first[b] + k)
                np.testing.assert_array_equal(got[l, b], want)
    tlt.kv8_read(code, c.kv, cuda(np.array([-1, 2 ** 31 - 2, 10 ** 6], np.int32)), None, *out)     # nothing there
    assert all(not o.any() for o in out)


# ---- attention

def run_attention(c, dtype, q, mask, layer=0, impl=-1, wide=False, ws=None):
    code, dt, _ = DTYPE[dtype]
    B, n, Hq, d = q.shape
    x = cuda(q.reshape(B, n, Hq * d)).to(dt)
    if wide:
        w = torch.full((B, n, Hq * d + 64), 99.0, dtype=dt, device="cuda")
        w[..., :Hq * d] = x
        x = w[..., :Hq * d]
    out = torch.full((B, n, Hq * d), 7.0, dtype=dt, device="cuda")
    ws = ws if ws is not None else tlt.kv8_attention_workspace(B, n, Hq, c.kv.k_pool.shape[2], d, int(c.ctx.max()) + n).fill_(0xAB)
    tlt.kv8_attention(code, Hq, x, None if mask is None else cuda(mask.view(np.int64)), c.kv, layer, out, ws, impl)
    torch.cuda.synchronize()
    return out.view(B, n, Hq, d)


def check_attention(c, dtype, q, mask, got, rows=None):
    """Element by element against 64 bits, for sequences `rows` (default: all)."""
    q64 = torch.from_numpy(q).to(DTYPE[dtype][1]).double().numpy()
    got = got.double().cpu().numpy()
    worst = 0.0
    for b in rows if rows is not None else range(len(c.ctx)):
        want, tol = m.attention(c, b, q64[b], None if mask is None else mask[b], rounded=dtype == "bf16")
        assert np.array_equal(np.isnan(want), np.isnan(got[b])), b
        err = np.abs(np.nan_to_num(got[b] - want))
        assert (err <= tol).all(), (b, float((err / np.maximum(tol, 1e-300)).max()))
        worst = max(worst, float((err / np.maximum(tol, 1e-300)).max()))
    print(f"  worst share of what is allowed: {worst:.3f}", flush=True)


CASES = [
    ("bf16", 28, 4, 128, 1, [8191], 16),
    ("bf16", 28, 4, 128, 1, [0, 1, 15, 16, 17, 62, 63, 64, 65, 1000], 16),
    ("bf16", 40, 8, 128, 1, [300, 4099], 16),
    ("bf16", 64, 8, 128, 2, [2047, 5], 16),                 # 16 rows per kv head
    ("bf16", 4, 4, 128, 1, [1, 16, 1000], 16),              # one row per kv head
    ("bf16", 28, 4, 128, 3, [700, 0, 128], 16),             # 21 rows
    ("bf16", 8, 2, 128, 13, [0, 37, 150], 16),
    ("bf16", 28, 4, 128, 16, [8000, 63], 16),               # 112 rows
    ("bf16", 28, 4, 128, 48, [700, 90, 4099], 16),          # 336 rows
    ("bf16", 40, 8, 128, 32, [1500, 64, 63, 65], 16),       # 160 rows
    ("bf16", 28, 4, 128, 64, [2100, 5], 16),                # 448 rows
    ("bf16", 64, 2, 128, 64, [130, 1], 16),                 # 2048 rows
    ("bf16", 8, 1, 128, 1, [30001], 16),
    ("bf16", 32, 1, 128, 1, [513, 90], 16),                 # 32 rows of one node
    ("bf16", 6, 2, 128, 7, [100, 33], 8),                   # pages of 8 and 5
    ("bf16", 5, 1, 128, 2, [77], 5),
    ("bf16", 4, 2, 64, 5, [130, 0], 16),
    ("bf16", 3, 1, 192, 2, [70], 16),
    ("bf16", 2, 2, 256, 9, [200, 31], 32),
    ("fp32", 4, 2, 64, 5, [128, 600], 16),
    ("fp32", 8, 2, 128, 13, [0, 37, 150], 16),
    ("fp32", 2, 1, 192, 1, [65], 16),
    ("fp32", 5, 5, 256, 3, [400, 2], 16),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,d,n,ctxs,page", CASES)
def test_attention(dtype, Hq, Hkv, d, n, ctxs, page):
    print("attention", dtype, Hq, Hkv, d, n, ctxs, page, flush=True)
    rng = np.random.default_rng(Hq + n)
    c = m.Cache(ctxs, n, Hkv, d, page, seed=n)
    q = (rng.standard_normal((len(ctxs), n, Hq, d)) * np.exp2(rng.integers(-2, 2, (len(ctxs), n, Hq, 1)))).astype(np.float32)
    mask = m.random_trees(rng, len(ctxs), n)[1]
    got = run_attention(c, dtype, q, mask)
    check_attention(c, dtype, q, mask, got)
    assert torch.equal(got, run_attention(c, dtype, q, mask, wide=True))                   # rows inside wider ones; the same bits again
    check_attention(c, dtype, q, None, run_attention(c, dtype, q, None))                   # a chain
    check_attention(c, dtype, q, mask, run_attention(c, dtype, q, mask, impl=0))


@pytest.mark.parametrize("dtype,Hq,Hkv,d,n", [("bf16", 28, 4, 128, 2), ("bf16", 28, 4, 128, 20), ("fp32", 4, 2, 64, 6), ("bf16", 8, 1, 128, 64), ("bf16", 4, 2, 64, 7)])
def test_rows_that_see_nothing_or_something_that_is_not_finite(dtype, Hq, Hkv, d, n):
    """Masks without a bit: zeros where there is no context, the context alone where there is one.  A row of the cache that is not finite reaches exactly
    the rows that see it."""
    print("attention, odd masks", dtype, Hq, Hkv, d, n, flush=True)
    ctxs = [0, 200, 70, 0, 17]
    rng = np.random.default_rng(1)
    c = m.Cache(ctxs, n, Hkv, d, 16, seed=9)
    q = rng.standard_normal((len(ctxs), n, Hq, d)).astype(np.float32)
    mask = m.random_trees(rng, len(ctxs), n)[1]
    mask[0, ::2], mask[1, 1::2] = 0, 0

    def spoil(x, b, slot, head):
        pg = c.table[b, slot // 16]
        c.codes[x][0, pg, head, slot % 16], c.exps[x][0, pg, head, slot % 16] = 0, 255

    spoil("k", 0, n - 1, 0)                   # the last node, seen by itself at most
    spoil("v", 1, 200 + n - 1, Hkv - 1)
    spoil("v", 1, 200, 0)                     # the root, seen by all that see anything
    spoil("k", 2, 70 + n // 2, 0)
    mask[3, :] = 0
    spoil("v", 4, 3, Hkv - 1)                 # in the context: seen by every row
    c.upload()
    got = run_attention(c, dtype, q, mask)
    assert not got[3].any()
    # (a value that is not finite makes its whole row of the cache NaN, and so every element of the output; the model's weights see it through the mean)
    q64 = torch.from_numpy(q).to(DTYPE[dtype][1]).double().numpy()
    g = got.double().cpu().numpy()
    for b in range(len(ctxs)):
        want, tol = m.attention(c, b, q64[b], mask[b], rounded=dtype == "bf16")
        assert np.array_equal(np.isnan(want).any(-1), np.isnan(g[b]).all(-1)) and np.array_equal(np.isnan(want).any(-1), np.isnan(g[b]).any(-1)), b
        ok = ~np.isnan(want).any(-1)
        assert (np.abs(g[b] - want)[ok] <= tol[ok]).all(), b


@pytest.mark.parametrize("dtype,Hq,Hkv,d,n", [("bf16", 28, 4, 128, 1), ("bf16", 28, 4, 128, 30), ("fp32", 4, 2, 64, 4)])
def test_queries_that_are_not_finite_stay_in_their_row(dtype, Hq, Hkv, d, n):
    c = m.Cache([100, 40], n, Hkv, d, 16, seed=9)
    rng = np.random.default_rng(1)
    q = rng.standard_normal((2, n, Hq, d)).astype(np.float32)
    print("attention, queries that are not finite", dtype, n, flush=True)
    clean = run_attention(c, dtype, q, None)
    q[0, n - 1, 1, 5], q[1, 0, Hq - 1, 0] = np.nan, np.inf
    got = run_attention(c, dtype, q, None)
    bad = torch.zeros((2, n, Hq), dtype=torch.bool)
    bad[0, n - 1, 1] = bad[1, 0, Hq - 1] = True
    assert torch.isnan(got.cpu()[bad]).all() and torch.equal(got.cpu()[~bad], clean.cpu()[~bad])


@pytest.mark.parametrize("dtype,Hq,Hkv,n", [("bf16", 28, 4, 1), ("bf16", 28, 4, 24), ("fp32", 8, 2, 3)])
def test_large_scores_and_far_exponents(dtype, Hq, Hkv, n):
    """Scores of several hundred (one key takes nearly all), and rows at both ends of the exponents' range."""
    d = 128
    c = m.Cache([900, 90], n, Hkv, d, 16, seed=9)
    rng = np.random.default_rng(1)
    c.exps["k"][0, :, :, ::5] = np.minimum(c.exps["k"][0, :, :, ::5] + 4, 254)
    c.exps["k"][0, :, :, 3::7] = rng.integers(1, 60, c.exps["k"][0, :, :, 3::7].shape)
    c.exps["v"][0, :, :, 2::7] = rng.integers(1, 60, c.exps["v"][0, :, :, 2::7].shape)
    c.upload()
    q = (rng.standard_normal((2, n, Hq, d)) * 2).astype(np.float32)
    q[:, 0] *= 2.0 ** -60
    q[0, 0, 1] *= 2.0 ** -60
    print("attention, large scores", dtype, n, flush=True)
    check_attention(c, dtype, q, None, run_attention(c, dtype, q, None))


@pytest.mark.parametrize("n", [1, 5, 40])
def test_pages_missing_from_the_table(n):
    """A visible slot without a page counts as a key and a value of zero; the other sequence keeps its bits."""
    Hq, Hkv, d = 28, 4, 128
    c = m.Cache([900, 700, 30], n, Hkv, d, 16, seed=9)
    q = np.random.default_rng(1).standard_normal((3, n, Hq, d)).astype(np.float32)
    print("attention, pages missing", n, flush=True)
    whole = run_attention(c, "bf16", q, None)
    for p, v in ((1, -1), (40, 10 ** 6), (55, -7)):
        c.table[0, p] = v
    c.table[2, 1] = -1
    c.kv.block_table.copy_(cuda(c.table.astype(np.int32)))
    got = run_attention(c, "bf16", q, None)
    assert torch.equal(got[1], whole[1])
    check_attention(c, "bf16", q, None, got)
    check_attention(c, "bf16", q, None, run_attention(c, "bf16", q, None, impl=0))


@pytest.mark.parametrize("B", [70, 700])
def test_many_sequences(B):
    Hq, Hkv, d = 4, 1, 128
    ctxs = [17 * (i % 9) + (900 if i % 50 == 5 else 0) for i in range(B)]
    c = m.Cache(ctxs, 2, Hkv, d, 16, seed=3)
    q = np.random.default_rng(1).standard_normal((B, 2, Hq, d)).astype(np.float32)
    print("attention,", B, "sequences", flush=True)
    check_attention(c, "bf16", q, None, run_attention(c, "bf16", q, None), rows=sorted(set(range(0, B, 7)) | set(range(5, B, 50))))


@pytest.mark.parametrize("B,n,Hq,Hkv", [(200, 1, 4, 1), (256, 12, 8, 1), (300, 2, 4, 1), (257, 12, 8, 1), (110, 2, 40, 20)])
def test_many_sequences_a_few_of_them_long(B, n, Hq, Hkv):
    """More sequences than a wave has lanes, some cut into several ranges: balanced ones, and those of a fixed length."""
    ctxs = [3 * (i % 11) for i in range(B)]
    long = {7: 9000, B // 2: 4095, B - 1: 4200}
    for b, x in long.items():
        ctxs[b] = x
    c = m.Cache(ctxs, n, Hkv, 128, 16, seed=4)
    q = np.random.default_rng(2).standard_normal((B, n, Hq, 128)).astype(np.float32)
    print("attention,", B, "sequences,", n, "rows", flush=True)
    check_attention(c, "bf16", q, None, run_attention(c, "bf16", q, None), rows=sorted(set(range(0, B, 13)) | set(long)))


def test_offsets_past_32_bits():
    """Pages beyond 4 GB of codes, in every operator."""
    Hq, Hkv, d, page, n = 8, 8, 128, 16, 3
    n_pages = (1 << 32) // (Hkv * page * d) + 40
    base = n_pages - 30
    pools = [torch.empty((1, n_pages, Hkv, page, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    exps = [torch.empty((1, n_pages, Hkv, page), dtype=torch.uint8, device="cuda") for _ in range(2)]
    c = m.Cache([300], n, Hkv, d, page, seed=1, dev="cpu")
    for p, x in zip(pools, ("k", "v")):
        p[:, base:base + c.codes[x].shape[1]] = cuda(c.codes[x])
    for p, x in zip(exps, ("k", "v")):
        p[:, base:base + c.exps[x].shape[1]] = cuda(c.exps[x])
    c.kv = tlt.KV8(*pools, *exps, cuda((c.table + base).astype(np.int32)), cuda(c.ctx), 300)
    rng = np.random.default_rng(0)
    print("offsets past 32 bits", flush=True)
    qkv = torch.from_numpy(rng.standard_normal((1, n, (Hq + 2 * Hkv) * d)).astype(np.float32)).bfloat16()
    q, _ = run_write(c, "bf16", Hq, qkv.float().numpy(), None, None, 1e6)
    for p, x in zip(pools, ("k", "v")):
        c.codes[x] = p[:, base:base + c.codes[x].shape[1]].cpu().numpy()
    for p, x in zip(exps, ("k", "v")):
        c.exps[x] = p[:, base:base + c.exps[x].shape[1]].cpu().numpy()
    np.testing.assert_array_equal(m.encode(qkv.double().numpy().reshape(n, Hq + 2 * Hkv, d)[:, Hq + Hkv:])[0],
                                  np.stack([c.codes["v"][0, c.table[0, s // 16], :, s % 16] for s in range(300, 300 + n)]))
    q = q.reshape(1, n, Hq, d).astype(np.float32)
    check_attention(c, "bf16", q, None, run_attention(c, "bf16", q, None))
    tlt.kv8_commit(c.kv, cuda(np.array([1], np.int32)), cuda(np.array([[0, 2]], np.int32)))
    out = [torch.zeros((1, 1, 302, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    tlt.kv8_read(tlt.TLT_BF16, c.kv, cuda(np.zeros(1, np.int32)), None, *out)
    want = np.concatenate([c.rows("k", 0, 0, 0, 301), c.rows("k", 0, 0, 302, 303)])
    np.testing.assert_array_equal(out[0][0, 0].double().cpu().numpy(), want)


# ---- commit

@pytest.mark.parametrize("Hkv,d,page,L,n", [(4, 128, 16, 5, 24), (2, 64, 16, 2, 64), (1, 192, 5, 1, 9), (3, 256, 16, 2, 17), (8, 256, 16, 16, 40)])
def test_commit(Hkv, d, page, L, n):
    """Accepted rows move in all layers, in the order that lets a written row have been a source; lengths advance; nothing else changes."""
    ctxs = [0, 5, 100, 33, 60, 7]
    B, stride = len(ctxs), min(n, 20)
    c = m.Cache(ctxs, n, Hkv, d, page, layers=L, seed=6)
    rng = np.random.default_rng(n)
    acc, path = np.zeros(B, np.int32), np.full((B, stride), -1, np.int32)
    for b in range(B):
        a = [0, stride - 1, 1, stride // 2, stride + 5, 3][b]
        acc[b] = a
        a = min(a, stride - 1)
        path[b, :a + 1] = np.concatenate([[0], np.sort(rng.permutation(np.arange(1, n))[:a])])
    acc[0] = -3                                              # nothing accepted, whatever the sign
    path[5, 2] = n + 70                                      # entries that mean nothing move nothing
    path[5, 3] = -4
    print("commit", Hkv, d, page, L, n, flush=True)
    want = {x: (c.codes[x].copy(), c.exps[x].copy()) for x in ("k", "v")}
    for b in range(B):
        a = min(max(acc[b], 0), stride - 1)
        for j in range(1, a + 1):
            p = path[b, j]
            if j < p < 64:
                s, t = ctxs[b] + p, ctxs[b] + j
                for x in ("k", "v"):
                    for arr in want[x]:
                        arr[:, c.table[b, t // page], :, t % page] = arr[:, c.table[b, s // page], :, s % page]
    tlt.kv8_commit(c.kv, cuda(acc), cuda(path))
    download(c)
    for x in ("k", "v"):
        np.testing.assert_array_equal(c.codes[x], want[x][0])
        np.testing.assert_array_equal(c.exps[x], want[x][1])
    np.testing.assert_array_equal(c.kv.seq_len.cpu().numpy(), np.array(ctxs) + np.clip(acc, 0, stride - 1) + 1)


def test_commit_takes_a_row_twice():
    c = m.Cache([40, 3], 12, 2, 128, 16, layers=2, seed=3)
    path = np.array([[0, 5, 5, 9, 9], [0, 2, 2, 4, 4]], np.int32)      # (sequence 1: row 2 is a place before it is a source again)
    want = {x: (c.codes[x].copy(), c.exps[x].copy()) for x in ("k", "v")}
    for b, ctx in enumerate((40, 3)):
        for j in range(1, 5):
            if path[b, j] > j:
                s, t = ctx + path[b, j], ctx + j
                for x in ("k", "v"):
                    for arr in want[x]:
                        arr[:, c.table[b, t // 16], :, t % 16] = arr[:, c.table[b, s // 16], :, s % 16]
    print("commit, a row twice", flush=True)
    tlt.kv8_commit(c.kv, cuda(np.array([4, 4], np.int32)), cuda(path))
    download(c)
    for x in ("k", "v"):
        np.testing.assert_array_equal(c.codes[x], want[x][0])
        np.testing.assert_array_equal(c.exps[x], want[x][1])
    assert c.kv.seq_len.tolist() == [45, 8]


# ---- together

@pytest.mark.parametrize("n", [1, 8, 20])
def test_padded_batch(n):
    """A place in the batch without a sequence: length 0, no pages, masks of zero.  Nothing is written for it, its outputs are zeros."""
    Hq, Hkv, d = 28, 4, 128
    c = m.Cache([90, 0, 200], n, Hkv, d, 16, seed=2)
    alone = m.Cache([90, 0, 200], n, Hkv, d, 16, seed=2)
    qkv = torch.randn((3, n, (Hq + 2 * Hkv) * d), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    mask = np.repeat(((np.uint64(2) << np.arange(n, dtype=np.uint64)) - np.uint64(1))[None], 3, 0)
    mask[1] = 0
    print("padded batch", n, flush=True)
    keep = {k: getattr(c.kv, k).clone() for k in ("k_pool", "v_pool", "k_exp", "v_exp")}
    own = [int(p) for p in c.table[1] if p >= 0]
    c.table[1] = -1
    c.kv.block_table.copy_(cuda(c.table.astype(np.int32)))
    q = torch.zeros((3, n, Hq * d), dtype=torch.bfloat16, device="cuda")
    tlt.kv8_write(tlt.TLT_BF16, Hq, 1e6, qkv, None, None, c.kv, 0, q)
    assert all(torch.equal(getattr(c.kv, k)[:, own], t[:, own]) for k, t in keep.items())
    tlt.kv8_write(tlt.TLT_BF16, Hq, 1e6, qkv, None, None, alone.kv, 0, q)
    others = [p for p in range(keep["k_pool"].shape[1]) if p not in own]
    assert all(torch.equal(getattr(c.kv, k)[:, others], getattr(alone.kv, k)[:, others]) for k in keep)
    download(c)
    got = run_attention(c, "bf16", q.float().cpu().numpy().reshape(3, n, Hq, d), mask)
    assert not got[1].any()
    check_attention(c, "bf16", q.float().cpu().numpy().reshape(3, n, Hq, d), mask, got)


@pytest.mark.parametrize("n", [1, 8, 20])
@pytest.mark.parametrize("impl", [-1, 0])
def test_lengths_above_the_bound_stay_inside(n, impl):
    """A length above the declared bound: that sequence's outputs mean nothing, the other's are right."""
    Hq, Hkv, d = 28, 4, 128
    c = m.Cache([500, 200], n, Hkv, d, 16, seed=2)
    c.kv.seq_len_bound = 200
    q = np.random.default_rng(1).standard_normal((2, n, Hq, d)).astype(np.float32)
    ws = tlt.kv8_attention_workspace(2, n, Hq, Hkv, d, 200 + n)
    for length in (500, 2 ** 31 - 1):
        print("length above the bound", n, impl, length, flush=True)
        c.kv.seq_len[0] = length
        check_attention(c, "bf16", q, None, run_attention(c, "bf16", q, None, impl=impl, ws=ws), rows=[1])

def steps(c, Hq, n, qkv, depth, mask, acc, path, out, ws, q, n_steps=3):
    """A few steps of a layer: write, attend, commit."""
    for s in range(n_steps):
        tlt.kv8_write(tlt.TLT_BF16, Hq, 1e6, qkv[s], None, depth, c.kv, 0, q)
        tlt.kv8_attention(tlt.TLT_BF16, Hq, q, mask, c.kv, 0, out[s], ws)
        tlt.kv8_commit(c.kv, acc, path)


@pytest.mark.parametrize("Hq,Hkv,n,ctxs", [(28, 4, 1, [500, 40]), (28, 4, 8, [600, 7]), (28, 4, 20, [300, 0, 61])])
def test_steps_in_a_graph_and_on_two_streams(Hq, Hkv, n, ctxs):
    """Three steps, each on what the ones before it left; captured and replayed several times between eager runs, the same bits; two caches on two streams."""
    d, B = 128, len(ctxs)
    rng = np.random.default_rng(2)
    depth, mask = m.random_trees(rng, B, n)
    a = min(3, n - 1)
    path = np.tile(np.concatenate([[0], np.sort(rng.permutation(np.arange(1, n))[:a])]).astype(np.int32), (B, 1)) if n > 1 else np.zeros((B, 1), np.int32)
    acc = np.full(B, a, np.int32)
    dev = dict(depth=cuda(depth), mask=cuda(mask.view(np.int64)), acc=cuda(acc), path=cuda(path))

    def setting(seed):
        c = m.Cache(np.array(ctxs) + 3 * (a + 1), n, Hkv, d, 16, seed=seed)
        c.ctx = np.array(ctxs, np.int32)
        c.kv.seq_len.copy_(cuda(c.ctx))
        c.kv.seq_len_bound = int(c.ctx.max()) + 2 * (a + 1)
        qkv = torch.randn((3, B, n, (Hq + 2 * Hkv) * d), generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()
        out = torch.zeros((3, B, n, Hq * d), dtype=torch.bfloat16, device="cuda")
        q = torch.zeros((B, n, Hq * d), dtype=torch.bfloat16, device="cuda")
        return c, qkv, out, q, tlt.kv8_attention_workspace(B, n, Hq, Hkv, d, c.kv.seq_len_bound + n)

    def go(x):
        c, qkv, out, q, ws = x
        c.kv.seq_len.copy_(start)
        steps(c, Hq, n, qkv, dev["depth"], dev["mask"], dev["acc"], dev["path"], out, ws, q)

    start = cuda(np.array(ctxs, np.int32))
    x = setting(1)
    print("steps", Hq, n, flush=True)
    go(x)
    torch.cuda.synchronize()
    want, lens = x[2].clone(), x[0].kv.seq_len.clone()
    assert lens.tolist() == [v + 3 * (a + 1) for v in ctxs]
    # the last step against 64 bits: its lengths, what the cache held, the queries that it left
    c = download(x[0])
    pools = {k: c.kv.__dict__[k].clone() for k in ("k_pool", "v_pool", "k_exp", "v_exp")}
    c.ctx = np.array(ctxs, np.int32) + 2 * (a + 1)
    c.kv.seq_len.copy_(cuda(c.ctx))
    tlt.kv8_write(tlt.TLT_BF16, Hq, 1e6, x[1][2], None, dev["depth"], c.kv, 0, x[3])      # (the commit moved rows of the tree: back to where they were)
    download(c)
    check_attention(c, "bf16", x[3].float().cpu().numpy().reshape(B, n, Hq, d), mask, want[2].view(B, n, Hq, d))
    for k, t in pools.items():
        c.kv.__dict__[k].copy_(t)
    # captured, replayed, with eager work in between
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        go(x)
    for _ in range(3):
        x[2].zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(x[2], want) and torch.equal(x[0].kv.seq_len, lens)
        go(x)
        torch.cuda.synchronize()
        assert torch.equal(x[2], want)
    # two at once, each with its own workspace
    y = setting(7)
    go(y)
    torch.cuda.synchronize()
    want_y = y[2].clone()
    x[2].zero_(), y[2].zero_()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s1):
            go(x)
        with torch.cuda.stream(s2):
            go(y)
    torch.cuda.synchronize()
    assert torch.equal(x[2], want) and torch.equal(y[2], want_y)
