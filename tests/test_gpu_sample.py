"""tlt_sample and tlt_sample_filter against the model in whole numbers: the same tokens, kept sets and counts exactly, log-probabilities to fp32's rounding."""
import math

import numpy as np
import pytest
import torch

import pick_model as pm
from paper_2511_16665_amd import binding as tlt

pytestmark = pytest.mark.gpu
INF = math.inf


def logits_of(kind, rows, V, rng):
    x = rng.normal(0, 2.0, (rows, V))
    if kind == "peaks":
        for r in range(rows):
            x[r, rng.integers(0, V, min(V, 12))] += 14 - 10 * rng.random(min(V, 12))
    if kind == "ties":
        x = np.rint(x)
    if kind == "equal":
        x[:] = 1.25
    if kind == "zeros":           # zeros of both signs are equal
        x = np.where(rng.random(x.shape) < 0.5, -0.0, 0.0)
    if kind == "masked":
        x[rng.random(x.shape) < 0.9] = -INF
        x[0] = -INF
    if kind == "front":           # the likely ones side by side
        x[:, :min(V, 700)] += 9
    if kind == "wide":
        x *= 40
    return x.astype(np.float32)


def asks(rng, B):
    """Settings of every kind, one per sequence."""
    some = [dict(), dict(top_k=1), dict(top_k=3), dict(top_k=50), dict(top_k=10 ** 9), dict(top_p=0.9), dict(top_p=0.5, tau=0.7), dict(top_p=0.999), dict(top_p=0.0), dict(top_p=1e-12),
            dict(min_p=0.1), dict(min_p=1.0), dict(min_p=2.0), dict(min_p=1e-8), dict(tau=0.0), dict(tau=-1.0), dict(tau=math.nan), dict(tau=0.01), dict(tau=30.0),
            dict(tau=1.3, top_k=40, top_p=0.95, min_p=0.02), dict(tau=0.8, top_k=700, top_p=0.99), dict(top_k=2000, top_p=0.97), dict(top_k=-5, top_p=math.nan, min_p=math.nan),
            dict(top_p=1.0 - 2.0 ** -24), dict(tau=INF, top_k=5), dict(tau=1e-30), dict(top_p=-3.0), dict(top_p=0.3, min_p=0.9)]
    return [some[i] for i in rng.permutation(np.arange(B) % len(some))]


def filter_of(asked):
    get = lambda name, default, dt: torch.tensor([a.get(name, default) for a in asked], dtype=dt).cuda()
    return tlt.SampleFilter(get("tau", 1.0, torch.float32), get("top_k", 0, torch.int32), get("top_p", 1.0, torch.float32), get("min_p", 0.0, torch.float32))


def check_rows(x, asked, n, u, token, logprob, kept, out=None):
    """x float64 [rows, V]; asked: per sequence of n rows.  A log-probability is rounded to fp32 once (2^-24 of it); in front of that the sums are off by a unit of 2^-32 of the
    largest weight for some of the V tokens at most (exponentials of two libraries): 2^-32 V."""
    for r in range(len(x)):
        want_t, want_lp, want_n = pm.draw(x[r], int(u[r]), **asked[r // n])
        assert (int(token[r]), int(kept[r])) == (want_t, want_n), (r, asked[r // n])
        for got, want in zip(logprob[r], want_lp):
            assert (math.isnan(want) and math.isnan(got)) or got == want or abs(float(got) - want) <= 2.0 ** -24 * abs(want) + 2.0 ** -32 * x.shape[1] + 1e-12, (r, got, want)
        if out is not None:
            keep, _, _ = pm.choose(x[r], **asked[r // n])
            row = x[r] if keep is None or not len(keep) else np.where(np.isin(np.arange(x.shape[1]), keep), x[r], -INF)
            np.testing.assert_array_equal(out[r], row, err_msg=str((r, asked[r // n])))


def run(code, x, asked, n, u, pad=0, in_place=False):
    """Both calls on rows that lie in wider ones."""
    B, V = x.shape[0] // n, x.shape[1]
    dt = tlt.torch_dtype(code)
    wide = torch.full((B, n, V + pad), 77.0, dtype=dt, device="cuda")
    wide[..., :V] = torch.from_numpy(x).view(B, n, V).cuda().to(dt)
    logits = wide[..., :V]
    token, kept, kept2 = (torch.full((B, n), 9, dtype=torch.int32, device="cuda") for _ in range(3))
    logprob = torch.zeros((B, n, 2), device="cuda")
    ws = tlt.sample_workspace(B * n, V)
    ws.fill_(255)
    ut = torch.from_numpy(u.astype(np.uint32).view(np.int32)).cuda().view(B, n)
    ask = filter_of(asked)
    tlt.sample(code, logits, ask, ut, token, logprob, kept, ws)
    values = logits.double().cpu().numpy().reshape(B * n, V)
    out = logits if in_place else torch.full((B, n, V + 3), 5.0, dtype=dt, device="cuda")[..., :V]
    tlt.sample_filter(code, logits, ask, out, kept2, ws)
    torch.cuda.synchronize()
    assert torch.equal(kept, kept2)
    if pad:
        assert bool((wide[..., V:] == 77.0).all())
    if not in_place:
        assert out.shape[-1] == V and bool((out.as_strided((B * n, 3), (V + 3, 1), V) == 5.0).all())
    got = out.double().cpu().numpy().reshape(B * n, V)
    return values, token.flatten().cpu().numpy(), logprob.view(-1, 2).cpu().numpy(), kept.flatten().cpu().numpy(), got


KINDS = ["bell", "peaks", "ties", "equal", "zeros", "masked", "front", "wide"]


@pytest.mark.parametrize("code", [tlt.TLT_F32, tlt.TLT_BF16])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("V", [1, 2, 5, 63, 65, 1000, 4097])
def test_small_vocabularies(code, kind, V):
    rng = np.random.default_rng(V + len(kind))
    rows = 28
    x = logits_of(kind, rows, V, rng)
    u = rng.integers(0, 2 ** 32, rows)
    u[:2] = 0, 2 ** 32 - 1
    asked = asks(rng, rows)
    values, *got = run(code, x, asked, 1, u, pad=V % 4)
    check_rows(values, asked, 1, u, *got)


@pytest.mark.parametrize("code", [tlt.TLT_F32, tlt.TLT_BF16])
@pytest.mark.parametrize("kind", KINDS)
def test_a_large_vocabulary(code, kind):
    rng = np.random.default_rng(7)
    rows, V = 14, 50001
    x = logits_of(kind, rows, V, rng)
    u = rng.integers(0, 2 ** 32, rows)
    asked = asks(rng, 28)[:rows] if kind != "equal" else asks(np.random.default_rng(1), 28)[:rows]
    values, *got = run(code, x, asked, 1, u, pad=3, in_place=True)
    check_rows(values, asked, 1, u, *got)


@pytest.mark.parametrize("B,n,V", [(1, 1, 152064), (3, 7, 20000), (40, 8, 3001), (300, 1, 2048), (5, 64, 1024), (11, 100, 4500)])
def test_batches_and_trees(B, n, V):
    rng = np.random.default_rng(B)
    x = np.concatenate([logits_of("peaks", B * n - B * n // 2, V, rng), logits_of("bell", B * n // 2, V, rng)])
    u = rng.integers(0, 2 ** 32, B * n)
    asked = asks(rng, B)
    values, *got = run(tlt.TLT_F32, x, asked, n, u, in_place=True)
    check_rows(values, asked, n, u, *got)


@pytest.mark.parametrize("code", [tlt.TLT_F32, tlt.TLT_BF16])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,V", [(112, 5003), (196, 4500), (280, 4099), (280, 9001), (28, 33000), (3, 33001)])
def test_rows_by_one_or_several_workgroups(code, kind, rows, V):
    """Few rows are cut into segments, more of them are a workgroup's; every setting on every kind of row."""
    rng = np.random.default_rng(rows + len(kind))
    x = logits_of(kind, rows, V, rng)
    u = rng.integers(0, 2 ** 32, rows)
    asked = asks(rng, 28) * 10
    values, *got = run(code, x, asked[:rows], 1, u, pad=V % 4)
    check_rows(values, asked[:rows], 1, u, *got)


@pytest.mark.parametrize("code", [tlt.TLT_F32, tlt.TLT_BF16])
@pytest.mark.parametrize("rows", [8, 264])
def test_more_tokens_asked_for_than_weigh_anything(code, rows):
    """At a low temperature most of the first top_k tokens weigh nothing: they are kept all the same, but never drawn."""
    rng = np.random.default_rng(rows)
    V = 20011
    x = logits_of("peaks", rows, V, rng)
    u = rng.integers(0, 2 ** 32, rows)
    u[:2] = 0, 2 ** 32 - 1
    asked = [dict(tau=0.05, top_k=4000), dict(tau=0.05, top_k=4000, top_p=0.9), dict(tau=0.02, top_k=15000, min_p=1e-6), dict(tau=0.1, top_k=19999), dict(tau=0.05, top_k=300),
             dict(tau=0.3, top_k=9000, top_p=0.999999), dict(tau=1e-3, top_k=20010), dict(tau=2.5, top_k=12000, top_p=0.95)] * (rows // 8)
    values, *got = run(code, x, asked, 1, u)
    check_rows(values, asked, 1, u, *got)


def test_values_at_the_ends():
    """NaN, infinities, the type's lowest value as a mask, denormals, differences past the weights' range."""
    low, tiny = float(np.finfo(np.float32).min), 1e-42
    rows = [[math.nan, 1.0, 2.0], [1.0, 2.0, math.nan], [INF, 1.0, INF], [-INF, -INF, -INF], [low, low, low], [low, 3.0, low], [tiny, -tiny, 0.0], [3e38, -3e38, 3e38], [0.0, -22.0, -22.5],
            [-INF, 5.0, -INF], [INF, INF, INF], [-INF, low, -INF]]
    few = rows
    for V, times in ((3, 1), (900, 1), (9000, 1), (9000, 9), (9000, 22)):
        rows = few * times
        x = np.full((len(rows), V), -INF, np.float32)
        x[:, [0, V // 2, V - 1]] = rows
        for ask in (dict(), dict(top_k=2), dict(top_p=0.6), dict(min_p=0.2), dict(tau=0.0), dict(top_k=2, top_p=0.99, min_p=0.01), dict(tau=INF, top_p=0.5), dict(tau=1e-38)):
            for u0 in (0, 2 ** 31, 2 ** 32 - 1):
                u = np.full(len(rows), u0)
                asked = [ask] * len(rows)
                values, token, logprob, kept, out = run(tlt.TLT_F32, x, asked, 1, u)
                check_rows(values, asked, 1, u, token, logprob, kept, out)


def test_nothing_asked_for():
    """No filter arrays at all: the whole row at temperature 1; the optional outputs left out."""
    rng = np.random.default_rng(0)
    x = torch.from_numpy(logits_of("peaks", 6, 5000, rng)).cuda()
    u = torch.from_numpy(rng.integers(0, 2 ** 32, 6).astype(np.uint32).view(np.int32)).cuda()
    token = torch.empty((6,), dtype=torch.int32, device="cuda")
    ws = tlt.sample_workspace(6, 5000)
    tlt.sample(tlt.TLT_F32, x, tlt.SampleFilter(), u, token, None, None, ws)
    out = torch.empty_like(x)
    tlt.sample_filter(tlt.TLT_F32, x, tlt.SampleFilter(), out, None, ws)
    for r in range(6):
        assert int(token[r]) == pm.draw(x[r].double().cpu().numpy(), int(u[r]) % 2 ** 32)[0]
    assert torch.equal(out, x)


@pytest.mark.parametrize("tau", [0.9, 0.37])
def test_the_draw_is_the_acceptance_rule_s(tau):
    """A one-node tree's final draw is tlt_sample's, and on filtered logits it is the draw of the filtered distribution."""
    rng = np.random.default_rng(5)
    B, V = 4, 20011
    x = torch.from_numpy(logits_of("peaks", B, V, rng)).cuda()
    u = torch.from_numpy(rng.integers(0, 2 ** 32, B).astype(np.uint32).view(np.int32)).cuda()
    zero = torch.zeros((B, 1), dtype=torch.int32, device="cuda")
    tree = tlt.Tree(zero, zero - 1, zero, torch.ones((B, 1), dtype=torch.int64, device="cuda"), zero.float())
    q, ws = torch.zeros((B, 1, V), device="cuda"), tlt.sample_workspace(B, V)

    def accepted(logits):
        al, n_out = (torch.empty((B,), dtype=torch.int32, device="cuda") for _ in range(2))
        path, out = (torch.empty((B, 1), dtype=torch.int32, device="cuda") for _ in range(2))
        assert tlt.accept_sample_static(B, V, tau, tree, logits, q, zero, u, 1, al, path, out, n_out) == 0
        return out[:, 0]

    for more in (dict(), dict(top_k=30), dict(top_p=0.8), dict(min_p=0.05), dict(top_k=100, top_p=0.9, min_p=0.01)):
        ask = filter_of([dict(tau=tau, **more)] * B)
        token, out = torch.empty((B,), dtype=torch.int32, device="cuda"), torch.empty_like(x)
        tlt.sample(tlt.TLT_F32, x, ask, u, token, None, None, ws)
        tlt.sample_filter(tlt.TLT_F32, x, ask, out, None, ws)
        assert torch.equal(token, accepted(out)), more
        if not more:
            assert torch.equal(token, accepted(x))


def test_captured_and_replayed_beside_other_work():
    """A captured call replayed on new inputs, with the program's own work between, two graphs and another stream."""
    rng = np.random.default_rng(9)
    B, V = 5, 30000
    make = lambda kind: torch.from_numpy(logits_of(kind, B, V, rng)).cuda()
    asked = asks(rng, B)
    ask = filter_of(asked)
    inputs = [make(k) for k in ("peaks", "bell", "ties", "peaks")]
    us = [torch.from_numpy(rng.integers(0, 2 ** 32, B).astype(np.uint32).view(np.int32)).cuda() for _ in inputs]
    x, u, out = inputs[0].clone(), us[0].clone(), torch.empty((B, V), device="cuda")
    token, kept, kept2 = (torch.empty((B,), dtype=torch.int32, device="cuda") for _ in range(3))
    logprob = torch.empty((B, 2), device="cuda")
    ws = [tlt.sample_workspace(B, V) for _ in range(2)]
    stream = torch.cuda.Stream()
    draw = lambda: tlt.sample(tlt.TLT_F32, x, ask, u, token, logprob, kept, ws[0])
    mask = lambda: tlt.sample_filter(tlt.TLT_F32, x, ask, out, kept2, ws[1])
    torch.cuda.synchronize()
    graphs = []
    for call in (draw, mask):
        with torch.cuda.stream(stream):
            call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            call()
        graphs.append(g)
    for xi, ui in zip(inputs, us):
        x.copy_(xi)
        u.copy_(ui)
        for t in (token, kept, kept2):
            t.fill_(-7)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(kept, kept2)
        check_rows(xi.double().cpu().numpy(), asked, 1, ui.cpu().numpy().astype(np.int64) % 2 ** 32, token.cpu().numpy(), logprob.cpu().numpy(), kept.cpu().numpy(), out.double().cpu().numpy())
        assert int((x == xi).sum()) == B * V


def test_the_same_call_twice_gives_the_same_bits():
    rng = np.random.default_rng(2)
    x = torch.from_numpy(logits_of("bell", 33, 40000, rng)).cuda()
    u = torch.from_numpy(rng.integers(0, 2 ** 32, 33).astype(np.uint32).view(np.int32)).cuda()
    ask, ws, got = filter_of(asks(rng, 33)), tlt.sample_workspace(33, 40000), []
    for _ in range(3):
        token, logprob, kept = torch.empty((33,), dtype=torch.int32, device="cuda"), torch.empty((33, 2), device="cuda"), torch.empty((33,), dtype=torch.int32, device="cuda")
        tlt.sample(tlt.TLT_F32, x, ask, u, token, logprob, kept, ws)
        got.append((token, logprob, kept))
    for g in got[1:]:
        assert all(torch.equal(a.view(torch.int32), b.view(torch.int32)) for a, b in zip(g, got[0]))
