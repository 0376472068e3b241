"""tlt_sample and tlt_sample_filter where their searches in lists and bins refine, run short, or join many segments; against the model in whole numbers."""
import math

import numpy as np
import pytest
import torch

import pick_model as pm
from paper_2511_16665_amd import binding as tlt
from test_gpu_sample import KINDS, asks, check_rows, filter_of, logits_of, run

pytestmark = pytest.mark.gpu


def as_stored(x, code):
    """The values that a row of this type holds, as fp32."""
    return torch.from_numpy(x.astype(np.float32)).to(tlt.torch_dtype(code)).float().numpy()


@pytest.mark.parametrize("code", [tlt.TLT_F32, tlt.TLT_BF16])
@pytest.mark.parametrize("V,likely,ask", [(152064, 200, dict(top_k=200)), (152064, 300, dict(top_k=2000, top_p=0.97)), (152064, 150, dict(top_k=150, top_p=0.999, tau=0.9)),
                                          (50001, 180, dict(top_k=180)), (152064, 120, dict(top_k=120, min_p=1e-6))])
def test_draws_among_many_tokens_of_low_index(code, V, likely, ask):
    """The kept tokens are 0 .. likely - 1, of which token 0 weighs most: far more of them in one 256th of the vocabulary than a search compares with each other.  The uniforms reach into
    token 0's share, both sides of its end (2^13 of 2^32, hundreds of times what a unit in every weight could move it), the rest, and the last of it."""
    rng = np.random.default_rng(likely)
    row = rng.normal(-25.0, 2.0, V)
    row[:likely] = 5.0 + rng.random(likely)
    row[0] = 9.0
    row = as_stored(row, code)
    kept, _, W = pm.choose(row, **ask)
    assert 0 in kept and len(kept) > 100 and kept.max() < likely
    share = int(W[0]) * 2 ** 32 // int(W[kept].sum())
    assert 2 ** 28 < share < 2 ** 31
    u = np.array([0, 1, share // 2, share - 2 ** 13, share + 2 ** 13, 2 ** 31, 3 * 2 ** 30, 2 ** 32 - 1, *rng.integers(0, 2 ** 32, 4)])
    x = np.tile(row, (len(u), 1))
    values, *got = run(code, x, [ask] * len(u), 1, u)
    check_rows(values, [ask] * len(u), 1, u, *got)
    assert got[0][:4].tolist() == [0] * 4 and (got[0][4:8] > 0).all()


def both_sides(x, asked, code, rng):
    """Eight rows, which segments take, against the model; and 33 times as many, which are a workgroup's each: the same."""
    u = rng.integers(0, 2 ** 32, 8)
    values, *few = run(code, x, asked, 1, u)
    check_rows(values, asked, 1, u, *few)
    _, *many = run(code, np.tile(x, (33, 1)), asked * 33, 1, np.tile(u, 33))
    for a, b in zip(few, many):
        np.testing.assert_array_equal(b.reshape(33, *a.shape), np.broadcast_to(a, (33, *a.shape)))


def shuffled(x, rng):
    return np.stack([row[rng.permutation(len(row))] for row in x]).astype(np.float32)


@pytest.mark.parametrize("code", [tlt.TLT_F32, tlt.TLT_BF16])
@pytest.mark.parametrize("V", [20000, 70001])
def test_differences_that_fp32_does_not_hold(code, V):
    """Logits at both ends of the type, and temperatures at which they weigh all the same: 400 tokens are within fp32's range of the largest, the first top_k reach behind them."""
    rng = np.random.default_rng(V)
    x = np.full((8, V), -math.inf)
    x[:, :400], x[:, 400:1400] = 3e38, -3e38
    asked = [dict(top_k=k, top_p=p, tau=tau) for k, p, tau in ((1000, 0.99, math.inf), (1300, 0.5, 1e38), (1399, 0.9, 3e38), (600, 0.9, 2e37), (1000, 0.3, math.inf), (1399, 0.2, math.inf), (700, 0.999, 2e38),
                                                               (500, 0.9, 1e38))]
    both_sides(shuffled(x, rng), asked, code, rng)


@pytest.mark.parametrize("code", [tlt.TLT_F32, tlt.TLT_BF16])
@pytest.mark.parametrize("kind", ["mask", "lowest", "two bells", "ends"])
@pytest.mark.parametrize("V", [20000, 70001])
def test_top_k_past_the_tokens_that_weigh_anything_with_top_p(code, kind, V):
    """The share of top_p is that of the first top_k tokens, of which most weigh nothing."""
    rng = np.random.default_rng(V + len(kind))
    x = rng.normal(0.0, 2.0, (8, V))
    if kind == "mask":            # a finite mask instead of -infinity
        x[:, 3000:] = -1e4
    if kind == "lowest":          # the lowest values of fp16 and fp32 as masks (in bf16 the latter is -infinity)
        x[:4, 4000:], x[4:, 4000:] = -65504.0, float(np.finfo(np.float32).min)
    if kind == "two bells":
        x[:, :3000] *= 0.5
        x[:, 3000:] = rng.normal(-40.0, 0.5, (8, V - 3000))
    if kind == "ends":            # differences that fp32 does not hold
        x[:, :400], x[:, 400:] = 3e38, -3e38
    asked = [dict(top_k=k, top_p=p, tau=tau) for k, p, tau in ((5000, 0.9, 1.0), (5000, 0.95, 0.8), (4500, 0.9, 0.7), (7000, 0.5, 0.3), (4001, 0.999, 1.0), (19000, 0.9, 0.6), (5000, 1e-9, 1.0),
                                                               (8100, 1.0 - 2.0 ** -24, 0.5))]
    both_sides(shuffled(x, rng), asked, code, rng)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("code,V", [(tlt.TLT_F32, 152064), (tlt.TLT_BF16, 131073), (tlt.TLT_F32, 70001), (tlt.TLT_BF16, 65536)])
def test_every_setting_on_rows_of_16_and_32_segments(code, V, kind):
    """Rows at the vocabularies of models (16 segments from 65536 tokens on, 32 from 131072): every setting, 28 rows at a time and three, which have as many segments."""
    rng = np.random.default_rng(V + len(kind))
    x = logits_of(kind, 28, V, rng)
    u = rng.integers(0, 2 ** 32, 28)
    asked = asks(rng, 28)
    values, *got = run(code, x, asked, 1, u, pad=V % 4)
    check_rows(values, asked, 1, u, *got)
    for r in range(0, 28, 3):
        _, *three = run(code, x[r:r + 3], asked[r:r + 3], 1, u[r:r + 3])
        for a, b in zip(three, got):
            np.testing.assert_array_equal(a, b[r:r + 3])


@pytest.mark.parametrize("code", [tlt.TLT_F32, tlt.TLT_BF16])
def test_rows_of_several_segments_in_two_passes(code):
    """More rows than are taken at a time: every pass finds its counters cleared, whatever the one before left."""
    rng = np.random.default_rng(13)
    V, rows = 8200, 1100                     # (two passes of 550 rows, of two segments each)
    x = np.concatenate([logits_of(kind, 25, V, rng) for kind in KINDS] * 6)[:rows]
    u = rng.integers(0, 2 ** 32, rows)
    asked = (asks(rng, 27) * 41)[:rows]
    dt = tlt.torch_dtype(code)
    logits = torch.from_numpy(x).cuda().to(dt)
    token, kept = (torch.full((rows,), 9, dtype=torch.int32, device="cuda") for _ in range(2))
    logprob, ws = torch.zeros((rows, 2), device="cuda"), tlt.sample_workspace(rows, V)
    ws.fill_(255)
    tlt.sample(code, logits, filter_of(asked), torch.from_numpy(u.astype(np.uint32).view(np.int32)).cuda(), token, logprob, kept, ws)
    check_rows(logits.double().cpu().numpy(), asked, 1, u, token.cpu().numpy(), logprob.cpu().numpy(), kept.cpu().numpy())
