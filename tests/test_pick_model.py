"""The model that the sampling kernels are held to, on cases worked by hand and against straightforward formulas."""
import math

import numpy as np
import pytest

import pick_model as pm


def keep(l, **ask):
    return pm.choose(l, **ask)[0].tolist()


def test_prefixes_by_hand():
    l = np.log(np.array([1.0, 8.0, 4.0, 2.0, 1.0]))           # order 1, 2, 3, 0, 4
    assert keep(l) == [1, 2, 3, 0, 4]
    assert keep(l, top_k=2) == [1, 2]
    assert keep(l, top_p=0.49) == [1]                 # 8 / 16 reaches 0.49
    assert keep(l, top_p=0.51) == [1, 2]
    assert keep(l, top_p=0.0) == [1]
    assert keep(l, top_k=3, top_p=0.6) == [1, 2]      # of 14: 8 is less than 8.4
    assert keep(l, top_k=3, top_p=0.5) == [1]
    assert keep(l, min_p=0.3) == [1, 2]
    assert keep(l, min_p=1.0) == [1]
    assert keep(l, tau=0.0) == keep(l, tau=-1.0) == keep(l, tau=math.nan) == [1]
    assert keep([2.0, 2.0, 2.0], top_k=2) == [0, 1]   # ties: the lower index
    assert keep([-math.inf, 0.0], top_k=2) == [1]
    assert keep([math.inf, 0.0, math.inf]) == [0, 2, 1] and keep([math.inf, 0.0, math.inf], min_p=0.1) == [0, 2]


@pytest.mark.parametrize("tau", [0.6, 1.0, 1.7])
def test_draws_follow_the_filtered_softmax(tau):
    rng = np.random.default_rng(3)
    l = rng.normal(0, 2, 40).astype(np.float32).astype(np.float64)
    kept, _, _ = pm.choose(l, tau=tau, top_k=9, top_p=0.9)
    p = np.exp(l / np.float64(np.float32(tau)))
    q = np.where(np.isin(np.arange(40), kept), p, 0.0)
    q /= q.sum()
    us = (np.arange(4000) + 0.5) / 4000 * 2 ** 32
    got = np.bincount([pm.draw(l, u, tau=tau, top_k=9, top_p=0.9)[0] for u in us], minlength=40) / 4000
    assert np.abs(got - q).max() <= 1.01 / 4000               # (a grid of uniforms: a token's share of it is off by one point at most)
    j, lp, n = pm.draw(l, 0, tau=tau, top_k=9, top_p=0.9)
    assert n == len(kept) and abs(lp[0] - math.log(q[j])) < 1e-7 and abs(lp[1] - math.log(p[j] / p.sum())) < 1e-7
