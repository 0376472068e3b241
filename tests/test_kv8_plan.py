"""How the attention over the 8-bit cache cuts sequences into ranges, on the host: the rule's properties, and the model against the workspace that the library asks for."""
import numpy as np
import pytest

import kv8_model as m
import kv8_plan_model as pm
from paper_2511_16665_amd import binding as tlt

HEADS = [(28, 4), (40, 8), (64, 8), (4, 1), (40, 20), (64, 2), (96, 32)]


@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_the_model_asks_for_the_librarys_workspace(Hq, Hkv):
    size = tlt.load().tlt_kv8_attention_workspace_bytes
    for B in (1, 2, 5, 16, 31, 33, 64, 80, 112, 129, 160, 200, 255, 256, 257, 700):
        for n in (1, 4, 16, 33, 64):
            for total in (1, 65, 300, 513, 4096, 4097, 8200, 30001, 100000):
                assert size(B, n, Hq, Hkv, 128, total) == max(256, *(pm.plan(B, k, Hq, Hkv, total).bytes for k in range(1, n + 1)), 0), (B, n, total)


@pytest.mark.parametrize("seed", range(8))
def test_ranges_fit_and_are_as_short_as_they_may_be(seed):
    """Every tile lies in one range of at most 64 tiles; the ranges are no more than the grid has items, and no more than the rounds that ranges of 64 would take;
    shorter ones would be more than that, or are not worth a joining."""
    rng = np.random.default_rng(seed)
    searched = 0
    for _ in range(400):
        B, n = int(np.exp(rng.uniform(0, np.log(300)))), int(rng.choice([1, 1, 2, 8, 16, 30, 48, 64]))
        Hq, Hkv = HEADS[rng.integers(len(HEADS))]
        lens = np.minimum(np.exp(rng.normal(np.log(rng.choice([40, 500, 4000, 20000])), rng.choice([0.0, 0.5, 1.5]), B)).astype(np.int64), 200000)
        bound = int(lens.max()) + int(rng.choice([0, 0, 100, 5000]))
        p = pm.plan(B, n, Hq, Hkv, bound + n)
        first, k = pm.segments(lens, n, p)
        tiles = -(-(lens + n) // 64)
        assert (k >= 1).all() and (-(-tiles // k) <= 64).all() and (k <= tiles).all()      # (ranges differ by a tile at most)
        assert not p.one_each or (k == 1).all()
        if p.planned:
            T = pm.range_length(tiles, p)
            items = lambda t: int((-(-tiles // t)).sum())
            assert first[-1] + k[-1] == items(T) <= p.max_items and 2 <= T <= 64
            if T > pm.shortest(int(tiles.max()), p.whole):
                searched += 1
                most = -(-items(64) // p.slots) * p.slots
                assert items(T) <= most < items(T - 1)
        else:
            assert int(((k - 1) * B + np.arange(B)).max()) < p.max_items
    assert searched > 20


def test_attention_of_single_rows_is_the_models():
    c = m.Cache([200, 40], 5, 2, 128, 16, seed=3, dev="cpu")
    rng = np.random.default_rng(0)
    q = rng.standard_normal((5, 6, 128))
    mask = m.random_trees(rng, 2, 5)[1]
    for b in range(2):
        out, tol = m.attention(c, b, q, mask[b])
        for h in (0, 2, 5):
            o, t = pm.attention_rows(c, b, q[[1, 4], h], mask[b], [1, 4], h, 3)
            np.testing.assert_allclose(o, out[[1, 4], h], rtol=1e-12, atol=1e-13)
            np.testing.assert_allclose(t, tol[[1, 4], h], rtol=1e-9)
