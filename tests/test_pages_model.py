"""What the page calls promise, on the model that the kernels are held to."""
import numpy as np

import pages_model as pm


def test_growing_and_giving_back_returns_to_the_same_state():
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 50, 9)
    m = pm.Model(*pm.state(rng, 9, 4, lens, 40, 60, over=2), page=4)
    before = (m.free.copy(), m.n_free, m.count.copy(), m.table.copy())
    held = m.count.copy()
    start, seq, pos, slot, granted = m.grow(lens, rng.integers(0, 20, 9), None, 200)
    real = slot >= 0
    assert granted.all() and len(set(slot[real])) == real.sum() == start[-1]             # every row has a slot of its own
    for t in np.flatnonzero(real):
        assert m.table[seq[t], pos[t] // 4] * 4 + pos[t] % 4 == slot[t]
    m.release(held.astype(np.int64) * 4)
    assert m.n_free == before[1] and all((a == b).all() for a, b in zip((m.free, m.count, m.table), (before[0], before[2], before[3])))


def test_served_in_order():
    free, n, count, table = np.arange(10, dtype=np.int32), 3, np.zeros(4, np.int32), np.full((4, 8), -1, np.int32)
    m = pm.Model(free, n, count, table, 4)
    start, seq, pos, slot, granted = m.grow(np.zeros(4, np.int32), np.array([5, 8, 0, 1]), None, 16)
    assert granted.tolist() == [1, 0, 1, 0] and m.n_free == 1 and m.table[0, :2].tolist() == [2, 1]
    assert slot[:5].tolist() == [8, 9, 10, 11, 4] and (slot[5:] == -1).all() and seq.tolist() == [0] * 5 + [1] * 8 + [3] + [-1] * 2
