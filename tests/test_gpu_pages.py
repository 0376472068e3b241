"""tlt_pages_grow and tlt_pages_release against the model, bit for bit: tables, stack, counts, slots."""
import numpy as np
import pytest
import torch

import pages_model as pm
from paper_2511_16665_amd import binding as tlt

pytestmark = pytest.mark.gpu


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Both:
    """The model and the device's state side by side."""

    def __init__(self, state, page):
        free, n_free, count, table = state
        self.m = pm.Model(free, n_free, count, table, page)
        self.pages = tlt.Pages(cuda(free), cuda(np.array([n_free], np.int32)), cuda(count), cuda(table), page)

    def grow(self, seq_len, n_new, depth, rows):
        B = len(seq_len)
        i32 = lambda n: torch.full((n,), 99, dtype=torch.int32, device="cuda")
        out = (i32(B + 1), i32(rows), i32(rows), torch.full((rows,), 99, dtype=torch.int64, device="cuda"), i32(B))
        tlt.pages_grow(self.pages, cuda(seq_len.astype(np.int32)), cuda(n_new.astype(np.int32)), None if depth is None else cuda(depth.astype(np.int32)), *out)
        for got, want in zip(out, self.m.grow(seq_len, n_new, depth, rows)):
            np.testing.assert_array_equal(got.cpu().numpy(), want)
        self.check()

    def release(self, keep):
        tlt.pages_release(self.pages, None if keep is None else cuda(keep.astype(np.int32)))
        self.m.release(keep)
        self.check()

    def check(self):
        for got, want in ((self.pages.free_page, self.m.free), (self.pages.page_count, self.m.count), (self.pages.block_table, self.m.table)):
            np.testing.assert_array_equal(got.cpu().numpy(), want)
        assert int(self.pages.n_free) == self.m.n_free


@pytest.mark.parametrize("B,page,most,new", [(1, 16, 1, 1), (1, 1, 300, 40), (3, 16, 500, 7), (32, 16, 900, 48), (64, 7, 200, 33), (1000, 16, 60, 3), (1025, 5, 20, 2), (4096, 16, 40, 4)])
@pytest.mark.parametrize("short", [False, True])
def test_steps(B, page, most, new, short):
    rng = np.random.default_rng(B + page)
    lens = rng.integers(0, most + 1, B)
    width = -(-(most + 3 * new) // page) + 2
    need = B * (-(-new // page) + 1)
    s = Both(pm.state(rng, B, page, lens, width, need // 3 if short else 3 * need, over=2), page)
    for step in range(3):
        n_new = rng.integers(0, new + 1, B)
        rows = max(1, int(n_new.sum()) + int(rng.integers(-3, 9)))
        before = s.m.count.copy()
        s.grow(lens, n_new, rng.integers(0, 5, rows) if step == 1 else None, rows)
        kept = np.where(rng.random(B) < 0.2, 0, lens + rng.integers(0, new + 1, B) // 2)
        served = s.m.count >= -(-kept // page)
        lens = np.where(served, kept, np.minimum(lens, before * page))
        s.release(lens)
    s.release(None)


@pytest.mark.parametrize("B", [3, 200])
def test_many_rows_by_many_workgroups(B):
    """Prompts: more rows than one workgroup takes, then all given back (tables of more entries than one workgroup takes)."""
    rng = np.random.default_rng(B)
    n_new = np.where(rng.random(B) < 0.7, rng.integers(1, 40000 // B * 2, B), 0)
    n_new[0] = 20000
    lens = np.zeros(B, np.int64)
    width = 160000 // B + 20
    for spare in (int((-(-n_new // 16)).sum()) + 5, int((-(-n_new // 16)).sum()) // 2):
        s = Both(pm.state(rng, B, 16, lens, width, spare), 16)
        s.grow(lens, n_new, None, int(n_new.sum()) + 100)
        s.grow(np.where(s.m.count > 0, n_new, 0), np.ones(B, np.int64), None, B)
        s.release(np.where(rng.random(B) < 0.5, 17, n_new))
        s.release(None)
        assert s.m.n_free == spare


def test_many_pages_given_back():
    rng = np.random.default_rng(1)
    lens = rng.integers(1, 800, 500)
    s = Both(pm.state(rng, 500, 1, lens, 801, 3), 1)
    s.release(lens // 3)
    s.release(None)


def test_states_that_cannot_be():
    """Counts outside the table, a table that is too narrow, lengths below zero, ids that are no pages, an overfull or negative stack."""
    rng = np.random.default_rng(2)
    lens = np.array([5, 9, 0, 20, 7, 3])
    free, n, count, table = pm.state(rng, 6, 4, lens, 8, 12)
    count[1], count[4] = -1, 9
    table[0, 0], free[n - 1], free[n - 2] = 10 ** 6, -5, 77777
    s = Both((free, n, count, table), 4)
    s.grow(np.array([5, 9, -3, 20, 7, 3]), np.array([4, 4, 3, 100, 4, -2]), None, 30)
    s.release(np.array([-4, 0, 1, 2, 0, 3]))
    for bad in (-3, 10 ** 6):
        s = Both((free, bad, count, table), 4)
        s.grow(np.array([5, 9, 0, 20, 7, 3]), np.array([0, 4, 9, 1, 4, 9]), None, 30)
        s.release(None)


def test_row_sums_past_32_bits():
    """Lengths whose sum does not fit 32 bits: starts are held at the largest number, nothing is granted that the table cannot hold."""
    rng = np.random.default_rng(3)
    free, n, count, table = pm.state(rng, 4, 16, np.zeros(4, np.int64), 8, 40)
    start, seq, slot, granted = torch.empty((5,), dtype=torch.int32).cuda(), torch.empty((40,), dtype=torch.int32).cuda(), torch.empty((40,), dtype=torch.int64).cuda(), torch.empty((4,), dtype=torch.int32).cuda()
    pages = tlt.Pages(cuda(free), cuda(np.array([n], np.int32)), cuda(count), cuda(table), 16)
    tlt.pages_grow(pages, cuda(np.zeros(4, np.int32)), cuda(np.array([30, 2 ** 31 - 1, 2 ** 31 - 1, 5], np.int32)), None, start, seq, None, slot, granted)
    assert start.tolist() == [0, 30] + [2 ** 31 - 1] * 3 and granted.tolist() == [1, 0, 0, 1] and int(pages.n_free) == n - 3
    assert seq.tolist() == [0] * 30 + [1] * 10 and bool((slot[30:] == -1).all()) and bool((slot[:30] >= 0).all())


def test_without_outputs_and_captured():
    """No outputs at all; a captured pair of calls replayed with eager work between."""
    pages = tlt.Pages.empty(3, 20, 6, 16)
    seq_len, n_new = cuda(np.array([0, 3, 40], np.int32)), cuda(np.array([17, 1, 0], np.int32))
    tlt.pages_grow(pages, seq_len, n_new, None, None, None, None, None, None)
    assert pages.page_count.tolist() == [2, 1, 3] and pages.block_table[0, :2].tolist() == [0, 1] and int(pages.n_free) == 14
    slot, position = torch.empty((24,), dtype=torch.int64, device="cuda"), torch.empty((24,), dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    step = lambda: (tlt.pages_grow(pages, seq_len, n_new, None, None, None, position, slot, None), tlt.pages_release(pages, seq_len))
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        step()
    rng = np.random.default_rng(0)
    for _ in range(4):
        lens, new = rng.integers(0, 30, 3), rng.integers(0, 9, 3)
        tlt.pages_release(pages, None)
        seq_len.copy_(cuda(lens.astype(np.int32)))
        tlt.pages_grow(pages, torch.zeros_like(seq_len), seq_len, None, None, None, None, None, None)
        n_new.copy_(cuda(new.astype(np.int32)))
        m = pm.Model(pages.free_page.cpu().numpy(), int(pages.n_free), pages.page_count.cpu().numpy(), pages.block_table.cpu().numpy(), 16)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        _, _, want_pos, want_slot, _ = m.grow(lens, new, None, 24)
        m.release(lens)
        np.testing.assert_array_equal(position.cpu().numpy(), want_pos)
        np.testing.assert_array_equal(slot.cpu().numpy(), want_slot)
        np.testing.assert_array_equal(pages.block_table.cpu().numpy(), m.table)
        np.testing.assert_array_equal(pages.free_page.cpu().numpy(), m.free)
        assert int(pages.n_free) == m.n_free
