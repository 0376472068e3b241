"""The page calls one page at a time on the host."""
import numpy as np


class Model:
    def __init__(self, free, n_free, count, table, page):
        self.free, self.n_free, self.count, self.table, self.page = free.copy(), int(n_free), count.copy(), table.copy(), page
        self.n_pages, self.width = len(free), table.shape[1]

    def grow(self, seq_len, n_new, depth, rows):
        B = len(seq_len)
        left, stop = min(max(self.n_free, 0), self.n_pages), False
        granted, start = np.zeros(B, np.int32), np.zeros(B + 1, np.int64)
        row_seq, position, slot = np.full(rows, -1, np.int32), np.zeros(rows, np.int32), np.full(rows, -1, np.int64)
        for b in range(B):
            n0, n = max(int(seq_len[b]), 0), max(int(n_new[b]), 0)
            held, need = int(self.count[b]), -(-(n0 + n) // self.page)
            ok = 0 <= held <= self.width and need <= self.width
            want = max(need - held, 0) if ok else 0
            stop = stop or want > left                # sequences are served in order: behind the first that does not fit nothing is taken
            granted[b] = ok and (want == 0 or not stop)
            if granted[b] and want:
                for j in range(want):
                    left -= 1
                    self.table[b, held + j] = self.free[left]
                self.count[b] += want
            start[b + 1] = start[b] + n
            for i in range(n):
                t = start[b] + i
                if t >= rows:
                    break
                row_seq[t], position[t] = b, n0 + (int(depth[t]) if depth is not None else i)
                at = n0 + i
                if granted[b] and at // self.page < self.count[b]:
                    pg = int(self.table[b, at // self.page])
                    if 0 <= pg < self.n_pages:
                        slot[t] = pg * self.page + at % self.page
        self.n_free = left
        return np.minimum(start, 2 ** 31 - 1).astype(np.int32), row_seq, position, slot, granted

    def release(self, keep_len):
        B, free = len(self.count), min(max(self.n_free, 0), self.n_pages)
        keep = np.zeros(B, np.int64) if keep_len is None else -(-np.maximum(keep_len.astype(np.int64), 0) // self.page)
        give = [max(int(self.count[b]) - int(keep[b]), 0) if 0 <= self.count[b] <= self.width else 0 for b in range(B)]
        if free + sum(give) > self.n_pages:
            return
        for b in reversed(range(B)):
            for j in reversed(range(int(self.count[b]) - give[b], int(self.count[b]))):
                self.free[free], self.table[b, j] = self.table[b, j], -1
                free += 1
            self.count[b] -= give[b]
        self.n_free = free


def state(rng, B, page, lens, width, spare, over=0):
    """Sequences that hold the pages of their lengths (and `over` more now and then), `spare` free pages, ids in random order."""
    held = -(-np.asarray(lens) // page) + (rng.integers(0, over + 1, B) if over else 0)
    n_pages = int(held.sum()) + spare
    order = rng.permutation(n_pages).astype(np.int32)
    table, o = np.full((B, width), -1, np.int32), 0
    for b in range(B):
        table[b, :held[b]] = order[o:o + held[b]]
        o += held[b]
    free = rng.integers(0, n_pages, n_pages).astype(np.int32)      # (what lies above the stack means nothing)
    free[:spare] = order[o:]
    return free, spare, held.astype(np.int32), table
