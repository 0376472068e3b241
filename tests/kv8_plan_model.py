"""How tlt_kv8_attention cuts sequences into ranges (plan_kv8, kv8_item, shortest_range), in plain Python, and attention of single rows of long caches."""
import dataclasses

import numpy as np

import kv8_model as m


@dataclasses.dataclass
class Plan:
    kernel: str
    slots: int
    whole: int
    planned: bool
    one_each: bool
    max_items: int
    bytes: int
    t_max: int = 64


def up(x):
    return -(-x // 256) * 256


def plan(B, n, Hq, Hkv, total):
    """The host's part, for lengths and new rows of `total` at most."""
    row_tiles, tiles = -(-n * (Hq // Hkv) // 16), -(-total // 64)
    kernel = "few" if row_tiles <= 2 else ("mid" if row_tiles <= 8 else "many")
    groups = 1 if kernel == "few" else -(-row_tiles // 24)
    slots = max(1, (256 if kernel == "many" else 512) // (Hkv * groups))
    whole = 8 if kernel == "few" else 4
    planned = B <= 256 and (B <= 4 * slots if tiles > 64 else B < slots)
    one_each = tiles <= (whole if planned else 64)
    longest = B * -(-tiles // 64)
    rounds = -(-min(longest, B * tiles // 64 + B) // slots)
    items = B if one_each else (rounds * slots if planned else longest)
    rows = items * Hkv * row_tiles * 16
    return Plan(kernel, slots, whole, planned, one_each, items, up(8 * B) + up(8 * rows) + up(512 * rows))


def shortest(tiles, whole):
    return min(max(tiles if tiles <= whole else int(np.sqrt(np.float32(tiles) * np.float32(1 / 7))), 2), 32)


def range_length(tiles, p):
    """Tiles of a range: the shortest worth while, or where those are more than run at once the smallest that needs no more rounds than ranges of 64."""
    items = lambda T: int((-(-tiles // T)).sum())
    T = shortest(int(tiles.max()), p.whole)
    if items(T) > p.slots:
        most = -(-items(p.t_max) // p.slots) * p.slots
        T = next(t for t in range(T, p.t_max + 1) if items(t) <= most)
    return T


def segments(lens, n, p):
    """(number of the first range, ranges) of every sequence."""
    tiles = -(-(np.asarray(lens, dtype=np.int64) + n) // 64)
    k = -(-tiles // (range_length(tiles, p) if p.planned else p.t_max))
    return (np.cumsum(k) - k if p.planned else np.arange(len(k))), k


def long_cache(lens, n, Hkv, seed):
    """A cache of head_dim 128 whose bytes are drawn directly: values up to 3.75 in magnitude, most of them small."""
    c = object.__new__(m.Cache)
    c.ctx, c.page, c.L, c.dev = np.asarray(lens, np.int32), 16, 1, "cuda"
    c.table, n_pages = m.random_block_table(c.ctx + n, 16, seed, extra_pages=3)
    rng = np.random.default_rng(seed + 1)
    shape = (1, n_pages, Hkv, 16)
    byte = lambda: np.frombuffer(rng.bytes(int(np.prod(shape)) * 128), np.uint8).reshape(*shape, 128)
    c.codes, c.exps = {}, {}
    for x in ("k", "v"):
        b = byte()
        c.codes[x] = np.where(b & 0x7f == 0x7f, 0x38, b).astype(np.uint8)
        c.exps[x] = rng.integers(117, 121, shape, dtype=np.uint8)
    return c


def attention_rows(c, b, q, masks, nodes, head, heads_per_kv):
    """q [len(nodes), d] float64, the rows of `nodes` and one query head of sequence b; masks [n] uint64 -> (out, allowed error), as kv8_model.attention in bf16."""
    n, d, T = len(masks), q.shape[1], int(c.ctx[b]) + len(masks)
    kh = head // heads_per_kv
    at = np.arange(T)
    pg = c.table[b, at // c.page]
    K, V = (m.decode(c.codes[x][0, pg, kh, at % c.page], c.exps[x][0, pg, kh, at % c.page]) for x in ("k", "v"))
    out, tol = np.zeros((len(nodes), d)), np.zeros((len(nodes), d))
    for r, i in enumerate(nodes):
        on = np.ones(T, bool)
        on[T - n:] = [(int(masks[i]) >> j) & 1 for j in range(n)]
        s = K[on] @ q[r] / np.sqrt(d)
        p = np.exp(s - s.max())
        p /= p.sum()
        out[r] = p @ V[on]
        absk = np.abs(K[on])
        ds = ((d + 8) * 2.0 ** -24 * (absk @ np.abs(q[r])) / np.sqrt(d) + 2.0 ** -20 * (np.abs(q[r]).max() * absk.sum(1) / np.sqrt(d) + 1)).max()
        tol[r] = 2.0 ** -8 * (p @ np.abs(V[on]) + 2 * np.abs(out[r])) + 2 * ds * np.abs(V[on]).max()
    return out, tol
