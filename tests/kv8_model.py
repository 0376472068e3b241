"""The 8-bit cache in float64 on the host: its format from the definition, caches for tests, attention with an error bound, commit and read."""
import numpy as np
import torch

from paper_2511_16665_amd import binding as tlt
from synth import random_block_table

# every e4m3 code's value (0x7f and 0xff do not occur)
E4M3 = np.array([(-1.0 if c & 128 else 1.0) * ((1 + (c & 7) / 8) * 2.0 ** ((c >> 3 & 15) - 7) if c >> 3 & 15 else (c & 7) / 8 * 2.0 ** -6)
                 for c in range(256)])
POSITIVE = E4M3[:127]


def encode(x):
    """Rows [..., d] (float64 holding fp32 values) -> (codes uint8, exponent bytes uint8), by the definition."""
    x = np.asarray(x, dtype=np.float64)
    finite = np.isfinite(x).all(-1)
    y = np.where(finite[..., None], x, 0.0)
    amax = np.abs(y).max(-1)
    e = np.full(amax.shape, -126)
    while True:                                   # the smallest e >= -126 with amax <= 448 * 2^e
        more = amax > 448.0 * np.exp2(e.astype(np.float64))
        if not more.any():
            break
        e = e + more
    z = y / np.exp2(e.astype(np.float64))[..., None]
    a = np.abs(z)
    hi = np.searchsorted(POSITIVE, a)             # first value >= a
    lo = np.maximum(hi - 1, 0)
    hi = np.minimum(hi, 126)
    down, up = a - POSITIVE[lo], POSITIVE[hi] - a
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    code = np.where(a == POSITIVE[hi], hi, code) | np.where(np.signbit(z), 128, 0)
    return np.where(finite[..., None], code, 0).astype(np.uint8), np.where(finite, e + 127, 255).astype(np.uint8)


def decode(codes, exps):
    s = np.where(exps == 255, np.nan, np.exp2(np.minimum(exps, 254).astype(np.float64) - 127.0))
    return E4M3[codes] * s[..., None]


class Cache:
    """A cache with random contents on the device, its tables, and what it holds on the host."""

    def __init__(self, ctxs, n, Hkv, d, page=16, layers=1, seed=0, extra=3, dev="cuda"):
        self.ctx, self.page, self.L = np.asarray(ctxs, np.int32), page, layers
        self.table, n_pages = random_block_table(self.ctx + n, page, seed, extra_pages=extra)
        rng = np.random.default_rng(seed + 1)
        shape = (layers, n_pages, Hkv, page)
        self.codes, self.exps = {}, {}
        for x in ("k", "v"):
            vals = rng.standard_normal((*shape, d), dtype=np.float32) * np.exp2(rng.integers(-3, 3, shape))[..., None]
            self.codes[x], self.exps[x] = encode(vals) if vals.size < 4e6 else _encode_fast(vals)
        self.dev = dev
        if dev == "cuda":
            self.upload()

    def upload(self):
        cu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        self.kv = tlt.KV8(cu(self.codes["k"]), cu(self.codes["v"]), cu(self.exps["k"]), cu(self.exps["v"]), cu(self.table.astype(np.int32)),
                          cu(self.ctx), int(self.ctx.max()))

    def rows(self, x, layer, b, lo, hi):
        """Values [hi - lo, Hkv, d] of slots lo .. hi - 1; slots without a page: zeros."""
        at = np.arange(lo, hi)
        lp = at // self.page
        pg = np.where(lp < self.table.shape[1], self.table[b, np.minimum(lp, self.table.shape[1] - 1)], -1)
        ok = (pg >= 0) & (pg < self.codes[x].shape[1])
        pg = np.where(ok, pg, 0)
        v = decode(self.codes[x][layer, pg, :, at % self.page], self.exps[x][layer, pg, :, at % self.page])
        return np.where(ok[:, None, None], v, 0.0)


def _encode_fast(x):
    """encode for many finite fp32 rows."""
    t = torch.from_numpy(x)
    m, e = torch.frexp(t.abs().amax(-1))
    e = torch.where(m > 0, (e - 9 + (m > 0.875).int()).clamp(min=-126), -126)
    return (t * torch.exp2(-e.float())[..., None]).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), (e + 127).to(torch.uint8).numpy()


def random_trees(rng, B, n, back=5):
    depth, mask = np.zeros((B, n), np.int32), np.zeros((B, n), np.uint64)
    for b in range(B):
        for i in range(n):
            p = int(rng.integers(max(0, i - back), i)) if i else -1
            depth[b, i] = depth[b, p] + 1 if i else 0
            mask[b, i] = (mask[b, p] if i else np.uint64(0)) | np.uint64(1 << i)
    return depth, mask


def attention(cache, b, q, mask, layer=0, rounded=True):
    """q [n, Hq, d] float64, mask [n] uint64 or None -> (out, allowed error), both [n, Hq, d].

    Allowed: with `rounded` (bf16) every weight is rounded by at most half a step, 2^-8 of it, in numerator and denominator alike, which moves
    the weighted mean o by at most 2^-8 * (mean of |v| + |o|), and the result by another 2^-8 |o|; fp32: 2^-22 instead, a few
    roundings of a weight and of a sum.  A score is a sum of d products and may be off by (d + 8) 2^-24 of the sum of their magnitudes (the
    queries of the matrix instructions are held to 2^-20 of the row's largest element: another 2^-20 max|q| sum|k|), and its exponential by as much
    again plus 2^-20; a weight off by a factor 1 + t moves the mean by 2 t max|v| at most."""
    n, Hq, d = q.shape
    T = int(cache.ctx[b]) + n
    K, V = cache.rows("k", layer, b, 0, T), cache.rows("v", layer, b, 0, T)
    G = Hq // K.shape[1]
    seen = np.ones((n, T), dtype=bool)
    for i in range(n):
        for j in range(n):
            seen[i, T - n + j] = j <= i if mask is None else bool((int(mask[i]) >> j) & 1)
    out, tol = np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
    u = 2.0 ** -8 if rounded else 2.0 ** -22
    for h in range(Hq):
        k, v = K[:, h // G], V[:, h // G]
        for i in range(n):
            on = seen[i]
            if not on.any():
                continue
            s = k[on] @ q[i, h] / np.sqrt(d)
            if not np.isfinite(s).all():
                out[i, h] = np.nan
                continue
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h] = p @ v[on]
            mags = np.abs(k[on]) @ np.abs(q[i, h]) / np.sqrt(d)
            ds = ((d + 8) * 2.0 ** -24 * mags + 2.0 ** -20 * (np.abs(q[i, h]).max() * np.abs(k[on]).sum(1) / np.sqrt(d) + 1)).max()
            tol[i, h] = u * (p @ np.abs(v[on]) + 2 * np.abs(out[i, h])) + 2 * ds * np.abs(v[on]).max()
    return out, tol
