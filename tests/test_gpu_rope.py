"""tlt_rope_write against rotation in float64: queries, keys and values in rows, in the cache of the model's type and in 8 bits.

Tolerance of a turned element, before it is rounded to its type: x = row + bias is one fp32 rounding (2^-24); the angle reaches the sine and cosine as a fraction of a half turn
rounded to fp32 (2^-25 of a turn of pi: 2^-23.3), they and the amplitude's product are good to 2^-22, and two products and a sum are three more roundings: together at most
2^-21 (|a| + |b|) times the amplitude.  Rounding to the type adds half a step; 8 bits half a step of four significant bits, 2^-4 of the value, or of the smallest step, 2^-10 of
a power of two below max / 224."""
import numpy as np
import pytest
import torch

import kv8_model
from paper_2511_16665_amd import binding as tlt

pytestmark = pytest.mark.gpu


def reference(x, bias, position, freq, amplitude, rot, interleaved, turned):
    """x [R, H, d] float64 -> (turned rows, error allowed before rounding)"""
    y = x if bias is None else x + bias
    tol = np.abs(y) * 2.0 ** -23
    if bias is not None:
        tol += 2.0 ** -24 * (np.abs(x) + np.abs(bias))
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    angle = position.astype(np.float64)[:, None] * freq
    c, s = np.cos(angle)[:, None] * amplitude, np.sin(angle)[:, None] * amplitude
    a, b = y[:, :turned, one], y[:, :turned, two]
    z, t = y.copy(), tol.copy()
    z[:, :turned, one], z[:, :turned, two] = a * c - b * s, a * s + b * c
    t[:, :turned, one] = t[:, :turned, two] = 2.0 ** -21 * (np.abs(a) + np.abs(b)) * max(abs(amplitude), 2.0 ** -30)
    return z, t


def near(got, want, tol, half_step):
    ok = np.abs(got - want) <= tol + half_step * np.abs(want) * (1 + 2.0 ** -7) + 1e-37
    assert ok.all(), (int((~ok).sum()), float(np.abs(got - want).max()), np.argwhere(~ok)[:3])


class Case:
    def __init__(self, code, R, Hq, Hkv, d, rot, interleaved, bias=True, amplitude=1.0, far=40000, page=16, seed=0, extra=0, offset=0):
        rng = np.random.default_rng(seed)
        self.code, self.R, self.Hq, self.Hkv, self.d, self.page = code, R, Hq, Hkv, d, page
        dt = self.dt = tlt.torch_dtype(code)
        W = (Hq + 2 * Hkv) * d
        base = torch.from_numpy(rng.normal(0, 1.5, R * (W + extra) + offset).astype(np.float32)).cuda().to(dt)
        self.qkv = base[offset:].view(R, W + extra)[:, :W]
        self.bias = torch.from_numpy(rng.normal(0, 0.5, W).astype(np.float32)).cuda().to(dt) if bias else None
        self.pos = rng.integers(0, far, R).astype(np.int32)
        self.freq = 1e6 ** (-np.arange(0, rot, 2) / rot)
        self.rope = tlt.Rope(torch.from_numpy(self.freq).cuda(), interleaved, amplitude)
        self.n_pages = -(-(R + 5) // page) + 1
        self.slot = rng.permutation(self.n_pages * page)[:R].astype(np.int64)
        self.slot[rng.random(R) < 0.1] = -1
        if R > 2:
            self.slot[:2] = self.n_pages * page, 2 ** 40
        self.position, self.slots = torch.from_numpy(self.pos).cuda(), torch.from_numpy(self.slot).cuda()
        self.x = self.qkv.double().cpu().numpy().reshape(R, -1, d)
        b = None if self.bias is None else self.bias.double().cpu().numpy().reshape(-1, d)
        self.want, self.tol = reference(self.x, b, self.pos, self.freq, np.float64(np.float32(amplitude)), rot, interleaved, Hq + Hkv)
        self.eps = torch.finfo(dt).eps / 2

    def pools(self, seed=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        return [torch.randn((2, self.n_pages, self.Hkv, self.page, self.d), generator=g, device="cuda").to(self.dt) for _ in range(2)]

    def call(self, kv, q, kv_out=None, layer=1):
        tlt.rope_write(self.code, self.Hq, self.Hkv, self.d, self.rope, self.qkv, self.bias, self.position, self.slots if kv is not None else None, kv, layer, q, kv_out)

    def check_rows(self, got, lo, hi):
        near(got.double().cpu().numpy().reshape(self.R, hi - lo, self.d), self.want[:, lo:hi], self.tol[:, lo:hi], self.eps)

    def check_pool(self, pool, before, lo):
        """The rows with a slot are there; all others, and the other layer, are what they were."""
        ok = (self.slot >= 0) & (self.slot < self.n_pages * self.page)
        flat = lambda p: p[1].permute(0, 2, 1, 3).reshape(-1, self.Hkv, self.d).double().cpu().numpy()
        got, old = flat(pool), flat(before)
        near(got[self.slot[ok]], self.want[ok, lo:lo + self.Hkv], self.tol[ok, lo:lo + self.Hkv], self.eps)
        rest = np.ones(len(got), bool)
        rest[self.slot[ok]] = False
        np.testing.assert_array_equal(got[rest], old[rest])
        assert torch.equal(pool[0], before[0])


SHAPES = [(1, 28, 4, 128), (37, 4, 2, 64), (130, 40, 8, 128), (9, 3, 1, 192), (5, 2, 2, 256), (6, 2, 1, 80), (7, 4, 4, 6), (3, 1, 1, 2), (50, 6, 2, 96), (1000, 2, 1, 128)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("code", [tlt.TLT_F32, tlt.TLT_BF16])
@pytest.mark.parametrize("R,Hq,Hkv,d", SHAPES)
def test_into_the_cache_and_into_rows(code, R, Hq, Hkv, d, interleaved):
    for rot in sorted({d, d // 2 // 2 * 2, d // 4 // 2 * 2, 2, max(2, d - 2)} - {0}):
        c = Case(code, R, Hq, Hkv, d, rot, interleaved, bias=rot != d, amplitude=1.0 if rot == d else 1.1386, seed=rot, page=16 if d != 96 else 5)
        k, v = c.pools()
        was = k.clone(), v.clone()
        q, rows = torch.empty((R, Hq * d), dtype=c.dt, device="cuda"), torch.empty((R, 2 * Hkv * d), dtype=c.dt, device="cuda")
        table, zero = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
        c.call(tlt.KV(k, v, table, zero, 0), q, rows)
        c.check_rows(q, 0, Hq)
        c.check_rows(rows, Hq, Hq + 2 * Hkv)
        c.check_pool(k, was[0], Hq)
        c.check_pool(v, was[1], Hq + Hkv)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("code", [tlt.TLT_F32, tlt.TLT_BF16])
@pytest.mark.parametrize("R,Hq,Hkv,d", [s for s in SHAPES if s[3] % 64 == 0])
def test_into_the_8_bit_cache(code, R, Hq, Hkv, d, interleaved):
    for rot in (d, d // 2, 2):
        c = Case(code, R, Hq, Hkv, d, rot, interleaved, bias=rot == 2, seed=rot)
        q = torch.empty((R, Hq * d), dtype=c.dt, device="cuda")
        table, zero = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
        kv = tlt.KV8.empty(2, c.n_pages, Hkv, c.page, d, table, zero, 0)
        for t in (kv.k_pool, kv.v_pool):
            t.fill_(0x11)
        c.call(kv, q)
        c.check_rows(q, 0, Hq)
        ok = (c.slot >= 0) & (c.slot < c.n_pages * c.page)
        for codes, exps, lo in ((kv.k_pool, kv.k_exp, Hq), (kv.v_pool, kv.v_exp, Hq + Hkv)):
            assert bool((codes[0] == 0x11).all()) and bool((exps[0] == 127).all())
            codes, exps = codes[1].permute(0, 2, 1, 3).reshape(-1, Hkv, d).cpu().numpy(), exps[1].permute(0, 2, 1).reshape(-1, Hkv).cpu().numpy()
            want, tol = c.want[ok, lo:lo + Hkv], c.tol[ok, lo:lo + Hkv]
            got = kv8_model.decode(codes[c.slot[ok]], exps[c.slot[ok]])
            top = np.abs(want).max(-1, keepdims=True)
            near(got, want, 1.07 * tol + top * (2.0 ** -10 / 224), 2.0 ** -4)
            rest = np.ones(len(codes), bool)
            rest[c.slot[ok]] = False
            assert (codes[rest] == 0x11).all() and (exps[rest] == 127).all()


def test_the_8_bit_cache_is_written_as_its_own_call_writes_it():
    """Plain frequencies, half layout, the whole head: the same codes as tlt_kv8_write but where its angle's last bit decides a rounding."""
    B, n, Hq, Hkv, d = 3, 20, 8, 2, 128
    rng = np.random.default_rng(4)
    ctx = np.array([5, 1000, 31000], np.int32)
    table = torch.from_numpy(rng.permutation(3 * 1940).astype(np.int32).reshape(3, -1)).cuda()
    seq_len = torch.from_numpy(ctx).cuda()
    qkv = torch.from_numpy(rng.normal(0, 1.5, (B, n, (Hq + 2 * Hkv) * d)).astype(np.float32)).cuda().bfloat16()
    bias = torch.from_numpy(rng.normal(0, 0.5, (Hq + 2 * Hkv) * d).astype(np.float32)).cuda().bfloat16()
    caches = [tlt.KV8.empty(1, 3 * 1940, Hkv, 16, d, table, seq_len, 31000) for _ in range(2)]
    qs = [torch.empty((B, n, Hq * d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    tlt.kv8_write(tlt.TLT_BF16, Hq, 1e6, qkv, bias, None, caches[0], 0, qs[0])
    at = seq_len.long()[:, None] + torch.arange(n, device="cuda")
    slot = (table.long().gather(1, at // 16) * 16 + at % 16).flatten()
    freq, amp = tlt.rope_freqs("plain", d, 1e6)
    tlt.rope_write(tlt.TLT_BF16, Hq, Hkv, d, tlt.Rope(torch.from_numpy(freq).cuda(), False, amp), qkv, bias, at.int().flatten(), slot, caches[1], 0, qs[1])
    assert torch.equal(caches[0].v_pool, caches[1].v_pool) and torch.equal(caches[0].v_exp, caches[1].v_exp)
    for a, b in ((caches[0].k_pool, caches[1].k_pool), (caches[0].k_exp, caches[1].k_exp), (qs[0], qs[1])):
        assert float((a != b).float().mean()) < 1e-3 * (B * n * 16 / a.numel() * d if a.numel() > 1e5 else 1)


@pytest.mark.parametrize("code", [tlt.TLT_F32, tlt.TLT_BF16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_and_odd_places(code, interleaved):
    """Rows inside wider ones at any alignment; queries, keys and values turned where they stand; what lies beside them untouched."""
    for extra, offset in ((0, 0), (8, 8), (3, 1), (1, 0), (0, 4)):
        c = Case(code, 21, 6, 2, 64, 48, interleaved, extra=extra, offset=offset, seed=extra)
        W = 10 * 64
        wide = c.qkv.as_strided((21, W + extra), (W + extra, 1))
        beside = wide[:, W:].clone()
        c.call(None, c.qkv[:, :6 * 64], c.qkv[:, 6 * 64:])
        c.check_rows(c.qkv[:, :6 * 64].contiguous(), 0, 6)
        c.check_rows(c.qkv[:, 6 * 64:].contiguous(), 6, 10)
        assert torch.equal(wide[:, W:], beside)
    c = Case(code, 5, 4, 2, 64, 64, interleaved)
    k, v = c.pools()
    was = k.clone(), v.clone()
    table, zero = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
    c.call(tlt.KV(k, v, table, zero, 0), None)          # keys and values alone
    c.check_pool(k, was[0], 4)
    c.check_pool(v, was[1], 6)


def test_far_positions_and_values_that_are_not_finite():
    """Positions to 2^31 - 1 and negative ones; a row's NaN or infinity stays in its head."""
    c = Case(tlt.TLT_F32, 64, 2, 1, 128, 128, False, bias=False, far=2 ** 31 - 1)
    c.pos[:4] = 2 ** 31 - 1, -1, -40000, 0
    c.position.copy_(torch.from_numpy(c.pos).cuda())
    c.want, c.tol = reference(c.x, None, c.pos, c.freq, 1.0, 128, False, 3)
    # (an angle of 2^31 radians is good to 2^-22 in double)
    c.tol = c.tol + 2.0 ** -20 * np.abs(c.x).max() * 2.0 ** -1
    q = torch.empty((64, 256), device="cuda")
    c.call(None, q)
    c.check_rows(q, 0, 2)
    c.qkv[5, 3], c.qkv[6, 130], c.qkv[7, 260] = float("nan"), float("inf"), float("nan")
    kv8 = tlt.KV8.empty(2, c.n_pages, 1, c.page, 128, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda"), 0)
    c.slot[:] = np.arange(64)
    c.slots.copy_(torch.from_numpy(c.slot).cuda())
    again = torch.empty_like(q)
    c.call(kv8, again)
    bad = ~torch.isfinite(again)
    assert bad[5, [3, 67]].all() and int(bad[5].sum()) == 2 and bad[6, [130, 194]].all() and int(bad[6].sum()) == 2 and int(bad.sum()) == 4
    assert torch.equal(again[~bad], q[~bad])
    exps = kv8.k_exp[1].permute(0, 2, 1).reshape(-1)
    assert int(exps[7]) == 255 and int((exps == 255).sum()) == 1


def test_captured_and_replayed_on_another_stream():
    c = Case(tlt.TLT_BF16, 33, 8, 2, 128, 64, True)
    k, v = c.pools()
    table, zero = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
    q, kv, stream = torch.empty((33, 8 * 128), dtype=torch.bfloat16, device="cuda"), tlt.KV(k, v, table, zero, 0), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        c.call(kv, q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        c.call(kv, q)
    for seed in range(3):
        other = Case(tlt.TLT_BF16, 33, 8, 2, 128, 64, True, seed=seed + 5)
        c.qkv.copy_(other.qkv), c.bias.copy_(other.bias), c.position.copy_(other.position), c.slots.copy_(other.slots)
        was = k.clone(), v.clone()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        other.check_rows(q, 0, 8)
        other.check_pool(k, was[0], 8)
        other.check_pool(v, was[1], 10)
