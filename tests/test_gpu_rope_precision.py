"""How precisely tlt_rope_write turns a pair, in fp32.

x = row + bias is rounded once.  The angle is reduced exactly from a product in double, of which three roundings (1 / 2 pi, its product with the frequency, that with the position) are at most
3 * 2^-53 of the angle, and what `position * freq` loses here is one more; sine and cosine are series in double that end below 2^-37, times the amplitude and rounded to fp32 once.  Two products
and their sum are rounded once each.  With A = |a cos| + |b sin| (of the amplitude) that is 2^-24 A for x, for sine and cosine, for the products and for the sum: 2^-22 A together, up to products of these
errors; and 2^-35 (|a| + |b|) of the amplitude for the series and the angle, up to 2^15 radians (2^-37 and 2^-36).  (An angle that passes through fp32, or sine and cosine of fp32, would be off by 2^-25 or more whatever a cos is: where
cos is small that is many times this.)"""
import numpy as np
import pytest
import torch

from paper_2511_16665_amd import binding as tlt
from test_gpu_rope import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R,Hq,Hkv,d,rot,bias,amplitude", [(300, 4, 2, 128, 128, True, 1.0), (300, 4, 2, 128, 128, False, 1.1386), (200, 3, 1, 80, 20, True, 1.0), (200, 2, 2, 64, 64, False, 0.75),
                                                           (100, 2, 1, 256, 250, True, 1.0), (100, 2, 1, 256, 256, False, 1.0)])
def test_turned_pairs_to_fp32(R, Hq, Hkv, d, rot, bias, amplitude, interleaved):
    c = Case(tlt.TLT_F32, R, Hq, Hkv, d, rot, interleaved, bias=bias, amplitude=amplitude, far=32000, seed=R + rot)
    q, rows = torch.empty((R, Hq * d), device="cuda"), torch.empty((R, 2 * Hkv * d), device="cuda")
    c.call(None, q, rows)
    got = torch.cat([q, rows], 1).double().cpu().numpy().reshape(R, -1, d)[:, :Hq + Hkv]
    x = c.x[:, :Hq + Hkv] + (0.0 if c.bias is None else c.bias.double().cpu().numpy().reshape(-1, d)[:Hq + Hkv])
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    angle, scale = c.pos.astype(np.float64)[:, None] * c.freq, float(np.float32(amplitude))
    cos, sin = np.cos(angle)[:, None] * scale, np.sin(angle)[:, None] * scale
    a, b = x[..., one], x[..., two]
    rest = 2.0 ** -35 * (np.abs(a) + np.abs(b)) * scale
    for part, want, A in ((one, a * cos - b * sin, np.abs(a * cos) + np.abs(b * sin)), (two, a * sin + b * cos, np.abs(a * sin) + np.abs(b * cos))):
        off = np.abs(got[..., part] - want) - (2.0 ** -22 * (1 + 2.0 ** -20) * A + rest)
        assert (off <= 0).all(), (int((off > 0).sum()), float(off.max()))
