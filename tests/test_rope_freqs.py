"""Frequencies of rotary positions: the scalings against their definitions, and what they do at their ends."""
import math

import numpy as np
import pytest

from paper_2511_16665_amd import binding as tlt


def plain(r, theta):
    return np.array([theta ** (-2.0 * j / r) for j in range(r // 2)])


@pytest.mark.parametrize("r,theta", [(2, 1e4), (64, 1e4), (128, 1e6), (96, 500000.0)])
def test_plain_and_linear(r, theta):
    f, amp = tlt.rope_freqs("plain", r, theta)
    np.testing.assert_allclose(f, plain(r, theta), rtol=1e-14)
    assert amp == 1.0 and f[0] == 1.0
    g, amp = tlt.rope_freqs("linear", r, theta, factor=8.0)
    np.testing.assert_allclose(g, f / 8.0, rtol=1e-15)
    assert amp == 1.0


def test_base():
    r, theta, s = 128, 1e4, 4.0
    f, amp = tlt.rope_freqs("base", r, theta, factor=s)
    g = plain(r, theta)
    assert amp == 1.0 and f[0] == 1.0
    np.testing.assert_allclose(f[-1], g[-1] / s, rtol=1e-12)      # the slowest pair as if interpolated
    assert (f[1:] < g[1:]).all() and (np.diff(f) < 0).all()


@pytest.mark.parametrize("scaling", ["ramp", "bands"])
def test_by_parts(scaling):
    r, theta, s, L, low, high = 128, 1e6, 4.0, 32768.0, 1.0, 32.0
    f, amp = tlt.rope_freqs(scaling, r, theta, factor=s, original_len=L, low=low, high=high)
    g, turns = plain(r, theta), L * plain(r, theta) / (2 * math.pi)
    if scaling == "ramp":
        pair = lambda n: r * math.log(L / (2 * math.pi * n)) / (2 * math.log(theta))
        a, b = math.floor(pair(high)), math.ceil(pair(low))
        slow = np.clip((np.arange(r // 2) - a) / (b - a), 0, 1)
        assert amp == np.float32(0.1 * math.log(s) + 1)
    else:
        slow = np.clip(1 - (turns - low) / (high - low), 0, 1)
        assert amp == 1.0
    np.testing.assert_allclose(f, g * (1 - slow) + g / s * slow, rtol=1e-13)
    assert f[0] == 1.0 and abs(f[-1] * s / g[-1] - 1) < 1e-13     # fast pairs as they were, slow ones interpolated
    one, amp = tlt.rope_freqs(scaling, r, theta, factor=1.0, original_len=L, low=low, high=high)
    np.testing.assert_allclose(one, g, rtol=1e-14)
    assert amp == 1.0


def test_a_ramp_without_width():
    f, _ = tlt.rope_freqs("ramp", 4, 1e4, factor=2.0, original_len=7.0, low=1.0, high=1.0000001)
    assert np.isfinite(f).all() and (f > 0).all()


def test_refusals():
    ok = dict(rot_dim=64, theta=1e4, factor=2.0, original_len=4096.0, low=1.0, high=32.0)
    for scaling in tlt.ROPE_SCALING:
        tlt.rope_freqs(scaling, **ok)
        for over in (dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=1 << 17), dict(theta=1.0), dict(theta=math.nan), dict(theta=math.inf)):
            with pytest.raises(tlt.TltError):
                tlt.rope_freqs(scaling, **{**ok, **over})
        if scaling != "plain":
            for factor in (0.5, 0.0, math.nan, math.inf):
                with pytest.raises(tlt.TltError):
                    tlt.rope_freqs(scaling, **{**ok, "factor": factor})
    f, amp = tlt.rope_freqs("plain", 64, 1e4, factor=0.0)          # unused there
    np.testing.assert_allclose(f, plain(64, 1e4), rtol=1e-14)
    with pytest.raises(tlt.TltError):
        tlt.rope_freqs("base", 2, 1e4, factor=2.0)
    for scaling in ("ramp", "bands"):
        for over in (dict(original_len=0.0), dict(original_len=math.nan), dict(low=0.0), dict(low=32.0), dict(high=math.inf)):
            with pytest.raises(tlt.TltError):
                tlt.rope_freqs(scaling, **{**ok, **over})
    assert tlt.load().tlt_rope_freqs(7, 64, 1e4, 1.0, 0.0, 0.0, 0.0, np.empty(32).ctypes.data, None) == -1
    assert tlt.load().tlt_rope_freqs(0, 64, 1e4, 1.0, 0.0, 0.0, 0.0, None, None) == -1
