"""What the calls on an 8-bit cache refuse, on the host: nothing is enqueued, so no GPU is needed and no address is touched."""
import ctypes as C

import numpy as np
import pytest

import kv8_model as m
from paper_2511_16665_amd import binding as tlt

P = 0x10000          # an address that nobody reads


def handle(**over):
    f = dict(k_pool=P, v_pool=P, k_exp=P, v_exp=P, n_pages=64, block_table=P, seq_len=P, max_pages=10, seq_len_bound=100)
    f.update(over)
    return C.byref(tlt.KV8C(*[f[k] for k, _ in tlt.KV8C._fields_]))


def write(kv=None, **over):
    a = dict(dtype=1, B=2, n=4, Hq=8, Hkv=2, d=128, page=16, theta=1e6, qkv=P, bias=P, depth=P, q=P, stride=8 * 128)
    a.update(over)
    return tlt.load().tlt_kv8_write(None, a["dtype"], a["B"], a["n"], a["Hq"], a["Hkv"], a["d"], a["page"], a["theta"], a["qkv"], a["bias"], a["depth"],
                                    kv or handle(), a["q"], a["stride"])


def attend(kv=None, **over):
    a = dict(dtype=1, B=2, n=4, Hq=8, Hkv=2, d=128, page=16, q=P, stride=8 * 128, mask=P, out=P, ws=P, bytes=1 << 30, impl=-1)
    a.update(over)
    return tlt.load().tlt_kv8_attention(None, a["dtype"], a["B"], a["n"], a["Hq"], a["Hkv"], a["d"], a["page"], a["q"], a["stride"], a["mask"], kv or handle(),
                                        a["out"], a["ws"], a["bytes"], a["impl"])


def commit(kv=None, **over):
    a = dict(B=2, L=3, Hkv=2, d=128, page=16, acc=P, path=P, stride=5)
    a.update(over)
    return tlt.load().tlt_kv8_commit(None, a["B"], a["L"], a["Hkv"], a["d"], a["page"], kv or handle(), a["acc"], a["path"], a["stride"])


def read(kv=None, **over):
    a = dict(dtype=1, L=3, B=2, n=4, Hkv=2, d=128, page=16, first=P, count=None, k=P, v=P)
    a.update(over)
    return tlt.load().tlt_kv8_read(None, a["dtype"], a["L"], a["B"], a["n"], a["Hkv"], a["d"], a["page"], kv or handle(), a["first"], a["count"], a["k"], a["v"])


BAD_KV = [dict(k_pool=None), dict(v_pool=None), dict(k_exp=None), dict(v_exp=None), dict(block_table=None), dict(seq_len=None), dict(n_pages=0),
          dict(max_pages=0), dict(seq_len_bound=-1), dict(k_pool=P + 8), dict(v_pool=P + 1)]


@pytest.mark.parametrize("call", [write, attend, commit, read])
def test_handles(call):
    for over in BAD_KV:
        assert call(handle(**over)) == -1, over
    for over in (dict(B=0), dict(B=65536), dict(Hkv=0), dict(d=32), dict(d=96), dict(d=320), dict(page=0)):
        assert call(**over) == -1, over
    full = handle(seq_len_bound=161)                      # 10 pages of 16
    assert call(full) == -3


def test_write():
    for over in (dict(dtype=2), dict(n=0), dict(Hq=7), dict(Hq=0), dict(theta=0.0), dict(theta=float("nan")), dict(qkv=None), dict(qkv=P + 2), dict(bias=P + 4),
                 dict(q=None), dict(q=P + 8), dict(stride=8 * 128 - 8), dict(stride=8 * 128 + 4), dict(stride=-1)):
        assert write(**over) == -1, over
    assert write(dtype=0, stride=8 * 128 + 2) == -1        # fp32 rows: 16 bytes are four elements
    assert write(n=61) == -3                              # 100 + 61 rows
    assert write(theta=float("inf")) == -1
    assert write(handle(max_pages=1 << 23), B=2, n=1 << 22) == -1   # more rows than a launch has workgroups


def test_attention():
    for over in (dict(dtype=-1), dict(n=0), dict(n=65), dict(Hq=9), dict(q=None), dict(q=P + 2), dict(stride=1000), dict(stride=8 * 128 + 1), dict(out=None),
                 dict(out=P + 4), dict(ws=None), dict(ws=P + 128), dict(impl=-2), dict(impl=9)):
        assert attend(**over) == -1, over
    assert attend(n=61) == -3
    size = tlt.load().tlt_kv8_attention_workspace_bytes
    assert size(2, 4, 8, 2, 128, 1000) > 0
    for bad in ((0, 4, 8, 2, 128, 1000), (2, 65, 8, 2, 128, 1000), (2, 4, 8, 3, 128, 1000), (2, 4, 8, 2, 100, 1000), (2, 4, 8, 2, 128, 0), (70000, 4, 8, 2, 128, 9)):
        assert size(*bad) == 0, bad


def test_commit_and_read():
    for over in (dict(L=0), dict(acc=None), dict(path=None), dict(stride=0)):
        assert commit(**over) == -1, over
    for over in (dict(dtype=5), dict(L=0), dict(n=0), dict(first=None), dict(k=None), dict(v=P + 8), dict(n=1 << 30), dict(L=1 << 24)):
        assert read(**over) == -1, over


def test_the_model_of_the_format():
    """Every code's value is found again, ties go to even codes, the exponent is the smallest that fits, and rows that are not finite are NaN."""
    vals = m.E4M3[np.r_[0:127, 128:255]]
    row = np.concatenate([vals, [448.0]])
    codes, e = m.encode(row)
    assert e == 127 and np.array_equal(m.decode(codes, e), row)
    mids = (m.POSITIVE[:-1] + m.POSITIVE[1:]) / 2
    codes, e = m.encode(np.concatenate([mids, [448.0]]))
    assert e == 127 and (codes[:-1] % 2 == 0).all()
    for scale, want in ((1.0, 127), (2.0, 128), (1.0000001, 128), (0.5, 126), (2.0 ** -120, 7), (2.0 ** -134, 1)):
        assert m.encode(np.array([448.0 * scale, 0.0]))[1] == want
    assert m.encode(np.zeros(4))[1] == 1
    c, e = m.encode(np.array([[1.0, np.inf], [np.nan, 2.0], [1.0, 2.0]]))
    assert e.tolist()[:2] == [255, 255] and not c[:2].any() and np.isnan(m.decode(c, e)[:2]).all()
    x = np.random.default_rng(3).standard_normal((50, 64)).astype(np.float32)
    for a, b in zip(m.encode(x), m._encode_fast(x)):
        np.testing.assert_array_equal(a, b)


def test_attention_past_what_a_launch_holds():
    size = tlt.load().tlt_kv8_attention_workspace_bytes
    long = dict(max_pages=1 << 23)
    assert attend(handle(seq_len_bound=(1 << 26) - 3, **long)) == -1 and size(2, 4, 8, 2, 128, (1 << 26) + 1) == 0   # n = 4
    assert size(2, 4, 8, 2, 128, 1 << 26) > 0
    # 65535 sequences of 8192 ranges each and 64 kv heads
    assert attend(handle(seq_len_bound=(1 << 25) - 4, **long), B=65535, Hq=64, Hkv=64, stride=64 * 128, bytes=1 << 62) == -2
    assert size(65535, 4, 64, 64, 128, 1 << 25) == 0


def test_a_workspace_serves_smaller_bounds_and_fewer_rows():
    size = tlt.load().tlt_kv8_attention_workspace_bytes
    for B in (1, 3, 33, 70, 96, 129, 192, 256, 257, 600):
        for Hq, Hkv in ((28, 4), (40, 8), (4, 1), (40, 20)):
            for n in (1, 2, 5, 8, 20, 64):
                by_length = [size(B, n, Hq, Hkv, 128, x) for x in (1, 64, 65, 128, 256, 257, 512, 513, 4095, 4096, 4097, 8192, 20000, 40000)]
                assert by_length == sorted(by_length), (B, n, Hq, Hkv)
            by_rows = [size(B, n, Hq, Hkv, 128, 5000) for n in range(1, 65)]
            assert by_rows == sorted(by_rows) and by_rows[0] > 0, (B, Hq, Hkv)
