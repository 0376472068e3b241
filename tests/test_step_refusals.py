"""What the page, rotary and sampling calls refuse, on the host: nothing is enqueued, so no GPU is needed and no address is touched."""
import ctypes as C

import pytest

from paper_2511_16665_amd import binding as tlt

P = 0x10000          # an address that nobody reads


def pages(**over):
    f = dict(free_page=P, n_free=P, page_count=P, block_table=P, n_pages=64, max_pages=10, page_size=16)
    f.update(over)
    return C.byref(tlt.PagesC(*[f[k] for k, _ in tlt.PagesC._fields_]))


def grow(pg=None, **over):
    a = dict(B=2, seq=P, new=P, depth=P, rows=8, out=P)
    a.update(over)
    return tlt.load().tlt_pages_grow(None, a["B"], pg or pages(), a["seq"], a["new"], a["depth"], a["rows"], *[a["out"]] * 5)


def release(pg=None, **over):
    a = dict(B=2, keep=P)
    a.update(over)
    return tlt.load().tlt_pages_release(None, a["B"], pg or pages(), a["keep"])


@pytest.mark.parametrize("call", [grow, release])
def test_pages(call):
    for over in (dict(free_page=None), dict(n_free=None), dict(page_count=None), dict(block_table=None), dict(n_pages=0), dict(n_pages=1 << 31), dict(max_pages=0), dict(page_size=0)):
        assert call(pages(**over)) == -1, over
    assert call(B=0) == -1 and call(B=-3) == -1
    assert call(B=4097) == -2


def test_grow():
    for over in (dict(seq=None), dict(new=None), dict(rows=-1)):
        assert grow(**over) == -1, over


def rope(**over):
    f = dict(freq=P, rot_dim=64, layout=0, amplitude=1.0)
    f.update(over)
    return C.byref(tlt.RopeC(*[f[k] for k, _ in tlt.RopeC._fields_]))


def kv(**over):
    f = dict(k_pool=P, v_pool=P, n_pages=64, block_table=None, seq_len=None, max_pages=0, seq_len_bound=0)
    f.update(over)
    return C.byref(tlt.KVC(*[f[k] for k, _ in tlt.KVC._fields_]))


def kv8(**over):
    f = dict(k_pool=P, v_pool=P, k_exp=P, v_exp=P, n_pages=64, block_table=None, seq_len=None, max_pages=0, seq_len_bound=0)
    f.update(over)
    return C.byref(tlt.KV8C(*[f[k] for k, _ in tlt.KV8C._fields_]))


def write(**over):
    a = dict(dtype=1, rows=4, Hq=8, Hkv=2, d=128, page=16, rope=rope(), qkv=P, step=12 * 128, bias=P, pos=P, slot=P, kv=kv(), kv8=None, q=P, q_step=8 * 128, kv_out=P, kv_step=4 * 128)
    a.update(over)
    return tlt.load().tlt_rope_write(None, a["dtype"], a["rows"], a["Hq"], a["Hkv"], a["d"], a["page"], a["rope"], a["qkv"], a["step"], a["bias"], a["pos"], a["slot"], a["kv"], a["kv8"],
                                     a["q"], a["q_step"], a["kv_out"], a["kv_step"])


def test_rope_write():
    for over in (dict(dtype=2), dict(rows=0), dict(rows=1 << 23), dict(Hq=7), dict(Hq=0), dict(Hkv=0), dict(d=0), dict(d=65), dict(d=258), dict(page=0), dict(rope=None), dict(qkv=None), dict(pos=None),
                 dict(step=12 * 128 - 1), dict(q_step=8 * 128 - 1), dict(kv_step=4 * 128 - 1), dict(qkv=P + 1), dict(bias=P + 1), dict(q=P + 1), dict(kv_out=P + 1), dict(slot=None), dict(slot=P + 4),
                 dict(kv8=kv8()), dict(kv=None, q=None, kv_out=None)):
        assert write(**over) == -1, over
    for over in (dict(freq=None), dict(freq=P + 4), dict(rot_dim=0), dict(rot_dim=-2), dict(rot_dim=63), dict(rot_dim=130), dict(layout=2), dict(layout=-1)):
        assert write(rope=rope(**over)) == -1, over
    for over in (dict(k_pool=None), dict(v_pool=None), dict(n_pages=0), dict(n_pages=1 << 31), dict(k_pool=P + 1)):
        assert write(kv=kv(**over)) == -1, over
    for over in (dict(k_pool=None), dict(v_pool=P + 8), dict(k_exp=None), dict(v_exp=None), dict(n_pages=0)):
        assert write(kv=None, kv8=kv8(**over)) == -1, over
    assert write(kv=None, kv8=kv8(), d=32, step=12 * 32, rope=rope(rot_dim=32)) == -1     # a head size that the 8-bit cache does not have
    assert write(rows=(1 << 23) - 1, Hq=64, Hkv=8, step=80 * 128) == -1                   # more rows and heads than a launch holds


def filt():
    return C.byref(tlt.FilterC(P, P, P, P))


def sample(**over):
    a = dict(dtype=0, rows=6, per=3, V=1000, logits=P, step=1000, f=filt(), u=P, token=P, lp=P, kept=P, ws=P, bytes=1 << 40)
    a.update(over)
    return tlt.load().tlt_sample(None, a["dtype"], a["rows"], a["per"], a["V"], a["logits"], a["step"], a["f"], a["u"], a["token"], a["lp"], a["kept"], a["ws"], a["bytes"])


def mask(**over):
    a = dict(dtype=0, rows=6, per=3, V=1000, logits=P, step=1000, f=filt(), out=2 * P, out_step=1000, kept=P, ws=P, bytes=1 << 40)
    a.update(over)
    return tlt.load().tlt_sample_filter(None, a["dtype"], a["rows"], a["per"], a["V"], a["logits"], a["step"], a["f"], a["out"], a["out_step"], a["kept"], a["ws"], a["bytes"])


@pytest.mark.parametrize("call", [sample, mask])
def test_sampling(call):
    for over in (dict(dtype=2), dict(rows=0), dict(rows=1 << 22, per=1), dict(per=0), dict(per=4), dict(V=0), dict(V=(1 << 20) + 1, step=1 << 25), dict(logits=None), dict(logits=P + 2), dict(step=999), dict(f=None),
                 dict(ws=None), dict(ws=P + 16)):
        assert call(**over) == -1, over
    assert call(bytes=16) == -2
    assert call(dtype=1, logits=P + 1) == -1


def test_sampling_outputs():
    assert sample(u=None) == sample(token=None) == -1
    assert mask(out=None) == mask(out_step=999) == mask(out=2 * P + 2) == -1
    assert mask(out=P, step=1004, out_step=1000) == -1                                   # in place, but with other rows
    size = tlt.load().tlt_sample_workspace_bytes
    assert size(0, 10) == size(10, 0) == size(1 << 22, 10) == size(1, (1 << 20) + 1) == 0
    assert size(1, 1) > 0 and size(1536, 152064) > 0 and size((1 << 22) - 1, 1 << 20) > 0


def test_a_greedy_engine_step_takes_no_filter():
    from paper_2511_16665_amd.engine import Engine
    with pytest.raises(ValueError):
        Engine.step(None, 4, 4, 8, asked=object())


def test_a_sampling_workspace_for_the_largest_call_serves_smaller_ones():
    size = tlt.load().tlt_sample_workspace_bytes
    for V in (4096, 4097, 8192, 9001, 50000, 152064, 1 << 20):
        sizes = [size(r, V) for r in [*range(1, 1500), 2047, 2048, 2049, 5000, (1 << 22) - 1]]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))
    for r in (1, 33, 363, 1024, 5000):
        sizes = [size(r, V) for V in (1, 4096, 4097, 8191, 8192, 16383, 16384, 40000, 152064, 1 << 20)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))
