"""The 8-bit cache's Python handle: its fields are checked against each other before any of them is taken."""
import pytest
import torch

from paper_2511_16665_amd import binding as tlt


class OnDevice(torch.Tensor):
    """A host tensor that says it is on a device: the handle's checks need no GPU."""
    is_cuda = property(lambda self: True)


def dev(*shape, dtype=torch.uint8):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


def cache(B=3, pages=8, max_pages=4):
    pool = lambda *s: dev(2, pages, 2, 16, *s)
    return tlt.KV8(pool(64), pool(64), pool(), pool(), dev(B, max_pages, dtype=torch.int32), dev(B, dtype=torch.int32), 50)


def test_a_field_that_does_not_fit_leaves_the_cache_as_it_was():
    kv = cache()
    for name, bad in (("block_table", dev(2, 4, dtype=torch.int32)), ("seq_len", dev(4, dtype=torch.int32)), ("k_pool", dev(2, 6, 2, 16, 64)), ("v_exp", dev(2, 8, 2, 8)),
                      ("seq_len", dev(3, dtype=torch.int64)), ("v_pool", dev(2, 8, 2, 16, 64, dtype=torch.int16)), ("k_exp", torch.zeros((2, 8, 2, 16), dtype=torch.uint8)),
                      ("block_table", dev(4, 3, dtype=torch.int32).t())):
        before, handle = dict(kv.__dict__), bytes(kv.c(1))
        with pytest.raises(AssertionError):
            setattr(kv, name, bad)
        assert getattr(kv, name) is before[name] and kv.__dict__.keys() == before.keys() and bytes(kv.c(1)) == handle, name
        assert all(kv.__dict__[k] is v for k, v in before.items()), name
    with pytest.raises(TypeError):
        kv.replace(bound=3)
    with pytest.raises(AssertionError):
        cache(B=3).replace(block_table=dev(2, 4, dtype=torch.int32), seq_len_bound=9)


def test_fields_that_fit_are_taken():
    kv = cache()
    table = dev(3, 9, dtype=torch.int32)
    kv.block_table, kv.seq_len_bound = table, 140
    c = kv.c()
    assert kv.block_table is table and (c.block_table, c.max_pages, c.seq_len_bound) == (table.data_ptr(), 9, 140)
    lens, table = dev(5, dtype=torch.int32), dev(5, 4, dtype=torch.int32)
    kv.replace(block_table=table, seq_len=lens, seq_len_bound=60)
    c = kv.c()
    assert kv.table_dims == (5, 4) and (c.block_table, c.seq_len, c.max_pages, c.seq_len_bound) == (table.data_ptr(), lens.data_ptr(), 4, 60)
    more = {x: dev(2, 20, 2, 16, 64) for x in ("k_pool", "v_pool")} | {x: dev(2, 20, 2, 16) for x in ("k_exp", "v_exp")}
    kv.replace(**more)
    c = kv.c(1)
    assert kv.dims == (2, 20, 2, 16, 64) and c.n_pages == 20 and c.k_pool == more["k_pool"].data_ptr() + 20 * 2 * 16 * 64 and c.v_exp == more["v_exp"].data_ptr() + 20 * 2 * 16
