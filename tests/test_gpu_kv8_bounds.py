"""The 8-bit cache's calls inside larger buffers: what lies before and behind is left alone, also with lengths above the declared bound."""
import numpy as np
import pytest
import torch

import kv8_model as m
from paper_2511_16665_amd import binding as tlt
from test_gpu_kv8 import check_attention, cuda
from test_gpu_kv8 import test_commit as commit_case

pytestmark = pytest.mark.gpu
GUARD = 4096


@pytest.mark.parametrize("impl", [-1, 0])
@pytest.mark.parametrize("Hq,Hkv,n", [(28, 4, 1), (28, 4, 4), (28, 4, 8), (28, 4, 20), (28, 4, 64), (64, 2, 64)])
def test_attention_stays_inside(Hq, Hkv, n, impl):
    """Exactly the workspace that is asked for; a sequence longer than the bound, whose outputs mean nothing, writes neither past it nor into another's output."""
    d, bound = 128, 600
    c = m.Cache([bound, 700, 40], n, Hkv, d, 16, seed=2)
    q = torch.from_numpy(np.random.default_rng(1).standard_normal((3, n, Hq, d)).astype(np.float32)).bfloat16()
    need = tlt.load().tlt_kv8_attention_workspace_bytes(3, n, Hq, Hkv, d, bound + n)
    c.kv.seq_len_bound = bound
    before = {x: getattr(c.kv, x).clone() for x in ("k_pool", "v_pool", "k_exp", "v_exp", "block_table")}
    x = q.view(3, n, Hq * d).cuda()
    for length in (bound, 700, 2 ** 31 - 1):
        c.kv.seq_len[1] = length
        c.ctx[1] = bound
        store = torch.full((need + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
        outs = torch.full((3 * n * Hq * d + 2 * GUARD,), 7.0, dtype=torch.bfloat16, device="cuda")
        out = outs[GUARD:-GUARD].view(3, n, Hq * d)
        print("attention inside larger buffers", Hq, Hkv, n, impl, length, flush=True)
        tlt.kv8_attention(tlt.TLT_BF16, Hq, x, None, c.kv, 0, out, store[GUARD:GUARD + need], impl)
        torch.cuda.synchronize()
        assert (store[:GUARD] == 0xA5).all() and (store[-GUARD:] == 0xA5).all()
        assert (outs[:GUARD] == 7.0).all() and (outs[-GUARD:] == 7.0).all()
        assert all(torch.equal(getattr(c.kv, k), t) for k, t in before.items())
        check_attention(c, "bf16", q.float().numpy(), None, out.view(3, n, Hq, d), rows=[0, 1, 2] if length == bound else [0, 2])


def test_write_and_read_stay_inside():
    """Rows of queries and rows read back, one layer of three: the layers beside it, and what surrounds the outputs, keep their bytes."""
    Hq, Hkv, d, n, L = 12, 4, 128, 7, 3
    c = m.Cache([33, 5], n, Hkv, d, 16, layers=L, seed=2)
    store = torch.full((2 * n * Hq * d + 2 * GUARD,), 7.0, dtype=torch.bfloat16, device="cuda")
    qkv = torch.randn((2, n, (Hq + 2 * Hkv) * d), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    before = {x: getattr(c.kv, x).clone() for x in ("k_pool", "v_pool", "k_exp", "v_exp")}
    print("write and read inside larger buffers", flush=True)
    tlt.kv8_write(tlt.TLT_BF16, Hq, 1e6, qkv, None, None, c.kv, 1, store[GUARD:-GUARD].view(2, n, Hq * d))
    assert (store[:GUARD] == 7.0).all() and (store[-GUARD:] == 7.0).all()
    assert all(torch.equal(getattr(c.kv, x)[l], t[l]) for x, t in before.items() for l in (0, 2))
    size = L * 2 * n * Hkv * d
    rows = [torch.full((size + 2 * GUARD,), 7.0, dtype=torch.float32, device="cuda") for _ in range(2)]
    tlt.kv8_read(tlt.TLT_F32, c.kv, cuda(np.array([33, 5], np.int32)), cuda(np.array([n, 0], np.int32)), *(r[GUARD:-GUARD].view(L, 2, n, Hkv, d) for r in rows))
    for r in rows:
        assert (r[:GUARD] == 7.0).all() and (r[-GUARD:] == 7.0).all() and (r[GUARD:-GUARD].view(L, 2, n, Hkv, d)[:, 1] == 7.0).all()


@pytest.mark.parametrize("Hkv,d,page,L,n", [(4, 128, 16, 20, 24), (4, 128, 16, 28, 12), (8, 64, 16, 26, 9), (4, 128, 16, 29, 64), (8, 128, 16, 28, 12), (5, 192, 5, 32, 20)])
def test_commit_on_both_sides_of_the_rule(Hkv, d, page, L, n):
    """1440, 2016, 2080, 2088, 4032 and 4160 columns: two turns of a thread in one launch, and two launches."""
    print(L * Hkv * (d // 8 + 2), "columns", flush=True)
    commit_case(Hkv, d, page, L, n)
