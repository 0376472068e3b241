"""Decoding steps of a caller with a forward of its own, from the page, rotary, attention and sampling calls together, against dense attention in float64 and the sampling model."""
import numpy as np
import pytest
import torch

import pick_model as pm
from paper_2511_16665_amd import binding as tlt

pytestmark = pytest.mark.gpu

HQ, HKV, D, V, PAGE = 4, 2, 64, 500, 16


@pytest.mark.parametrize("eight_bits", [False, True])
def test_steps_of_a_small_decoder(eight_bits):
    """One attention layer: rows = embedding[token] (queries, keys, values), logits = attention output . W.  Sequences join with prompts of different lengths, decode, and one leaves; a cache that
    the calls themselves page.  Every step's slots are the table's, its attention is the dense one over all tokens so far, its tokens are the model's draws from the logits it gave."""
    rng = np.random.default_rng(0)
    B, W = 3, (HQ + 2 * HKV) * D
    emb = torch.from_numpy(rng.normal(0, 1, (V, W)).astype(np.float32)).cuda()
    head = torch.from_numpy(rng.normal(0, 0.6, (HQ * D, V)).astype(np.float32)).cuda()
    pages = tlt.Pages.empty(B, 40, 12, PAGE)
    seq_len = torch.zeros((B,), dtype=torch.int32, device="cuda")
    freq, amp = tlt.rope_freqs("ramp", D, 1e4, factor=4.0, original_len=2048.0)
    rope = tlt.Rope(torch.from_numpy(freq).cuda(), True, amp)
    if eight_bits:
        kv = tlt.KV8.empty(1, 40, HKV, PAGE, D, pages.block_table, seq_len, 150)
    else:
        pool = lambda: torch.zeros((1, 40, HKV, PAGE, D), device="cuda")
        kv = tlt.KV(pool(), pool(), pages.block_table, seq_len, 150)
    ask = tlt.SampleFilter(torch.tensor([0.8, 1.0, 0.0]).cuda(), torch.tensor([40, 0, 0], dtype=torch.int32).cuda(), torch.tensor([0.9, 0.95, 1.0]).cuda(), None)
    asked = [dict(tau=0.8, top_k=40, top_p=0.9), dict(top_p=0.95), dict(tau=0.0)]
    ws = tlt.sample_workspace(B, V)
    history = [[] for _ in range(B)]
    i32 = lambda n: torch.zeros((n,), dtype=torch.int32, device="cuda")

    def write(tokens, rows):
        """New tokens of every sequence, in a buffer of `rows` rows (the last ones unused)."""
        n_new = torch.tensor([len(t) for t in tokens], dtype=torch.int32).cuda()
        position, slot, granted, q = i32(rows), torch.empty((rows,), dtype=torch.int64, device="cuda"), i32(B), torch.empty((rows, HQ * D), device="cuda")
        tlt.pages_grow(pages, seq_len, n_new, None, None, None, position, slot, granted)
        flat = torch.tensor(sum(tokens, []) + [0] * (rows - sum(map(len, tokens)))).cuda()
        tlt.rope_write(tlt.TLT_F32, HQ, HKV, D, rope, emb[flat], None, position, slot, kv, 0, q)
        assert granted.tolist() == [1] * B
        for b, t in enumerate(tokens):
            history[b] += t
        return q

    def dense(b):
        """Attention of sequence b's last token over all of them, float64; keys and values as a cache in 8 bits holds them would be off by 2^-4 of each row's largest."""
        t = np.array(history[b])
        x = emb.double().cpu().numpy()[t].reshape(len(t), -1, D)
        angle = np.arange(len(t))[:, None] * freq
        c, s = np.cos(angle)[:, None] * amp, np.sin(angle)[:, None] * amp
        y = x.copy()
        y[:, :HQ + HKV, 0::2], y[:, :HQ + HKV, 1::2] = x[:, :HQ + HKV, 0::2] * c - x[:, :HQ + HKV, 1::2] * s, x[:, :HQ + HKV, 0::2] * s + x[:, :HQ + HKV, 1::2] * c
        if eight_bits:
            import kv8_model
            for h in range(HQ, HQ + 2 * HKV):
                y[:, h] = kv8_model.decode(*kv8_model.encode(y[:, h].astype(np.float32)))
        out = np.zeros((HQ, D))
        for h in range(HQ):
            k, v = y[:, HQ + h // (HQ // HKV)], y[:, HQ + HKV + h // (HQ // HKV)]
            w = np.exp((k @ y[-1, h]) / 8 - ((k @ y[-1, h]) / 8).max())
            out[h] = w @ v / w.sum()
        return out.ravel()

    prompts = [rng.integers(0, V, n).tolist() for n in (17, 1, 60)]
    write(prompts, 80)                                      # (the prompt's rows; its last token is decoded with the next step)
    seq_len.copy_(torch.tensor([len(p) for p in prompts], dtype=torch.int32).cuda())
    token = torch.from_numpy(rng.integers(0, V, B).astype(np.int32)).cuda()
    for step in range(20):
        q = write([[int(t)] for t in token], B + 2)[:B]
        out = torch.empty((B, 1, HQ * D), device="cuda")
        mask = torch.ones((B, 1), dtype=torch.int64, device="cuda")
        if eight_bits:
            aws = tlt.kv8_attention_workspace(B, 1, HQ, HKV, D, 151)
            tlt.kv8_attention(tlt.TLT_F32, HQ, q.view(B, 1, -1), mask, kv, 0, out, aws)
        else:
            aws = tlt.attention_workspace(B, 1, HQ, HKV, D, 151)
            qkv = torch.zeros((B, 1, W), device="cuda")
            qkv[:, 0, :HQ * D] = q
            assert tlt.attention(tlt.TLT_F32, HQ, PAGE, qkv, mask, kv, out, aws) == 0
        logits = out[:, 0] @ head
        u = rng.integers(0, 2 ** 32, B)
        logprob, kept = torch.empty((B, 2), device="cuda"), i32(B)
        tlt.sample(tlt.TLT_F32, logits, ask, torch.from_numpy(u.astype(np.uint32).view(np.int32)).cuda(), token, logprob, kept, ws)
        for b in range(B):
            want = dense(b)
            # fp32 sums of up to 80 terms around scores of a few units: 2^-16 of the largest value; codes that a last bit moved to their neighbour: 2^-3 of one row in many
            assert np.abs(out[b, 0].double().cpu().numpy() - want).max() <= (2.0 ** -16 if not eight_bits else 2.0 ** -6) * 4
            t, lp, n = pm.draw(logits[b].double().cpu().numpy(), int(u[b]), **asked[b])
            assert (int(token[b]), int(kept[b])) == (t, n)
        seq_len += 1
        tlt.pages_release(pages, seq_len)
        if step == 10:                                      # one rollout ends, another one takes its place
            seq_len[0] = 0
            tlt.pages_release(pages, seq_len)
            assert int(pages.page_count[0]) == 0
            history[0] = []
            new = rng.integers(0, V, 33).tolist()
            write([new, [], []], 40)
            seq_len[0] = 33
    assert int(pages.n_free) == 40 - sum(-(-int(n) // PAGE) for n in seq_len.tolist())
    tlt.pages_release(pages, None)
    assert sorted(pages.free_page.tolist()) == list(range(40)) and int(pages.n_free) == 40
