"""Engine steps whose target distribution is reduced by top-k, top-p and min-p."""
import numpy as np
import pytest
import torch

import pick_model as pm
from gpu_util import make_engine, make_models
from oracle import accept as oacc
from oracle import sample_draft as osd
from paper_2511_16665_amd import binding as tlt
from synth import TINY, prompts

pytestmark = pytest.mark.gpu
B, K, D, N, P = 4, 3, 4, 12, 24


def u32(rng, *shape):
    return rng.integers(0, 2 ** 32, size=shape, dtype=np.uint64).astype(np.uint32)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int32)).cuda()


def engine(seed):
    tw_dev, dw_dev, _, _ = make_models(TINY, 7, "fp32", std=0.08)
    e, _, _ = make_engine(TINY, "fp32", tw_dev, dw_dev, B, max(N, P), D, K, P + 6 * (D + 1) + N + 32, seed=seed)
    pr = np.stack(prompts(B, P, TINY.vocab, seed=4)).astype(np.int32)
    e.prefill(pr)
    return e, pr


@pytest.mark.parametrize("target_only", [False, True])
def test_steps_follow_the_oracle_s_rule_on_reduced_logits(target_only):
    """Every step's logits are the forward's with what is not kept at -infinity, and its acceptance is the oracle's rule on them; every emitted token is one that its node keeps."""
    tau = 0.3 if target_only else 0.9
    e, pr = engine(2)
    asked = [dict(tau=tau, top_k=5), dict(tau=tau, top_p=0.6), dict(tau=tau, min_p=0.3), dict(tau=tau, top_k=40, top_p=0.8, min_p=0.05)]
    col = lambda name, default, dt: torch.tensor([a.get(name, default) for a in asked], dtype=dt).cuda()
    filt = tlt.SampleFilter(col("tau", 1, torch.float32), col("top_k", 0, torch.int32), col("top_p", 1, torch.float32), col("min_p", 0, torch.float32))
    n = N if target_only else len(osd.static_template(K, D, N)[0])
    rng, lens = np.random.default_rng(9), np.full(B, P - 1)
    for step in range(5):
        u_a, u_f = u32(rng, B, n), u32(rng, B)
        if target_only:
            al, out = e.step(K, D, N, sample=(tau, dev(u_a), dev(u_f)), asked=filt)
        else:
            al, out = e.step_sampled(K, D, N, tau, dev(u32(rng, B, n)), dev(u_a), dev(u_f), asked=filt)
        tree, logits = e.tree(n), e.logits(n).cpu().numpy()
        tok, par = tree.token.cpu().numpy(), tree.parent.cpu().numpy()
        if target_only:
            want = oacc.accept_target_only(tok, par, logits, u_a, u_f, tau, e.stride)
        else:
            want = oacc.accept_sample(tok, par, logits, e.draft_q(n).cpu().numpy(), u_a, u_f, tau, e.stride)
        np.testing.assert_array_equal(al, want[0])
        np.testing.assert_array_equal(out, want[2])
        path = e.path_idx.cpu().numpy()
        for b in range(B):
            for j in range(al[b] + 1):
                assert np.isfinite(logits[b, path[b, j], out[b, j]]), (step, b, j)
            for i in range(n):
                # as many tokens as the sequence's own settings can keep; min-p keeps all of what it kept once
                row, k = logits[b, i].astype(np.float64), int(np.isfinite(logits[b, i]).sum())
                a = asked[b]
                assert 1 <= k <= (a["top_k"] if "top_k" in a else TINY.vocab - 1)
                if "min_p" in a:
                    assert len(pm.choose(row, tau=a["tau"], min_p=a["min_p"])[0]) == k
        lens = lens + al + 1
        np.testing.assert_array_equal(e.kv.seq_len.cpu().numpy(), lens)
    e.ctx.close()


def test_one_token_kept_is_greedy_decoding():
    """top_k = 1 leaves one token per node: sampled steps emit the greedy rollout whatever the uniforms."""
    rng, n = np.random.default_rng(1), len(osd.static_template(K, D, N)[0])
    one = tlt.SampleFilter(torch.full((B,), 0.9).cuda(), torch.ones((B,), dtype=torch.int32).cuda())
    e, _ = engine(3)
    greedy = [[] for _ in range(B)]
    for _ in range(6):
        al, out = e.step(K, D, N)
        for b in range(B):
            greedy[b] += out[b, :al[b] + 1].tolist()
    e.ctx.close()
    e, _ = engine(3)
    got = [[] for _ in range(B)]
    for _ in range(6):
        al, out = e.step_sampled(K, D, N, 0.9, dev(u32(rng, B, n)), dev(u32(rng, B, n)), dev(u32(rng, B)), asked=one)
        for b in range(B):
            got[b] += out[b, :al[b] + 1].tolist()
    e.ctx.close()
    for b in range(B):
        m = min(len(greedy[b]), len(got[b]))
        assert m >= 6 and greedy[b][:m] == got[b][:m]


@pytest.mark.parametrize("target_only", [False, True])
def test_a_filter_without_a_temperature_takes_the_step_s(target_only):
    """The same steps as with that temperature given for every sequence, and not those of temperature 1; one that is given as 0 leaves its sequence greedy."""
    tau, n = 0.4, N if target_only else len(osd.static_template(K, D, N)[0])
    top_p = torch.full((B,), 0.7).cuda()
    given = [None, torch.full((B,), tau).cuda(), torch.ones((B,)).cuda(), torch.tensor([0.0] + [tau] * (B - 1)).cuda()]
    runs = []
    for temperature in given:
        filt, rng, kept = tlt.SampleFilter(temperature, None, top_p), np.random.default_rng(6), []
        e, _ = engine(5)
        for _ in range(4):
            draws = [dev(u32(rng, B, n)) for _ in range(2)] + [dev(u32(rng, B))]
            al, out = e.step(K, D, N, sample=(tau, *draws[1:]), asked=filt) if target_only else e.step_sampled(K, D, N, tau, *draws, asked=filt)
            kept.append((al.copy(), out.copy(), e.logits(n).cpu().numpy()))
        assert filt.temperature is temperature
        e.ctx.close()
        runs.append(kept)
    for a, b in zip(runs[0], runs[1]):
        for x, y in zip(a, b):
            np.testing.assert_array_equal(x, y)
    counts = [np.isfinite(r[0][2]).sum(-1) for r in runs]         # of the first step, whose tree is the same
    assert (counts[0] <= counts[2]).all() and (counts[0] < counts[2]).any()
    assert (counts[3][0] == 1).all() and (counts[3][1:] == counts[0][1:]).all()
