"""The operators around attention in a decoding step of a caller with a forward of its own, as measured cases, with their plain forms.

kind "sample"   one token per row of logits, drawn at a temperature from what top-k, top-p and min-p leave, with its log-probabilities
kind "filter"   the same choice for the rows of token trees: logits with all other tokens at -infinity, for an acceptance rule
kind "rope"     rotary positions for new rows of a layer (half and interleaved layouts, part of the head, scaled frequencies), keys and values
                written to the slots of a paged cache in the model's type or in 8 bits
kind "pages"    pages for the rows that a step adds to every sequence, their slots, and afterwards the pages given back

A token's weight is the whole number floor(exp(l / tau - max / tau) * 2^32), the one that the acceptance rules draw with, so all sums are exact and the
drawn tokens are the same however they are added up.  Tokens are ordered by falling logit, then rising index.  Kept are the first top_k of them; of
these the ones before which less than top_p of the kept weight lies; of these the ones of at least min_p times the largest weight.  The token
drawn is the first, by index, whose running sum of kept weights exceeds (u * sum) >> 32.  A temperature that is not positive keeps the first
token alone (weights as at temperature 1).

Head shapes are those of synth/inputs.py: "tiny" 4 / 2 of 64 in fp32, "7b" 28 / 4, "32b" 40 / 8 and "70b" 64 / 8 of 128 in bf16.
"""
import math
import statistics

import numpy as np
import torch

own = False

HEADS = {"tiny": (4, 2, 64), "7b": (28, 4, 128), "32b": (40, 8, 128), "70b": (64, 8, 128)}   # query heads, kv heads, head_dim
PAGE, THETA, LONG = 16, 1e6, 32768


def listed():
    return [
        # the smallest calls: a tiny decoder's vocabulary, two sequences
        dict(name="sample 2 x 1024", kind="sample", batch=2, nodes=1, vocab=1024, dtype="fp32", mode="p", masked=False),
        # the last sequence of a rollout, decoded without drafts
        dict(name="sample 1 x 152064", kind="sample", batch=1, nodes=1, vocab=152064, dtype="fp32", mode="kp", masked=False),
        # a serving batch whose requests ask for different things, logits in bf16, some behind a grammar's mask
        dict(name="sample 64 x 128256 bf16", kind="sample", batch=64, nodes=1, vocab=128256, dtype="bf16", mode="mixed", masked=True),
        # a rollout's first phase: many sequences, nucleus sampling
        dict(name="sample 256 x 152064", kind="sample", batch=256, nodes=1, vocab=152064, dtype="fp32", mode="p", masked=False),
        # the tail of a rollout with the largest trees, and the benchmark's trees
        dict(name="filter 4 x 64", kind="filter", batch=4, nodes=64, vocab=152064, dtype="fp32", mode="kp", masked=False),
        dict(name="filter 32 x 48", kind="filter", batch=32, nodes=48, vocab=152064, dtype="fp32", mode="mixed", masked=False),
        # one new row of one sequence, far out; a batch decoded with a rotated quarter of the head; a verification's rows into the 8-bit cache
        dict(name="rope 1 x 1", kind="rope", heads="7b", batch=1, nodes=1, ctx=31000, spread=0.0, rot=128, pairs="half", scaled="no", cache="model", bias=True, pad=0),
        dict(name="rope 96 x 1 quarter", kind="rope", heads="32b", batch=96, nodes=1, ctx=4096, spread=0.8, rot=32, pairs="interleaved", scaled="no", cache="model", bias=False, pad=0),
        dict(name="rope 32 x 48 into 8 bits", kind="rope", heads="7b", batch=32, nodes=48, ctx=4096, spread=0.8, rot=128, pairs="half", scaled="parts", cache="8 bits", bias=True, pad=0),
        # prompts of a group of rollouts in one pass, the last rows of the buffer unused
        dict(name="rope 5 x 1638", kind="rope", heads="70b", batch=5, nodes=1638, ctx=20000, spread=0.3, rot=128, pairs="half", scaled="parts", cache="model", bias=False, pad=17),
        # a verification step of a batch, and prompts of all lengths admitted beside running sequences when there are hardly pages enough
        dict(name="pages 32 x 48", kind="pages", batch=32, nodes=48, ctx=4096, spread=0.8, admit=False, short=False),
        dict(name="pages 256 x ~2000", kind="pages", batch=256, nodes=2000, ctx=6000, spread=0.6, admit=True, short=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["sample", "sample", "sample", "filter", "rope", "rope", "rope", "pages"])
    if kind in ("sample", "filter"):
        vocab = rng.choice([1024, 4096, 128256, 152064, _log(rng, 5, 160000), _log(rng, 20000, 160000) | 1])
        batch = _log(rng, 1, 256 if kind == "sample" else 64)
        nodes = 1 if kind == "sample" else _log(rng, 2, min(64, 1536 // batch))
        return dict(kind=kind, batch=batch, nodes=nodes, vocab=vocab, dtype=rng.choice(["fp32", "fp32", "bf16"]), mode=rng.choice(["none", "k", "p", "min", "kp", "mixed", "mixed"]),
                    masked=rng.random() < 0.3)
    spread = rng.choice([0.0, 0.3, 0.8])
    if kind == "rope":
        heads = rng.choice(["7b", "7b", "32b", "70b", "tiny"])
        d = HEADS[heads][2]
        batch = _log(rng, 1, 128)
        nodes = rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 2, max(2, 8000 // batch))])
        return dict(kind=kind, heads=heads, batch=batch, nodes=nodes, ctx=_log(rng, 20, min(30000, 400000 // batch)), spread=spread, rot=rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)]),
                    pairs=rng.choice(["half", "interleaved"]), scaled=rng.choice(["no", "linear", "parts"]), cache=rng.choice(["model", "model", "8 bits"]), bias=rng.random() < 0.5, pad=rng.choice([0, 0, rng.randint(1, 9)]))
    batch = _log(rng, 1, 512)
    return dict(kind=kind, batch=batch, nodes=_log(rng, 1, max(1, min(4000, 500000 // batch))), ctx=_log(rng, 1, min(30000, 1500000 // batch)), spread=spread, admit=rng.random() < 0.4, short=rng.random() < 0.4)


# ---- inputs

def _cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _lengths(case):
    """Committed tokens of a batch: ctx, or the quantiles of lognormal lengths whose mean it is (whose sequence is which goes by the seed)."""
    at = np.array([statistics.NormalDist().inv_cdf((i + 0.5) / case["batch"]) for i in range(case["batch"])])
    ctx = case["ctx"] * np.exp((at - case["spread"] / 2) * case["spread"])
    return np.clip(np.rint(ctx), 1, max(4 * case["ctx"] if case["ctx"] < 8192 else 32768, 1)).astype(np.int32)


def _settings(mode, B, rng):
    """What a batch's requests ask for: temperature, top_k (0: off), top_p, min_p of every sequence; None where no request asks."""
    tau = rng.uniform(0.6, 1.1, B).astype(np.float32)
    k, p, m = rng.integers(20, 200, B).astype(np.int32), rng.uniform(0.8, 0.98, B).astype(np.float32), rng.uniform(0.01, 0.1, B).astype(np.float32)
    if mode == "mixed":      # every sequence for itself: some greedy, some unfiltered, some with very wide or narrow settings
        tau[rng.random(B) < 0.1] = 0.0
        k[rng.random(B) < 0.5] = 0
        k[rng.random(B) < 0.1] = 5000
        p[rng.random(B) < 0.4] = 1.0
        p[rng.random(B) < 0.05] = 0.01
        m[rng.random(B) < 0.6] = 0.0
    use = {"none": "", "k": "k", "p": "p", "min": "m", "kp": "kp", "mixed": "kpm"}[mode]
    return tuple(_cuda(v) if on else None for v, on in ((tau, True), (k, "k" in use), (p, "p" in use), (m, "m" in use)))


def _prepare_logits(case, seed):
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, n, V = case["batch"], case["nodes"], case["vocab"]
    # as a trained model's: a wide bell of unlikely tokens, and in seven rows of eight a few dozen that stand out by up to ten
    x = torch.randn((B * n, V), generator=g, device="cuda") * 2.0
    stand = min(48, V)
    at = torch.randint(0, V, (B * n, stand), generator=g, device="cuda")
    up = 14.0 - 10.0 * torch.rand((B * n, stand), generator=g, device="cuda")
    up[torch.rand((B * n,), generator=g, device="cuda") < 0.125] = 0.0
    x.scatter_add_(1, at, up)
    if case["masked"]:       # a grammar leaves one token in fifty, in every third row; now and then none
        third = torch.arange(B * n, device="cuda") % 3 == 1
        x.masked_fill_(third[:, None] & (torch.rand((B * n, V), generator=g, device="cuda") > 0.02), -math.inf)
    x = x.to(torch.float32 if case["dtype"] == "fp32" else torch.bfloat16).view(B, n, V)
    s = dict(kind=case["kind"], B=B, n=n, V=V, logits=x, filter=_settings(case["mode"], B, rng))
    s["u"] = torch.randint(-2 ** 31, 2 ** 31, (B, n), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)   # 32 random bits
    s["token"], s["kept"] = (torch.empty((B, n), dtype=torch.int32, device="cuda") for _ in range(2))
    s["logprob"] = torch.empty((B, n, 2), dtype=torch.float32, device="cuda")
    s["out"] = torch.empty_like(x) if case["kind"] == "filter" else None
    return s


def _frequencies(r, scaled):
    """(radians per position of the r / 2 pairs, amplitude): theta^(-2j/r); "linear" positions divided by 4; "parts" for contexts four times as long as the original:
    slow pairs as "linear", fast ones as they were, a ramp over the pairs in between."""
    f = THETA ** (-np.arange(0, r, 2, dtype=np.float64) / r)
    if scaled == "linear":
        return f / 4, 1.0
    if scaled == "parts":
        at = lambda turns: r * math.log(LONG / (2 * math.pi * turns)) / (2 * math.log(THETA))
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), r - 1)
        slow = np.clip((np.arange(r // 2) - lo) / max(hi - lo, 1e-3), 0, 1)
        return f * (1 - slow) + f / 4 * slow, 0.1 * math.log(4.0) + 1.0
    return f, 1.0


def _prepare_rope(case, seed):
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    Hq, Hkv, d = HEADS[case["heads"]]
    B, n = case["batch"], case["nodes"]
    R = B * n + case["pad"]
    ctx = rng.permutation(_lengths(case))
    # the pages that the new rows reach into; the older ones are not touched here
    first, behind = ctx // PAGE, (ctx + n + PAGE - 1) // PAGE
    pages = B * ((n + 2 * PAGE - 2) // PAGE) + 3
    order, o = rng.permutation(pages).astype(np.int32), 0
    table = np.full((B, int(behind.max())), -1, np.int32)
    for b in range(B):
        table[b, first[b]:behind[b]] = order[o:o + behind[b] - first[b]]
        o += behind[b] - first[b]
    # rows of chains (one row, prompts) or small trees: positions lag behind slots
    depth = np.arange(n)[None].repeat(B, 0) if n > 64 else np.minimum(np.arange(n)[None], 1 + rng.integers(0, n + 1, (B, n)) // 2)
    slot_of = ctx[:, None].astype(np.int64) + np.arange(n)
    slot = np.take_along_axis(table, slot_of // PAGE, 1).astype(np.int64) * PAGE + slot_of % PAGE
    pad = lambda a, v: np.concatenate([a.reshape(-1), np.full(case["pad"], v, a.dtype)])
    dtype = torch.float32 if case["heads"] == "tiny" else torch.bfloat16
    freq, amplitude = _frequencies(case["rot"], case["scaled"])
    s = dict(kind="rope", Hq=Hq, Hkv=Hkv, d=d, B=B, n=n, R=R, dtype=dtype, rot=case["rot"], interleaved=case["pairs"] == "interleaved", freq=_cuda(freq), amplitude=amplitude, cache=case["cache"],
             n_pages=pages, table=_cuda(table), ctx=_cuda(ctx), bound=int(ctx.max()), position=_cuda(pad((ctx[:, None] + depth).astype(np.int32), 0)), slot=_cuda(pad(slot, -1)))
    s["qkv"] = (torch.randn((R, (Hq + 2 * Hkv) * d), generator=g, device="cuda") * 1.5).to(dtype)
    s["bias"] = (torch.randn(((Hq + 2 * Hkv) * d,), generator=g, device="cuda") * 0.5).to(dtype) if case["bias"] else None
    s["q"] = torch.empty((R, Hq * d), dtype=dtype, device="cuda")
    pool = (pages, Hkv, PAGE)
    if case["cache"] == "model":
        s["k"], s["v"] = (torch.randn((1, *pool, d), generator=g, device="cuda").to(dtype) for _ in range(2))
    else:
        for x in "kv":
            s[x], s[x + "_exp"] = torch.zeros((1, *pool, d), dtype=torch.uint8, device="cuda"), torch.full((1, *pool), 127, dtype=torch.uint8, device="cuda")
        s["k_rows"], s["v_rows"] = (torch.zeros((1, B, n, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return s


def _prepare_pages(case, seed):
    rng = np.random.default_rng(seed)
    B = case["batch"]
    seq_len, n_new = _lengths(case), np.full(B, case["nodes"], np.int32)
    if case["admit"]:        # a third are new, with prompts of all lengths; of the others some have ended and the rest decode a token or two
        of = np.random.default_rng(B)
        new = of.random(B) < 0.34
        new[0] = True
        prompt = np.maximum(1, np.rint(case["nodes"] * np.exp(of.normal(-0.3, 0.6, B)))).clip(1, 4 * case["nodes"])
        n_new = np.where(new, prompt, of.integers(0, 3, B)).astype(np.int32)
        seq_len = np.where(new, 0, seq_len)
    which = rng.permutation(B)
    seq_len, n_new = seq_len[which].astype(np.int32), n_new[which]
    held = (seq_len + PAGE - 1) // PAGE
    want = np.maximum((seq_len + n_new + PAGE - 1) // PAGE - held, 0)
    n_free = int(want.sum()) * 15 // 16 if case["short"] else int(want.sum()) + 37
    n_pages = int(held.sum()) + n_free
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((B, max(1, int((held + want).max()))), -1, np.int32)
    for b, o in enumerate(np.cumsum(held) - held):
        table[b, :held[b]] = order[o:o + held[b]]
    free = np.full(max(1, n_pages), -1, np.int32)
    free[:n_free] = order[int(held.sum()):]
    rows = int(n_new.sum()) + 5      # a buffer of a few rows more than the step has
    i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")
    return dict(kind="pages", B=B, rows=rows, n_pages=n_pages, table=_cuda(table), free=_cuda(free), n_free=_cuda(np.array([n_free], np.int32)), held=_cuda(held.astype(np.int32)),
                seq_len=_cuda(seq_len), n_new=_cuda(n_new), row_start=i32(B + 1), row_seq=i32(rows), position=i32(rows), slot=torch.empty((rows,), dtype=torch.int64, device="cuda"), granted=i32(B))


def prepare(case, seed):
    return {"sample": _prepare_logits, "filter": _prepare_logits, "rope": _prepare_rope, "pages": _prepare_pages}[case["kind"]](case, seed)


# ---- the plain forms

def _share(s31, S):
    """ceil(s31 * S / 2^31) of whole numbers in 64 bits, s31 <= 2^31."""
    return 2 * s31 * (S >> 32) + ((s31 * (S & 0xffffffff) + 0x7fffffff) >> 31)


def _plain_logits(s):
    B, n, V = s["B"], s["n"], s["V"]
    tau, top_k, top_p, min_p = (None if v is None else v.repeat_interleave(n, output_size=B * n)[:, None] for v in s["filter"])
    x = s["logits"].float().view(B * n, V)
    top = x.amax(-1, keepdim=True)
    greedy = ~(tau > 0)
    tau = torch.where(greedy, 1.0, tau.double())
    z = torch.where(x == top, 0.0, x.double() / tau - top.double() / tau)
    W = torch.where(x > -math.inf, torch.floor(torch.exp(z) * 2.0 ** 32), 0.0).long()
    xs, order = torch.sort(x, dim=-1, descending=True, stable=True)
    Ws = W.gather(1, order)
    rank = torch.arange(V, device="cuda")[None]
    limit = torch.where(greedy, 1, V if top_k is None else torch.where(top_k > 0, top_k, V))
    keep = (xs > -math.inf) & (rank < limit)
    if top_p is not None:
        Wk = torch.where(keep, Ws, 0)
        run = Wk.cumsum(-1)
        share = _share(torch.floor(top_p.double().clamp(0, 1) * 2.0 ** 31).long(), run[:, -1:]).clamp(min=1)
        keep &= (run - Wk < share) | ~(top_p < 1)
    if min_p is not None:
        keep &= (Ws >= torch.floor(min_p.double().clamp(0, 1) * 2.0 ** 32).long())
    kept = torch.zeros_like(keep).scatter_(1, order, keep)
    count = kept.sum(-1).int().view(B, n)
    if s["kind"] == "filter":
        return s["logits"].masked_fill(~kept.view(B, n, V), -math.inf), count
    run = torch.where(kept, W, 0).cumsum(-1)
    S, all_ = run[:, -1:], W.sum(-1, keepdim=True)
    u = s["u"].view(B * n, 1).long() & 0xffffffff
    lo = S & 0xffffffff
    thr = u * (S >> 32) + (((u >> 16) * lo + (((u & 0xffff) * lo) >> 16)) >> 16)
    token = (run <= thr).sum(-1, keepdim=True)
    some = S > 0
    zt = z.gather(1, token.clamp(max=V - 1))
    lp = torch.cat([torch.where(some, zt - torch.log(t.double() * 2.0 ** -32), -math.inf) for t in (S, all_)], -1)
    return torch.where(some, token, -1).int().view(B, n), lp.float().view(B, n, 2), count


def _codes(x):
    """(e4m3 codes, exponent bytes) of finite fp32 rows: values are code * 2^(E - 127), E - 127 the smallest e >= -126 with max|x| <= 448 * 2^e."""
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m > 0, (e - 9 + (m > 0.875).to(e.dtype)).clamp(min=-126), -126)
    return (x * torch.exp2(-e.float())[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _pairs(x, r, interleaved):
    return (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])


def _plain_rope(s):
    Hq, Hkv, d, R, r = s["Hq"], s["Hkv"], s["d"], s["R"], s["rot"]
    x = s["qkv"].float()
    if s["bias"] is not None:
        x = x + s["bias"].float()
    x = x.view(R, Hq + 2 * Hkv, d)
    angle = s["position"].double()[:, None] * s["freq"]
    c, sn = ((f(angle) * s["amplitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    a, b = _pairs(x[:, :Hq + Hkv], r, s["interleaved"])
    y = (a * c - b * sn, a * sn + b * c)
    y = torch.stack(y, -1).flatten(-2) if s["interleaved"] else torch.cat(y, -1)
    y = torch.cat([y, x[:, :Hq + Hkv, r:]], -1)
    new = {"k": y[:, Hq:], "v": x[:, Hq + Hkv:]}
    q = y[:, :Hq].reshape(R, Hq * d).to(s["dtype"])
    ok = s["slot"] >= 0
    pg, row = s["slot"][ok] // PAGE, s["slot"][ok] % PAGE
    if s["cache"] == "model":
        for t in "kv":
            s[t][0, pg, :, row] = new[t][ok].to(s["dtype"])
        return q, s["k"], s["v"]
    for t in "kv":
        s[t][0, pg, :, row], s[t + "_exp"][0, pg, :, row] = _codes(new[t][ok])
    rows = [s[t][0, pg, :, row].view(torch.float8_e4m3fn).float() * torch.exp2(s[t + "_exp"][0, pg, :, row].float() - 127.0)[..., None] for t in "kv"]
    return (q, *(t.view(1, s["B"], s["n"], Hkv, d).to(torch.bfloat16) for t in rows))


def _plain_pages(s):
    B, rows, table, free, held = s["B"], s["rows"], s["table"], s["free"], s["held"]
    width = table.shape[1]
    # grow: sequences in order, as long as all of the pages that they need are left
    need = (s["seq_len"] + s["n_new"] + PAGE - 1) // PAGE
    want = (need - held).clamp(min=0)
    run = want.cumsum(0)
    granted = (run <= s["n_free"]) | (want == 0)
    take = torch.where(granted, want, 0)
    first = take.cumsum(0) - take
    j = torch.arange(width, device="cuda")[None]
    fresh = (j >= held[:, None]) & (j < (held + take)[:, None])
    at = s["n_free"] - 1 - (first[:, None] + j - held[:, None])
    table.copy_(torch.where(fresh, free[at.clamp(0, free.numel() - 1)], table))
    held += take
    s["n_free"] -= take.sum()
    # the rows of all sequences side by side: where each belongs, its position and its slot
    start = torch.cat([s["n_new"].new_zeros(1), s["n_new"].cumsum(0).int()])
    t = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(start[1:].contiguous(), t.int(), right=True)
    real = seq < B
    b = seq.clamp(max=B - 1)
    pos = torch.where(real, s["seq_len"][b] + t - start[b], 0)
    page = table[b, (pos // PAGE).clamp(max=width - 1)].long()
    slot = torch.where(real & granted[b], page * PAGE + pos % PAGE, -1)
    # release: what lies behind the committed tokens again, so that the stack is as it was
    keep = (s["seq_len"] + PAGE - 1) // PAGE
    give = (held - keep).clamp(min=0)
    after = give.sum() - give.cumsum(0)
    back = (j >= keep[:, None]) & (j < held[:, None])
    to = s["n_free"] + after[:, None] + held[:, None] - 1 - j
    spare = torch.cat([free, free.new_zeros(1)])
    spare[torch.where(back, to, free.numel()).long()] = torch.where(back, table, 0)
    free.copy_(spare[:-1])
    table.masked_fill_(back, -1)
    held -= give
    s["n_free"] += give.sum()
    return start, torch.where(real, seq, -1).int(), pos.int(), slot, granted.int(), table, held, free, s["n_free"]


# ---- the framework's calls

def _own_logits(s):
    from paper_2511_16665_amd import binding as tlt
    code = tlt.TLT_F32 if s["logits"].dtype == torch.float32 else tlt.TLT_BF16
    if "ws" not in s:    # what a program keeps
        s["ws"] = tlt.sample_workspace(s["B"] * s["n"], s["V"])
        s["asked"] = tlt.SampleFilter(*s["filter"])
    if s["kind"] == "filter":
        tlt.sample_filter(code, s["logits"], s["asked"], s["out"], s["kept"], s["ws"])
        return s["out"], s["kept"]
    tlt.sample(code, s["logits"], s["asked"], s["u"], s["token"], s["logprob"], s["kept"], s["ws"])
    return s["token"], s["logprob"], s["kept"]


def _own_rope(s):
    from paper_2511_16665_amd import binding as tlt
    code = tlt.TLT_F32 if s["dtype"] == torch.float32 else tlt.TLT_BF16
    if "kv" not in s:
        s["rope"] = tlt.Rope(s["freq"], s["interleaved"], s["amplitude"])
        s["kv"] = tlt.KV(s["k"], s["v"], s["table"], s["ctx"], s["bound"]) if s["cache"] == "model" else tlt.KV8(s["k"], s["v"], s["k_exp"], s["v_exp"], s["table"], s["ctx"], s["bound"])
    tlt.rope_write(code, s["Hq"], s["Hkv"], s["d"], s["rope"], s["qkv"], s["bias"], s["position"], s["slot"], s["kv"], 0, s["q"])
    if s["cache"] == "model":
        return s["q"], s["k"], s["v"]
    tlt.kv8_read(tlt.TLT_BF16, s["kv"], s["ctx"], None, s["k_rows"], s["v_rows"])
    return s["q"], s["k_rows"], s["v_rows"]


def _own_pages(s):
    from paper_2511_16665_amd import binding as tlt
    if "pages" not in s:
        s["pages"] = tlt.Pages(s["free"], s["n_free"], s["held"], s["table"], PAGE)
    tlt.pages_grow(s["pages"], s["seq_len"], s["n_new"], None, s["row_start"], s["row_seq"], s["position"], s["slot"], s["granted"])
    tlt.pages_release(s["pages"], s["seq_len"])
    return s["row_start"], s["row_seq"], s["position"], s["slot"], s["granted"], s["table"], s["held"], s["free"], s["n_free"]


def run(state):
    if own:
        return {"sample": _own_logits, "filter": _own_logits, "rope": _own_rope, "pages": _own_pages}[state["kind"]](state)
    return {"sample": _plain_logits, "filter": _plain_logits, "rope": _plain_rope, "pages": _plain_pages}[state["kind"]](state)


# ---- what a pass cannot do without

def work(case):
    B, n, kind = case["batch"], case["nodes"], case["kind"]
    if kind in ("sample", "filter"):
        e = 4 if case["dtype"] == "fp32" else 2
        values = B * n * case["vocab"]
        return {"bytes": float(values * e * (2 if kind == "filter" else 1) + B * n * 20), "flops": 30.0 * values}     # (an exponential in double per value)
    if kind == "rope":
        Hq, Hkv, d = HEADS[case["heads"]]
        e, R = 4 if case["heads"] == "tiny" else 2, B * n + case["pad"]
        rows = R * ((2 * Hq + 2 * Hkv) * d * e + 12)
        cached = B * n * 2 * Hkv * (d + 1) if case["cache"] == "8 bits" else B * n * 2 * Hkv * d * e
        back = B * n * Hkv * (2 * (d + 1) + 4 * d) if case["cache"] == "8 bits" else 0
        return {"bytes": float(rows + cached + back), "flops": 3.0 * R * (Hq + Hkv) * case["rot"]}
    rows = B * n // (3 if case["admit"] else 1)
    return {"bytes": float(B * 24 + rows * 16 + 4 * rows // PAGE * 4), "flops": float(10 * rows)}


# ---- the definitions, a row or a sequence at a time, in 64 bits

def _exact_logits(case, s):
    B, n, V = s["B"], s["n"], s["V"]
    tau, top_k, top_p, min_p = (None if v is None else v.tolist() for v in s["filter"])
    logits = s["logits"].view(B * n, V)
    tokens, logprobs, counts, rows = [], [], [], []
    for i in range(B * n):
        b, l = i // n, logits[i].double()
        t = tau[b] if tau[b] > 0 else 1.0
        best = l.max()
        d = l / t - best / t
        w = torch.where(l == best, 2.0 ** 32, torch.floor(2.0 ** 32 * torch.exp(d)))
        w = torch.where(l == -math.inf, 0.0, w).long()
        order = torch.argsort(-l, stable=True)                  # (ties: the lower index first)
        order = order[l[order] != -math.inf]
        if not tau[b] > 0:
            order = order[:1]
        elif top_k is not None and top_k[b] > 0:
            order = order[:top_k[b]]
        if top_p is not None and top_p[b] < 1 and len(order):
            run = torch.cumsum(w[order], 0)
            # kept while what comes before is less than the share: whole numbers, so compare with the share rounded up
            share = -((-int(math.floor(max(top_p[b], 0.0) * 2 ** 31)) * int(run[-1])) // 2 ** 31)
            order = order[:1 + int((run < max(share, 1)).sum())]
        if min_p is not None:
            order = order[w[order] >= int(math.floor(min(max(min_p[b], 0.0), 1.0) * 2 ** 32))]
        counts.append(len(order))
        if s["kind"] == "filter":
            row = torch.full((V,), -math.inf, dtype=torch.float64, device="cuda")
            row[order] = l[order]
            rows.append(row)
            continue
        chosen = torch.sort(order).values
        if not len(chosen):
            tokens.append(-1), logprobs.append([-math.inf, -math.inf])
            continue
        run = torch.cumsum(w[chosen], 0)
        aim = (int(s["u"].view(-1)[i]) % 2 ** 32) * int(run[-1]) >> 32
        token = int(chosen[int(torch.searchsorted(run, aim, right=True))])
        tokens.append(token)
        at = 0.0 if bool(l[token] == best) else float(d[token])
        logprobs.append([at - math.log(int(run[-1]) / 2 ** 32), at - math.log(int(w.sum()) / 2 ** 32)])
    count = torch.tensor(counts, dtype=torch.int32).view(B, n)
    if s["kind"] == "filter":
        return torch.stack(rows).view(B, n, V), count
    return torch.tensor(tokens, dtype=torch.int32).view(B, n), torch.tensor(logprobs, dtype=torch.float64).view(B, n, 2), count


def _nearest(x):
    """Rows in 64 bits as the 8-bit cache keeps them: the nearest of e4m3's values times the row's power of two (halves to the even fraction)."""
    a = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(a / 448.0)).clamp(min=-126.0)
    e = torch.where(448.0 * torch.pow(2.0, e - 1) >= a, e - 1, e)
    e = torch.where(448.0 * torch.pow(2.0, e) < a, e + 1, e).clamp(min=-126.0)
    y = x / torch.pow(2.0, e)
    step = torch.pow(2.0, torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(y / step) * step * torch.pow(2.0, e)


def _exact_rope(case, s):
    Hq, Hkv, d, R, r = s["Hq"], s["Hkv"], s["d"], s["R"], s["rot"]
    x = s["qkv"].double()
    if s["bias"] is not None:
        x = x + s["bias"].double()
    x = x.view(R, Hq + 2 * Hkv, d)
    one = slice(0, r, 2) if s["interleaved"] else slice(0, r // 2)
    two = slice(1, r, 2) if s["interleaved"] else slice(r // 2, r)
    turn = s["position"].double()[:, None] * s["freq"][None]
    z = torch.complex(x[:, :Hq + Hkv, one].contiguous(), x[:, :Hq + Hkv, two].contiguous()) * torch.polar(torch.full_like(turn, s["amplitude"]), turn)[:, None]
    y = x.clone()
    y[:, :Hq + Hkv, one], y[:, :Hq + Hkv, two] = z.real, z.imag
    q, k, v = y[:, :Hq].reshape(R, Hq * d), y[:, Hq:Hq + Hkv], y[:, Hq + Hkv:]
    if s["cache"] == "8 bits":
        rows = s["B"] * s["n"]
        return (q, *(_nearest(t[:rows]).view(1, s["B"], s["n"], Hkv, d) for t in (k, v)))
    pools = []
    for pool, new in ((s["k"], k), (s["v"], v)):
        flat = pool[0].double().permute(0, 2, 1, 3).reshape(-1, Hkv, d)      # slots
        flat[s["slot"][s["slot"] >= 0]] = new[s["slot"] >= 0]
        pools.append(flat.view(s["n_pages"], PAGE, Hkv, d).permute(0, 2, 1, 3).contiguous()[None])
    return (q, *pools)


def exact(case, seed):
    if case["kind"] == "pages":
        return None          # whole numbers alone
    if case["kind"] != "rope" and case["batch"] * case["nodes"] * case["vocab"] > 5e8:
        return None
    s = prepare(case, seed)
    return _exact_rope(case, s) if case["kind"] == "rope" else _exact_logits(case, s)
