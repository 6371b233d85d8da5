"""Operators of a decoder trained on packed documents, beside the layer shard: what is measured of them.

Kinds of case:
  rope   rotary positions on the rows of a fused QKV projection (tp_layer_rope_fwd, tp_layer_rope_bwd)
  attn   attention of packed sequences with grouped heads (tp_layer_attn_packed_fwd, tp_layer_attn_packed_bwd)
  loss   softmax cross entropy of a vocabulary shard without kept logits (tp_layer_lm_loss_fwd, _join, _bwd)

Rows of qkv are [(nq + 2 nkv) dh] with columns (q | k | v, head, dh), as in the layer; sequences lie one after another in the
rows, sequence b in rows offsets[b] .. offsets[b + 1]. Weights of the vocabulary are [V, H], a row per token of the vocabulary.

Sizes are those of the named configurations of synthetic/configs.py (local heads, hidden sizes, tokens of a micro-batch), of
the tests, or generic ones of the same ranges. Activations and upstream gradients are N(0, 1), weights N(0, 0.02).
"""
import math
import random

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def _rope(name, dtype, tokens, nq, nkv, head_dim, rot, pairs, scaling, far, train):
    case = {"kind": "rope", "dtype": dtype, "tokens": tokens, "nq": nq, "nkv": nkv, "head_dim": head_dim, "rot": rot, "pairs": pairs,
            "scaling": scaling, "far": far, "train": train}
    return {"name": name, **case} if name else case


def _attn(name, dtype, tokens, docs, shortest, nq, nkv, head_dim, causal, train):
    case = {"kind": "attn", "dtype": dtype, "tokens": tokens, "docs": docs, "shortest": shortest, "nq": nq, "nkv": nkv,
            "head_dim": head_dim, "causal": causal, "train": train}
    return {"name": name, **case} if name else case


def _loss(name, dtype, tokens, hidden, vocab, ranks, rank, ignored):
    """vocab: rows of this rank's shard; ranks: how many shards the vocabulary has."""
    case = {"kind": "loss", "dtype": dtype, "tokens": tokens, "hidden": hidden, "vocab": vocab, "ranks": ranks, "rank": rank,
            "ignored": ignored}
    return {"name": name, **case} if name else case


def listed():
    return [
        # a short micro-batch of a narrow shard: a launch and little else
        _rope("rope-short", "bf16", 64, 8, 2, 64, 64, "half", "none", 0, False),
        # forward and backward beside the layer of GPT-3 175B TP 8 (12 local heads of 128), four micro-batches packed
        _rope("rope-train-175b-tp8", "bf16", 8192, 12, 12, 128, 128, "half", "none", 0, True),
        # float, neighbouring pairs, part of an 80-wide head, a context stretched by parts, positions far out, odd rows
        _rope("rope-part-stretched-f32", "f32", 3001, 32, 8, 80, 32, "adjacent", "parts", 120000, True),
        # the tiny float GPT: two sequences of 128, one key head (bring-up and parity)
        _attn("attn-tiny-f32", "f32", 256, 2, 128, 2, 1, 64, True, True),
        # an encoder's micro-batch with its padding taken out: 4096 tokens of sentences from 8 tokens on, no mask
        _attn("attn-encoder-bert-large-tp4", "bf16", 4096, 24, 8, 4, 4, 64, False, True),
        # a decoder's training step on packed documents, eight query heads to a key head
        _attn("attn-decoder-grouped", "bf16", 8192, 12, 64, 16, 2, 128, True, True),
        # evaluation: forward only, one long document and a few short ones (12 local heads of GPT-3 175B TP 8, grouped by three)
        _attn("attn-long-forward", "bf16", 16384, 3, 500, 12, 4, 128, True, False),
        # sizes that divide by nothing: head size 80, groups of five, lengths from one token on
        _attn("attn-ragged", "bf16", 3003, 17, 1, 10, 2, 80, True, True),
        # float at a real width
        _loss("loss-encoder-f32", "f32", 512, 1024, 7631, 4, 1, 0.85),
        # the last layer of GPT-3 13B TP 4: two micro-batches, a quarter of the padded vocabulary
        _loss("loss-13b-tp4", "bf16", 4096, 5120, 12576, 4, 0, 0.0),
        # the whole vocabulary, an odd number of rows, on one rank: in pieces
        _loss("loss-whole-vocabulary", "bf16", 8192, 2048, 50257, 1, 0, 0.02),
        # a few tokens against many weights: bound by reading and writing them
        _loss("loss-few-tokens", "bf16", 37, 4096, 50257, 1, 0, 0.1),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _draw_rope(rng):
    while True:
        head_dim = rng.choice([64, 64, 128, 128, 32, 80, 96, 104])
        rot = rng.choice([head_dim, head_dim, head_dim // 2 // 8 * 8, head_dim // 4 // 8 * 8]) or head_dim
        nkv = rng.choice([1, 2, 4, 8])
        case = _rope(None, rng.choice(["bf16", "bf16", "f32"]), round(_log_uniform(rng, 1, 16384)), nkv * rng.choice([1, 2, 3, 5, 8]), nkv,
                     head_dim, rot, rng.choice(["half", "adjacent"]), rng.choice(["none", "linear", "base", "parts"]),
                     rng.choice([0, 0, 1000, 120000]), rng.random() < 0.6)
        if work(case)["bytes"] <= 3.1e8:
            return case


def _draw_attn(rng):
    while True:
        tokens = round(_log_uniform(rng, 1, 12000))
        nkv = rng.choice([1, 1, 2, 4, 8])
        case = _attn(None, rng.choice(["bf16", "bf16", "bf16", "f32"]), tokens, max(1, min(tokens, round(_log_uniform(rng, 1, 64)))), 1,
                     nkv * rng.choice([1, 1, 2, 3, 4, 5, 8]), nkv, rng.choice([64, 64, 128, 128, 80, 32, 96, 104]), rng.random() < 0.7, rng.random() < 0.7)
        if case["nq"] <= 32 and case["tokens"] ** 2 * case["nq"] <= 1.2e9 and work(case)["flops"] <= (3.0e11 if case["dtype"] == "bf16" else 3.0e10):
            return case


def _draw_loss(rng):
    while True:
        dtype, ranks = rng.choice(["bf16", "bf16", "bf16", "f32"]), rng.choice([1, 1, 2, 4, 8])
        vocab = round(_log_uniform(rng, 500, 128256) / ranks)
        case = _loss(None, dtype, round(_log_uniform(rng, 1, 8192)), 8 * round(_log_uniform(rng, 256, 12288) / 8), max(vocab, 1), ranks,
                     rng.randrange(ranks), rng.choice([0.0, 0.0, 0.1, 0.85]))
        if work(case)["flops"] <= (2.5e12 if dtype == "bf16" else 1.0e11) and case["hidden"] * case["vocab"] <= 2.5e8:
            return case


def draw(rng):
    return rng.choice([_draw_rope, _draw_attn, _draw_attn, _draw_loss, _draw_loss])(rng)


def _lengths(case, seed):
    """Lengths of the packed documents: drawn by their logarithm from `shortest` on, scaled to fill the rows."""
    rng, n, short = random.Random(seed), case["docs"], case["shortest"]
    spare = case["tokens"] - n * short
    share = [_log_uniform(rng, 1.0, 60.0) for _ in range(n)]
    got = [short + int(spare * s / sum(share)) for s in share]
    got[rng.randrange(n)] += case["tokens"] - sum(got)
    return got


class _Random:
    """Seeded normal tensors on the GPU."""

    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.dtype = _TORCH[dtype]

    def __call__(self, *shape, sigma=1.0, dtype=None):
        t = torch.randn(*shape, generator=self.g, device="cuda", dtype=torch.float32)
        return t.mul_(sigma).to(dtype or self.dtype)

    def whole(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda", dtype=torch.int32)


def _frequencies(rot, scaling):
    """Radians per position of each pair, and the factor of the rotated values: base 10000, a context of 4096 stretched eightfold.
    linear: positions divided; base: a larger base; parts: pairs of few turns over the context divided, of many kept, a ramp
    between (Peng et al. 2023)."""
    base, stretch, context = 10000.0, 8.0, 4096.0
    if scaling == "base" and rot > 2:
        base *= stretch ** (rot / (rot - 2))
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [x / stretch for x in f], 1.0
    if scaling == "parts":
        keep = [min(1.0, max(0.0, (context * x / (2 * math.pi) - 1.0) / (32.0 - 1.0))) for x in f]
        return [k * x + (1 - k) * x / stretch for k, x in zip(keep, f)], 0.1 * math.log(stretch) + 1.0
    return f, 1.0


def work(case):
    es = _BYTES[case["dtype"]]
    if case["kind"] == "rope":
        n = case["tokens"] * (case["nq"] + 2 * case["nkv"]) * case["head_dim"]
        passes = 2 if case["train"] else 1
        return {"bytes": passes * 2 * n * es + 4 * case["tokens"], "flops": passes * 3 * case["tokens"] * (case["nq"] + case["nkv"]) * case["rot"]}
    if case["kind"] == "attn":
        M, nq, nkv, dh = case["tokens"], case["nq"], case["nkv"], case["head_dim"]
        pairs = sum(n * (n + 1) // 2 if case["causal"] else n * n for n in _lengths(case, 1))
        w, o = M * (nq + 2 * nkv) * dh * es, M * nq * dh * es
        lse = M * nq * 4
        return {"bytes": w + o + lse + (2 * w + 2 * o + lse if case["train"] else 0), "flops": (14 if case["train"] else 4) * nq * dh * pairs}
    M, H, V = case["tokens"], case["hidden"], case["vocab"]
    # logits, dx and dw; x and w read forward and again backward
    return {"bytes": es * (3 * M * H + 3 * V * H) + 16 * M, "flops": 6 * M * H * V}


def prepare(case, seed):
    rnd = _Random(seed, case["dtype"])
    return {"rope": _prepare_rope, "attn": _prepare_attn, "loss": _prepare_loss}[case["kind"]](case, rnd, seed)


def _prepare_rope(case, rnd, seed):
    M, width = case["tokens"], (case["nq"] + 2 * case["nkv"]) * case["head_dim"]
    freq, factor = _frequencies(case["rot"], case["scaling"])
    # positions restart with every document; with `far` they go on from far out, as in a stretched context
    rng = random.Random(seed)
    start = torch.arange(M, device="cuda", dtype=torch.int32)
    pos = start % rng.randrange(max(1, M // 8), max(2, M)) + (rng.randrange(case["far"], 2 * case["far"]) if case["far"] else 0)
    s = {"case": case, "positions": pos.to(torch.int32), "freq": torch.tensor(freq, dtype=torch.float64, device="cuda"), "factor": factor,
         "qkv": rnd(M, width)}
    s["out"] = torch.empty_like(s["qkv"])
    if case["train"]:
        s["dqkv"] = rnd(M, width)
        s["dout"] = torch.empty_like(s["dqkv"])
    return s


def _prepare_attn(case, rnd, seed):
    M, nq, nkv, dh = case["tokens"], case["nq"], case["nkv"], case["head_dim"]
    offsets = [0]
    for n in _lengths(case, seed):
        offsets.append(offsets[-1] + n)
    f32 = dict(dtype=torch.float32, device="cuda")
    s = {"case": case, "qkv": rnd(M, (nq + 2 * nkv) * dh), "offsets": torch.tensor(offsets, dtype=torch.int32, device="cuda"),
         "o": torch.empty(M, nq * dh, dtype=rnd.dtype, device="cuda"), "lse": torch.empty(M, nq, **f32)}
    if case["train"]:
        s.update(d_o=rnd(M, nq * dh), dqkv=torch.empty_like(s["qkv"]), dsum=torch.empty(M, nq, **f32))
    if own:
        # the plan of the batch, which every layer of a step shares, and a workspace
        import paper_2111_05972_amd as pkg
        dt, n = pkg.TPL_BF16 if case["dtype"] == "bf16" else pkg.TPL_F32, case["docs"]
        s["plan"] = torch.empty(pkg.tp_layer_pack_plan_bytes(n, M, nq, nkv), dtype=torch.uint8, device="cuda")
        pkg.tp_layer_pack_plan(n, M, s["offsets"], nq, nkv, case["causal"], s["plan"], stream=torch.cuda.current_stream())
        s["ws"] = torch.empty(max(pkg.tp_layer_attn_packed_workspace_bytes(dt, n, M, nq, nkv, dh, case["causal"], bwd) for bwd in (False, True)),
                              dtype=torch.uint8, device="cuda")
    return s


def _prepare_loss(case, rnd, seed):
    M, H, V, T = case["tokens"], case["hidden"], case["vocab"], case["ranks"]
    first = V * case["rank"]
    s = {"case": case, "first": first, "x": rnd(M, H), "w": rnd(V, H, sigma=0.02), "labels": rnd.whole(0, V * T, M)}
    gone = torch.rand(M, generator=rnd.g, device="cuda") < case["ignored"]
    s["labels"] = torch.where(gone, torch.full_like(s["labels"], -100), s["labels"])
    s["dloss"] = torch.full((M,), 1.0 / max(1, int((~gone).sum())), dtype=torch.float32, device="cuda")    # the mean over the labelled tokens
    # what the other ranks' gathered statistics look like: log-sum-exp of their logits, and the target's logit where it is theirs
    spread = 0.02 * math.sqrt(H)
    s["stats"] = torch.empty(T, M, 2, dtype=torch.float32, device="cuda")
    s["stats"][:, :, 0] = math.log(V) + 0.5 * spread ** 2 + 0.01 * rnd(T, M, dtype=torch.float32)
    theirs = (s["labels"] // V) == torch.arange(T, device="cuda", dtype=torch.int32).view(T, 1)
    s["stats"][:, :, 1] = torch.where(theirs, spread * rnd(T, M, dtype=torch.float32), torch.full((T, M), -math.inf, device="cuda"))
    s["loss"], s["lse"] = (torch.empty(M, dtype=torch.float32, device="cuda") for _ in range(2))
    s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
    if own:
        import paper_2111_05972_amd as pkg
        dt = pkg.TPL_BF16 if case["dtype"] == "bf16" else pkg.TPL_F32
        s["ws"] = torch.empty(max(pkg.tp_layer_lm_loss_workspace_bytes(dt, M, H, V, bwd) for bwd in (False, True)), dtype=torch.uint8, device="cuda")
    return s


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"rope": _own_rope, "attn": _own_attn, "loss": _own_loss}[kind](state)
    return {"rope": _plain_rope, "attn": _plain_attn, "loss": _plain_loss}[kind](state)


# ---- the framework's entry points -------------------------------------------------------------------------------------
def _own_rope(s):
    import paper_2111_05972_amd as pkg
    c = s["case"]
    st = torch.cuda.current_stream()
    args = (pkg.TPL_BF16 if c["dtype"] == "bf16" else pkg.TPL_F32, c["tokens"], c["nq"], c["nkv"], c["head_dim"], c["rot"],
            pkg.TPL_ROPE_HALF if c["pairs"] == "half" else pkg.TPL_ROPE_ADJACENT, s["freq"], s["factor"], s["positions"])
    pkg.tp_layer_rope_fwd(*args, s["qkv"], s["out"], stream=st)
    if not c["train"]:
        return s["out"]
    pkg.tp_layer_rope_bwd(*args, s["dqkv"], s["dout"], stream=st)
    return s["out"], s["dout"]


def _own_attn(s):
    import paper_2111_05972_amd as pkg
    c = s["case"]
    st = torch.cuda.current_stream()
    args = (pkg.TPL_BF16 if c["dtype"] == "bf16" else pkg.TPL_F32, c["docs"], c["tokens"], c["nq"], c["nkv"], c["head_dim"], c["causal"], s["plan"])
    pkg.tp_layer_attn_packed_fwd(*args, s["qkv"], s["o"], s["lse"], ws=s["ws"], stream=st)
    if not c["train"]:
        return s["o"], s["lse"]
    pkg.tp_layer_attn_packed_bwd(*args, s["qkv"], s["o"], s["lse"], s["d_o"], s["dqkv"], s["dsum"], ws=s["ws"], stream=st)
    return s["o"], s["lse"], s["dqkv"]


def _own_loss(s):
    import paper_2111_05972_amd as pkg
    c = s["case"]
    st = torch.cuda.current_stream()
    dt, M, H, V, T = pkg.TPL_BF16 if c["dtype"] == "bf16" else pkg.TPL_F32, c["tokens"], c["hidden"], c["vocab"], c["ranks"]
    pkg.tp_layer_lm_loss_fwd(dt, M, H, V, s["first"], s["x"], s["w"], s["labels"], s["stats"][c["rank"]], s["ws"], stream=st)
    pkg.tp_layer_lm_loss_join(M, T, V * T, s["stats"], s["labels"], s["loss"], s["lse"], stream=st)
    pkg.tp_layer_lm_loss_bwd(dt, M, H, V, s["first"], V * T, s["x"], s["w"], s["labels"], s["lse"], s["dloss"], s["dx"], s["dw"], s["ws"], stream=st)
    return s["loss"], s["lse"], s["dx"], s["dw"]


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _rotate(c, s, rows, back):
    M, nq, nkv, dh, rot = c["tokens"], c["nq"], c["nkv"], c["head_dim"], c["rot"]
    x = rows.view(M, nq + 2 * nkv, dh)
    angle = s["positions"].to(torch.float64)[:, None] * s["freq"]
    cos = (angle.cos() * s["factor"]).float()[:, None, :]
    sin = (angle.sin() * (-s["factor"] if back else s["factor"])).float()[:, None, :]
    turned = x[:, :nq + nkv, :rot].float()
    if c["pairs"] == "half":
        a, b = turned[..., :rot // 2], turned[..., rot // 2:]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    else:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    out = x.clone()
    out[:, :nq + nkv, :rot] = turned.to(rows.dtype)
    return out.view(M, -1)


def _plain_rope(s):
    c = s["case"]
    out = _rotate(c, s, s["qkv"], False)
    return (out, _rotate(c, s, s["dqkv"], True)) if c["train"] else out


def _plain_attn(s):
    c = s["case"]
    M, nq, nkv, dh = c["tokens"], c["nq"], c["nkv"], c["head_dim"]
    group, scale = nq // nkv, 1.0 / math.sqrt(dh)
    rows = s["qkv"].float().view(M, nq + 2 * nkv, dh).transpose(0, 1)
    q = rows[:nq].contiguous()
    k = rows[nq:nq + nkv].repeat_interleave(group, dim=0).contiguous()
    v = rows[nq + nkv:].repeat_interleave(group, dim=0).contiguous()
    at = torch.arange(M, device=q.device)
    doc = torch.searchsorted(s["offsets"][1:].to(at.dtype), at, right=True)
    seen = doc[:, None] == doc[None, :]
    if c["causal"]:
        seen &= at[:, None] >= at[None, :]
    p = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(scale).masked_fill_(~seen, -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(total)
    lse = (top + total.log()).squeeze(-1).transpose(0, 1).contiguous()
    o = torch.matmul(p, v)
    wide = o.transpose(0, 1).reshape(M, nq * dh).to(s["qkv"].dtype)
    if not c["train"]:
        return wide, lse
    d_o = s["d_o"].float().view(M, nq, dh).transpose(0, 1).contiguous()
    dv = torch.matmul(p.transpose(1, 2).contiguous(), d_o)
    ds = torch.matmul(d_o, v.transpose(1, 2).contiguous()).sub_((d_o * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(1, 2).contiguous(), q)
    dk, dv = (t.view(nkv, group, M, dh).sum(1) for t in (dk, dv))
    return wide, lse, torch.cat([dq, dk, dv]).transpose(0, 1).reshape(M, -1).to(s["qkv"].dtype)


def _plain_loss(s):
    c = s["case"]
    M, V, T, rank = c["tokens"], c["vocab"], c["ranks"], c["rank"]
    x, w = s["x"].float(), s["w"].float()
    logits = torch.matmul(x, w.t())
    at = s["labels"].long() - s["first"]
    mine = (at >= 0) & (at < V)
    known = (s["labels"] >= 0) & (s["labels"] < V * T)
    others = torch.arange(T, device=x.device)[:, None] != rank
    top = logits.amax(-1)
    own_lse = top + (logits - top[:, None]).exp().sum(-1).log()
    all_lse = torch.where(others, s["stats"][:, :, 0], own_lse)
    most = all_lse.amax(0)
    lse = most + (all_lse - most).exp().sum(0).log()
    picked = torch.where(mine, logits.gather(1, at.clamp(0, V - 1)[:, None])[:, 0], torch.full_like(lse, -math.inf))
    target = torch.where(others, s["stats"][:, :, 1], picked).amax(0)
    loss = torch.where(known, lse - target, torch.zeros_like(lse))
    d = torch.where(known, s["dloss"], torch.zeros_like(lse))
    p = logits.sub_(lse[:, None]).exp_()
    p -= (torch.arange(V, device=x.device)[None, :] == at[:, None]).float()
    p *= d[:, None]
    return loss, lse, torch.matmul(p, w).to(s["x"].dtype), torch.matmul(p.t(), x).to(s["w"].dtype)


# ---- definitions in 64 bits -------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "attn": _exact_attn, "loss": _exact_loss}[case["kind"]](case, s, seed)


def _exact_rope(case, s, seed):
    """Pairs as complex numbers, multiplied by factor * e^(i angle) (backward: by its conjugate)."""
    M, rot, heads = case["tokens"], case["rot"], case["nq"] + case["nkv"]
    turn = torch.polar(torch.full((M, rot // 2), float(s["factor"]), dtype=torch.float64, device="cuda"),
                       s["positions"].double().outer(s["freq"])).unsqueeze(1)

    def turned(rows, by):
        y = rows.double().view(M, -1, case["head_dim"]).clone()
        z = y[:, :heads, :rot]
        first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if case["pairs"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        r = torch.complex(z[..., first].contiguous(), z[..., second].contiguous()) * by
        y[:, :heads, first], y[:, :heads, second] = r.real, r.imag
        return y.view(M, -1)
    out = turned(s["qkv"], turn)
    return (out, turned(s["dqkv"], turn.conj())) if case["train"] else out


def _exact_attn(case, s, seed):
    """Document by document and head by head."""
    nq, nkv, dh = case["nq"], case["nkv"], case["head_dim"]
    rows = s["qkv"].double().view(case["tokens"], nq + 2 * nkv, dh)
    o = torch.zeros(case["tokens"], nq, dh, dtype=torch.float64, device="cuda")
    lse = torch.zeros(case["tokens"], nq, dtype=torch.float64, device="cuda")
    grad = torch.zeros_like(rows) if case["train"] else None
    begin = 0
    for n in _lengths(case, seed):
        b, begin = slice(begin, begin + n), begin + n
        hidden = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1) if case["causal"] else None
        for h in range(nq):
            kh, vh = nq + h // (nq // nkv), nq + nkv + h // (nq // nkv)
            q, k, v = rows[b, h], rows[b, kh], rows[b, vh]
            scores = q @ k.t() / math.sqrt(dh)
            if hidden is not None:
                scores.masked_fill_(hidden, -math.inf)
            lse[b, h] = torch.logsumexp(scores, -1)
            weights = (scores - lse[b, h][:, None]).exp()
            o[b, h] = weights @ v
            if grad is not None:
                up = s["d_o"].double().view(case["tokens"], nq, dh)[b, h]
                grad[b, vh] += weights.t() @ up
                inner = weights * (up @ v.t() - (up * o[b, h]).sum(-1, keepdim=True)) / math.sqrt(dh)
                grad[b, h] = inner @ k
                grad[b, kh] += inner.t() @ q
    out = (o.view(case["tokens"], -1), lse)
    return out if grad is None else (*out, grad.view(case["tokens"], -1))


def _exact_loss(case, s, seed):
    V, T, rank = case["vocab"], case["ranks"], case["rank"]
    x, w, labels = s["x"].double(), s["w"].double(), s["labels"].long()
    z = x @ w.t()
    parts = [z.logsumexp(1) if r == rank else s["stats"][r, :, 0].double() for r in range(T)]
    lse = torch.stack(parts).logsumexp(0)
    valid = (labels >= 0) & (labels < V * T)
    owner, place = labels // V, labels % V
    target = torch.zeros_like(lse)
    for r in range(T):
        value = z[torch.arange(case["tokens"], device="cuda"), place] if r == rank else s["stats"][r, :, 1].double()
        target = torch.where(valid & (owner == r), value, target)
    loss = torch.where(valid, lse - target, 0.0)
    grad = (z - lse[:, None]).exp_()
    grad[(valid & (owner == rank)).nonzero()[:, 0], place[valid & (owner == rank)]] -= 1.0
    grad *= torch.where(valid, s["dloss"].double(), 0.0)[:, None]
    return loss, lse, grad @ w, grad.t() @ x
