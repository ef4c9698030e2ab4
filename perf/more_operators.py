"""The operators at the two ends of a model of tokens or nodes whose speed matters, as cases that can be timed.

A case names an operator (`op`) and its sizes:

  scores    log probabilities that rows of logits give to a token each, entropies, and the likeliest alternatives
  gradient  log probabilities and entropies, and then the logits' gradient for gradients of both (the loss is not known
            before the log probabilities are)
  loss      log probabilities and the gradient of their weighted sum, whose weights are known, in one call
  bias      position bias of attention: a table's row for the bucket of every distance of a key from a query, alone or added
            to scores [batch, heads, queries, keys]
  sums      the table's gradient: sums of the scores' gradients over all places of a bucket

Logits are [rows, cols], fp32, bf16 or fp16.  Widths are 10 to 47 classes of nodes (the example's 10) and generic
vocabularies of language models; `pad` is the share of positions without a token (-1), `mask` that of logits set to -inf, as
constrained decoding does, `gap` the unused columns behind a row.  Distances fall into logarithmic buckets on both sides of a
query or (`causal`) before it, or every distance up to a limit has a bucket of its own; `ragged`: every sequence of a batch has
an offset of its own between its first query and key, as in decoding with caches of different lengths.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


def _logits(name, op, rows, cols, kind, out="", scale=1.0, pad=0.0, mask=0.0, gap=0, tokens=True, entropy=False, top=0,
            weights="one"):
    c = {"op": op, "rows": rows, "cols": cols, "type": kind, "out": out or kind, "scale": scale, "pad": pad, "mask": mask,
         "gap": gap, "tokens": tokens, "entropy": entropy, "top": top, "weights": weights}
    return dict(c, name=name) if name else c


def _scores(name, op, batch, heads, queries, keys, kind, table, buckets, span, map="both", ragged=False, add=False):
    c = {"op": op, "batch": batch, "heads": heads, "queries": queries, "keys": keys, "type": kind, "table": table,
         "buckets": buckets, "span": span, "map": map, "ragged": ragged, "add": add}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one sequence decoding: the eight likeliest next tokens
        _logits("scores_token", "scores", 1, 32_000, "bf16", tokens=False, top=8),
        # a batch of sequences decoding at a temperature under a grammar that forbids a third of a large vocabulary
        _logits("scores_decode", "scores", 48, 128_000, "bf16", scale=1 / 0.7, mask=0.33, entropy=True, top=20),
        # answers of a node classifier (47 classes, as many as ogbn-products has): class, the three likeliest, doubt
        _logits("scores_nodes", "scores", 200_000, 47, "fp32", entropy=True, top=3),
        # fine-tuning on one short text, odd vocabulary, gradient in fp32
        _logits("gradient_short", "gradient", 129, 50_257, "fp16", out="fp32", pad=0.1),
        # rewards for sampled tokens and for entropy: both have gradients, a third of the places is padding
        _logits("gradient_policy", "gradient", 4096, 32_000, "bf16", pad=0.33, entropy=True),
        # the loss of a pre-training batch over a large vocabulary
        _logits("loss_prompt", "loss", 4096, 128_000, "bf16", pad=0.02),
        # a node classifier's loss with a weight for each node
        _logits("loss_nodes", "loss", 200_000, 47, "fp32", pad=0.05, gap=1, weights="each"),
        # a batch of sequences decoding, caches of different lengths, keys behind a sequence's end masked
        _scores("bias_token", "bias", 64, 16, 1, 4097, "bf16", "bf16", 32, 128, map="causal", ragged=True),
        # padded short texts: added to their scores, a bucket for every distance up to 64
        _scores("bias_ragged", "bias", 7, 12, 509, 1021, "fp32", "fp32", 129, 64, map="each", ragged=True, add=True),
        # a long prompt: the bias of all its heads
        _scores("bias_prompt", "bias", 1, 16, 4096, 4096, "bf16", "bf16", 32, 128),
        # gradient of a small batch, every distance up to 500 with a bucket
        _scores("sums_short", "sums", 3, 12, 129, 515, "fp32", "fp32", 1001, 500, map="each", ragged=True),
        # gradient of a training batch
        _scores("sums_prompt", "sums", 8, 16, 2048, 2048, "bf16", "fp32", 32, 128),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


# a drawn case moves no more than half of what the largest listed one (loss_prompt) does
_BYTES_MOST = 1.0e9


def _drawn(rng):
    op = rng.choice(["scores", "scores", "gradient", "loss", "bias", "bias", "sums", "sums"])
    kind = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    if op in ("bias", "sums"):
        batch, heads = round(_log_uniform(rng, 1, 64)), round(_log_uniform(rng, 1, 32))
        queries, keys = round(_log_uniform(rng, 1, 4096)), round(_log_uniform(rng, 1, 8192))
        map = rng.choice(["both", "causal", "each"])
        span = round(_log_uniform(rng, 16, 2000 if map == "each" else 20_000))
        buckets = 2 * span + 1 if map == "each" else rng.choice([8, 16, 32, 64])
        span = span if map == "each" else max(span, buckets)
        return _scores("", op, batch, heads, queries, keys, kind, rng.choice(["fp32", kind]), buckets, span, map,
                       rng.random() < 0.5, op == "bias" and rng.random() < 0.5)
    cols = round(_log_uniform(rng, 2, 262_144))
    cols = cols | 1 if rng.random() < 0.5 else -(-cols // 8) * 8
    rows = round(_log_uniform(rng, 1, 200_000))
    top = rng.choice([0, 0, 1, 5, 20, 64]) if op == "scores" and rows * cols <= 1e7 else 0
    tokens = op != "scores" or top == 0 or rng.random() < 0.5
    return _logits("", op, rows, cols, kind, out="" if op == "scores" else rng.choice(["fp32", kind]),
                   scale=rng.choice([1.0, 1.0, 1 / 0.7, 0.25]), pad=rng.choice([0.0, 0.0, 0.1, 0.6]) if tokens else 0.0,
                   mask=rng.choice([0.0, 0.0, 0.3]), gap=rng.choice([0, 0, 0, 1, 24]), tokens=tokens,
                   entropy=op != "loss" and rng.random() < 0.5, top=min(top, cols), weights=rng.choice(["one", "each"]))


def draw(rng):
    while True:
        c = _drawn(rng)
        if work(c)["bytes"] <= _BYTES_MOST:
            return c


# ---- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _prepare_logits(case, g):
    rows, cols = case["rows"], case["cols"]
    x = torch.empty((rows, cols + case["gap"]), dtype=_TYPES[case["type"]], device="cuda").normal_(0.0, 2.5, generator=g)
    s = {"logits": x[:, :cols], "tokens": None}
    if case["mask"]:
        for part in s["logits"].split(max(1, (1 << 26) // cols)):
            part.masked_fill_(torch.rand(part.shape, generator=g, device="cuda") < case["mask"], -math.inf)
    # tokens are those that the model tends to, and allowed: their logits are raised
    tokens = torch.randint(0, cols, (rows,), generator=g, device="cuda")
    s["logits"][torch.arange(rows, device="cuda"), tokens] = torch.randn(rows, generator=g, device="cuda").add_(6).to(x.dtype)
    if case["tokens"]:
        tokens[torch.rand(rows, generator=g, device="cuda") < case["pad"]] = -1
        s["tokens"] = tokens
    unit = 64.0 if case["out"] == "fp16" else 1.0 / rows  # gradients in fp16 come with the loss scaled
    s["d_logprobs"] = torch.randn(rows, generator=g, device="cuda") * unit
    s["d_entropy"] = torch.randn(rows, generator=g, device="cuda") * (0.1 * unit) if case["entropy"] else None
    s["weights"] = unit if case["weights"] == "one" else torch.rand(rows, generator=g, device="cuda") * unit
    if case["op"] != "scores":
        s["d_logits"] = torch.empty((rows, cols), dtype=_TYPES[case["out"]], device="cuda")
    return s


def _bucket_of(case):
    """The bucket of every distance (key - query) from -span to span, which stand for all beyond them."""
    span, buckets = case["span"], case["buckets"]
    if case["map"] == "each":
        return list(range(2 * span + 1))
    side = buckets // 2 if case["map"] == "both" else buckets
    near = side // 2                # distances with a bucket of their own; then they grow by a constant factor up to span
    ends = [near * (span / near) ** (k / (side - near)) for k in range(1, side - near)]
    before = [d if d < near else near + sum(d >= e for e in ends) for d in range(span + 1)]
    after = [-1] * span if case["map"] == "causal" else [side + b for b in before[1:]]
    return before[::-1] + after


def _prepare_scores(case, g):
    batch, queries, keys = case["batch"], case["queries"], case["keys"]
    shape = (batch, case["heads"], queries, keys)
    s = {"table": torch.empty((case["buckets"], case["heads"]), dtype=_TYPES[case["table"]], device="cuda").normal_(
        0.0, 1.0, generator=g)}
    s["bucket_of"] = torch.tensor(_bucket_of(case), dtype=torch.int32, device="cuda")
    # the first key's position less the first query's: the last query meets the last key, or (ragged) some key before it
    s["offset"] = queries - keys
    if case["ragged"]:
        s["offset"] = queries - 1 - torch.randint(0, keys, (batch,), generator=g, device="cuda")
    if case["op"] == "sums" or case["add"]:
        s["scores"] = torch.empty(shape, dtype=_TYPES[case["type"]], device="cuda").normal_(0.0, 1.0, generator=g)
    if case["op"] == "bias":
        # without an offset for each sequence, sequences share their bias
        s["out"] = torch.empty(shape if case["ragged"] or case["add"] else (1, *shape[1:]), dtype=_TYPES[case["type"]],
                               device="cuda")
    else:
        s["sums"] = torch.empty_like(s["table"])
    return s


def prepare(case, seed):
    g = _generator(seed)
    s = _prepare_logits(case, g) if "rows" in case else _prepare_scores(case, g)
    s["case"] = case
    if own:
        import paper_2206_10581_amd as tt
        if "rows" in case:
            s["own"] = tt.TokenScores(scale=case["scale"])
        else:
            s["own"] = tt.PositionBias(s["table"], s["bucket_of"], fill=-math.inf)
    return s


# ---- one pass

def _distribution(s):
    """Per row: (logit - largest) * scale, exp of it, the logarithm of its sum, entropy; and which rows count."""
    case, tokens = s["case"], s["tokens"]
    x = s["logits"].float()
    most = x.amax(1, keepdim=True)
    z = (x - torch.where(most == -math.inf, 0.0, most)) * case["scale"]
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    entropy = None
    if case["entropy"]:
        entropy = torch.log(total) - torch.where(e > 0, e * z, 0.0).sum(1, keepdim=True) / total
    counts = None if tokens is None else ((tokens >= 0) & (tokens < x.shape[1]))[:, None]
    return x, z, e, total, entropy, counts


def _plain_scores(s):
    case, tokens = s["case"], s["tokens"]
    x, z, e, total, entropy, counts = _distribution(s)
    logprobs = ids = values = None
    if tokens is not None:
        logprobs = torch.where(counts, z.gather(1, tokens.clamp(min=0)[:, None]) - torch.log(total), 0.0)[:, 0]
        entropy = torch.where(counts, entropy, 0.0) if entropy is not None else None
    if case["top"]:
        ids = x.sort(dim=1, descending=True, stable=True)[1][:, :case["top"]]
        values = z.gather(1, ids) - torch.log(total)
        if counts is not None:
            ids, values = torch.where(counts, ids, -1), torch.where(counts, values, -math.inf)
    return [logprobs, entropy[:, 0] if entropy is not None else None, ids, values]


def _plain_gradient(s, d_logprobs, d_entropy):
    tokens = s["tokens"]
    _, z, e, total, entropy, counts = _distribution(s)
    at = tokens.clamp(min=0)[:, None]
    log_total = torch.log(total)
    logprobs = torch.where(counts, z.gather(1, at) - log_total, 0.0)[:, 0]
    p = e / total
    d = p * -d_logprobs[:, None]
    d.scatter_add_(1, at, d_logprobs[:, None])
    if d_entropy is not None:
        d -= torch.where(p > 0, p * (z - log_total + entropy), 0.0) * d_entropy[:, None]
        entropy = torch.where(counts, entropy, 0.0)[:, 0]
    s["d_logits"].copy_(torch.where(counts, d * s["case"]["scale"], 0.0))
    return [logprobs, entropy, s["d_logits"]]


def _buckets(s):
    """The bucket of every place, [1 or batch, queries, keys]."""
    case, offset = s["case"], s["offset"]
    apart = torch.arange(case["keys"], device="cuda") - torch.arange(case["queries"], device="cuda")[:, None]
    apart = apart[None] + (offset[:, None, None] if torch.is_tensor(offset) else offset)
    return s["bucket_of"][apart.clamp(-case["span"], case["span"]) + case["span"]].long()


def _plain_bias(s):
    buckets, table = _buckets(s), s["table"].float()
    lines = torch.cat([table, torch.full_like(table[:1], -math.inf)]).t()  # the last: for no bucket
    bias = lines[:, buckets].transpose(0, 1)
    s["out"].copy_(s["scores"].float() + bias if s["case"]["add"] else bias)
    return s["out"]


def _plain_sums(s):
    case, offset = s["case"], s["offset"]
    queries, keys, span = case["queries"], case["keys"], case["span"]
    # rows from the last to the first, each one place further to the right: columns are diagonals
    g = s["scores"].double() if case["ragged"] else s["scores"].sum(0, keepdim=True, dtype=torch.float64)
    g = torch.nn.functional.pad(g.flip(2), (0, queries)).flatten(2)
    g = g[:, :, :queries * (keys + queries - 1)].unflatten(2, (queries, keys + queries - 1)).sum(2)
    apart = torch.arange(1 - queries, keys, device="cuda") + (offset[:, None] if torch.is_tensor(offset) else offset)
    buckets, g = s["bucket_of"][apart.clamp(-span, span) + span].long().flatten(), g.transpose(1, 2).flatten(0, 1)
    if case["buckets"] <= 64:
        s["sums"].copy_((buckets == torch.arange(case["buckets"], device="cuda")[:, None]).double() @ g)
        return s["sums"]
    total = torch.zeros((case["buckets"] + 1, case["heads"]), dtype=torch.float64, device="cuda")
    total.index_add_(0, torch.where(buckets < 0, case["buckets"], buckets), g)
    s["sums"].copy_(total[:-1])
    return s["sums"]


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        if op == "scores":
            return _plain_scores(state)
        if op == "gradient":
            return _plain_gradient(state, state["d_logprobs"], state["d_entropy"])
        if op == "loss":
            weights = torch.as_tensor(state["weights"], dtype=torch.float32, device="cuda").expand(case["rows"])
            logprobs, _, d = _plain_gradient(state, -weights, None)
            return [logprobs, None, d]
        return _plain_bias(state) if op == "bias" else _plain_sums(state)
    if op == "scores":
        r = state["own"].forward(state["logits"], state["tokens"], entropy=case["entropy"], top=case["top"])
        return [r.logprobs, r.entropy, r.top_ids, r.top_logprobs]
    if op == "gradient":
        r = state["own"].forward(state["logits"], state["tokens"], entropy=case["entropy"], state=True)
        state["own"].backward(state["logits"], state["tokens"], r.state, state["d_logprobs"], state["d_entropy"],
                              out=state["d_logits"])
        return [r.logprobs, r.entropy, state["d_logits"]]
    if op == "loss":
        logprobs, d = state["own"].loss(state["logits"], state["tokens"], state["weights"], out=state["d_logits"])
        return [logprobs, None, d]
    if op == "bias":
        if case["add"]:
            return state["own"].add_to(state["scores"], state["offset"], out=state["out"])
        return state["own"].forward(case["queries"], case["keys"], state["offset"], out=state["out"])
    return state["own"].backward(state["scores"], state["offset"], out=state["sums"])


# ---- what a pass cannot do without

def work(case):
    if "rows" in case:
        rows, cols = case["rows"], case["cols"]
        held = rows * (1.0 - case["pad"])
        moved = held * cols * _BYTES[case["type"]] + rows * ((8 if case["tokens"] else 0) + 4 + 12 * case["top"])
        if case["op"] != "scores":
            moved += rows * cols * _BYTES[case["out"]]
        return {"bytes": moved, "flops": held * cols * (4 if case["op"] == "scores" else 7)}
    shared = case["op"] == "bias" and not case["ragged"] and not case["add"]
    places = (1 if shared else case["batch"]) * case["heads"] * case["queries"] * case["keys"]
    moved = places * _BYTES[case["type"]] * (2 if case["add"] else 1)
    return {"bytes": moved + case["buckets"] * case["heads"] * _BYTES[case["table"]] + 4 * (2 * case["span"] + 1),
            "flops": places if case["op"] == "sums" or case["add"] else 0}


# ---- the definitions in 64 bits

def _exact_logits(case, s):
    rows, cols = case["rows"], case["cols"]
    tokens, upstream = s["tokens"], s["d_logprobs"]
    if case["op"] == "loss":
        upstream = -torch.as_tensor(s["weights"], dtype=torch.float64, device="cuda").expand(rows)
    d = torch.zeros((rows, cols), dtype=torch.float64, device="cuda") if case["op"] != "scores" else None
    logprobs = torch.zeros(rows, dtype=torch.float64, device="cuda") if tokens is not None else None
    entropy = torch.zeros(rows, dtype=torch.float64, device="cuda") if case["entropy"] else None
    ids = torch.full((rows, case["top"]), -1, device="cuda") if case["top"] else None
    values = torch.full((rows, case["top"]), -math.inf, dtype=torch.float64, device="cuda") if case["top"] else None
    kept = torch.arange(rows, device="cuda")
    if tokens is not None:
        kept = kept[(tokens >= 0) & (tokens < cols)]
    for r in kept.split(max(1, (1 << 26) // cols)):
        x = s["logits"][r].double() * case["scale"]
        logp = torch.log_softmax(x, 1)
        p = logp.exp()
        finite = torch.nan_to_num(logp, neginf=0.0)
        h = -(p * finite).sum(1)
        if tokens is not None:
            logprobs[r] = logp.gather(1, tokens[r][:, None])[:, 0]
        if entropy is not None:
            entropy[r] = h
        if ids is not None:
            order = s["logits"][r].double().sort(dim=1, descending=True, stable=True)[1][:, :case["top"]]
            ids[r], values[r] = order, logp.gather(1, order)
        if d is not None:
            part = -p * upstream[r].double()[:, None]
            part[torch.arange(len(r), device="cuda"), tokens[r]] += upstream[r].double()
            if case["op"] == "gradient" and s["d_entropy"] is not None:
                part -= p * (finite + h[:, None]) * s["d_entropy"][r].double()[:, None]
            d[r] = part * case["scale"]
    return [logprobs, entropy, ids, values] if case["op"] == "scores" else [logprobs, entropy, d]


def _exact_scores(case, s):
    batch, queries, keys, span = case["batch"], case["queries"], case["keys"], case["span"]
    offsets = s["offset"].tolist() if case["ragged"] else [s["offset"]] * batch
    bucket_of = s["bucket_of"].tolist()
    every = [[bucket_of[min(max(a + o, -span), span) + span] for a in range(1 - queries, keys)] for o in offsets]
    if case["op"] == "bias":
        out = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
        table = torch.cat([s["table"].double(), torch.full((1, case["heads"]), -math.inf, dtype=torch.float64, device="cuda")])
        for b in range(out.shape[0]):
            line = table[torch.tensor(every[b], device="cuda")].t().contiguous()     # [heads, diagonals]
            out[b] = line.unfold(1, keys, 1).flip(1)                                # a query sees one diagonal less
            if case["add"]:
                out[b] += s["scores"][b].double()
        return out
    if batch * (queries + keys) > 200_000:
        return None
    total = torch.zeros((case["buckets"], case["heads"]), dtype=torch.float64, device="cuda")
    shared = [(range(batch), every[0])] if not case["ragged"] else [([b], every[b]) for b in range(batch)]
    for which, buckets in shared:
        g = torch.zeros(s["scores"].shape[1:], dtype=torch.float64, device="cuda")
        for b in which:
            g += s["scores"][b].double()
        for k, bucket in enumerate(buckets):
            if bucket >= 0:
                total[bucket] += g.diagonal(k + 1 - queries, 1, 2).sum(1)
    return total


def exact(case, seed):
    global own
    kept, own = own, False  # the inputs alone
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    return _exact_logits(case, s) if "rows" in case else _exact_scores(case, s)
