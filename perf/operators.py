"""The operators beside the tensor-train table whose speed matters, as cases that can be timed.

A case names an operator (`op`) and its sizes:

  lookup    rows of a plain table [rows, dim] by id, times a scale; ids outside the table give zeros
  gradient  the table's gradient: the scaled sum of the rows' gradients of every id, all table rows written;
            with `micro` = 2, two micro-batches, the second added to the gradient of the first
  norm      the 2-norm over all values of many tensors
  clip      that norm, and the tensors scaled down to a largest norm (in place or into another buffer)

Table heights, widths and batches are the node tables of `workloads.CONFIGS` kept as plain matrices (136^3 x 128,
56^3 x 64, 125*140*140 x 100) and generic vocabularies of language models; batches of one to 200,000 ids.
Ids are uniform, or log-uniform in their rank, which is Zipf's law of exponent one: `zipf` with the rank
as the id, as in a vocabulary ordered by frequency, `spread` with ranks mapped over the table, as in a graph.
`pad` is the share of positions that hold no id (-1), `hot` the share that holds one and the same id.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


def _lookup(name, rows, dim, batch, kind, out_kind, ids, scale=1.0, pad=0.0, gap=0):
    c = {"op": "lookup", "rows": rows, "dim": dim, "batch": batch, "type": kind, "out": out_kind, "ids": ids,
         "scale": scale, "pad": pad, "hot": 0.0, "gap": gap}
    return dict(c, name=name) if name else c


def _gradient(name, rows, dim, batch, kind, out_kind, ids, scale=1.0, pad=0.0, hot=0.0, micro=1, gap=0):
    c = {"op": "gradient", "rows": rows, "dim": dim, "batch": batch, "type": kind, "out": out_kind, "ids": ids,
         "scale": scale, "pad": pad, "hot": hot, "micro": micro, "gap": gap}
    return dict(c, name=name) if name else c


def _tensors(name, op, count, values, kinds, out="", scale=1.0, clipped=True):
    c = {"op": op, "count": count, "values": values, "types": kinds, "out": out, "scale": scale, "clipped": clipped}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one sequence decoding: the row of its latest token
        _lookup("lookup_token", 32_000, 2048, 1, "bf16", "bf16", "zipf", scale=math.sqrt(2048)),
        # a prefill or training batch of 16,384 tokens of a large vocabulary
        _lookup("lookup_prompt", 128_000, 4096, 16_384, "bf16", "bf16", "zipf", scale=64.0),
        # a sampled minibatch of ogbn-products' nodes, width 100, some places empty, written into the left part
        # of a wider feature matrix
        _lookup("lookup_nodes", 125 * 140 * 140, 100, 200_000, "fp32", "fp32", "spread", pad=0.03, gap=28),
        # fine-tuning on one short text
        _gradient("gradient_short", 32_000, 512, 129, "bf16", "bf16", "zipf", scale=math.sqrt(512)),
        # pre-training: 16,384 tokens, a large vocabulary, all in bf16
        _gradient("gradient_prompt", 128_000, 4096, 16_384, "bf16", "bf16", "zipf", scale=64.0),
        # two micro-batches accumulated in fp32
        _gradient("gradient_micro", 32_000, 2048, 8192, "bf16", "fp32", "zipf", micro=2),
        # the benchmark's node table (136^3 x 128) kept plain, its degree-skewed batch of 200,000
        _gradient("gradient_nodes", 136 ** 3, 128, 200_000, "fp32", "fp32", "spread"),
        # odd width, half of the batch padding, one token in a fifth of the rest's places
        _gradient("gradient_ragged", 50_257, 1001, 5003, "fp16", "fp16", "zipf", pad=0.5, hot=0.2),
        # the gradients of a small model: a few short tensors, where launches and host time count
        _tensors("norm_small", "norm", 7, 60_000, "fp32"),
        # gradients of 300 layers' weights and biases in two types, as they come from mixed precision
        _tensors("norm_model", "norm", 300, 400_000_000, "mixed"),
        # a step whose norm stays below the limit: in place, nothing to scale
        _tensors("clip_within", "clip", 40, 3_200_000, "fp32", clipped=False),
        # bf16 gradients of a model, unscaled and clipped into the optimiser's fp32 buffer
        _tensors("clip_model", "clip", 300, 300_000_000, "bf16", out="fp32", scale=1.0 / 128),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


# a drawn case moves no more than the largest listed one (clip_model)
_BYTES_MOST = 1.8e9


def _drawn(rng):
    op = rng.choice(["lookup", "lookup", "gradient", "gradient", "gradient", "norm", "clip"])
    if op in ("norm", "clip"):
        count, values = round(_log_uniform(rng, 1, 400)), round(_log_uniform(rng, 1000, 4e8))
        kinds = rng.choice(["fp32", "bf16", "fp16", "mixed"])
        if op == "norm":
            return _tensors("", op, count, values, kinds, scale=rng.choice([1.0, 1.0 / 64]))
        clipped = rng.random() < 0.7
        out = rng.choice(["fp32", "same"]) if clipped else ""
        return _tensors("", op, count, values, kinds, out=out, scale=rng.choice([1.0, 1.0 / 64]) if clipped else 1.0,
                        clipped=clipped)
    dim = round(_log_uniform(rng, 8, 8192))
    dim = dim // 16 * 16 + 8 if rng.random() < 0.6 else dim | 1  # whole 16-byte pieces, or odd
    rows = round(_log_uniform(rng, 1000, 2_600_000)) | 1
    batch = round(_log_uniform(rng, 1, 200_000)) | 1
    kind = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    out = rng.choice(["fp32", kind])
    ids = rng.choice(["uniform", "zipf", "zipf", "spread"])
    scale = rng.choice([1.0, math.sqrt(dim)])
    pad, gap = rng.choice([0.0, 0.0, 0.1, 0.6]), rng.choice([0, 0, 0, 1, 24])
    if op == "lookup":
        return _lookup("", rows, dim, batch, kind, out, ids, scale, pad, gap)
    micro = 2 if out == "fp32" and rng.random() < 0.3 else 1
    return _gradient("", rows, dim, batch, kind, out, ids, scale, pad, rng.choice([0.0, 0.0, 0.1, 0.5]), micro, gap)


def draw(rng):
    while True:
        c = _drawn(rng)
        held = 0
        if c["op"] in ("lookup", "gradient"):
            held = c["rows"] * c["dim"] * _BYTES[c["type"] if c["op"] == "lookup" else c["out"]]
        if max(work(c)["bytes"], held) <= _BYTES_MOST:
            return c


# ---- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _ids(case, g):
    rows, batch = case["rows"], case["batch"]
    u = torch.rand(batch, generator=g, device="cuda", dtype=torch.float64)
    if case["ids"] == "uniform":
        ids = (u * rows).long()
    else:
        ids = (torch.exp(u * math.log(rows + 1)).long() - 1)
    ids = ids.clamp_(0, rows - 1)
    if case["ids"] == "spread":
        step = 1_000_003
        while math.gcd(step, rows) != 1:
            step += 2
        ids = ids * step % rows
    for share, value in ((case["hot"], rows // 2), (case["pad"], -1)):
        if share:
            ids[torch.rand(batch, generator=g, device="cuda") < share] = value
    return ids


def _normal(shape, kind, g, scale=1.0, gap=0):
    """Normal values; gap: unused columns behind every row."""
    x = torch.empty((shape[0], shape[1] + gap), dtype=_TYPES[kind], device="cuda")
    x.normal_(0.0, scale, generator=g)
    return x[:, :shape[1]]


def _sizes(case):
    """(values, type) of every tensor of a model: matrices and short vectors, and now and then an empty tensor."""
    rng = random.Random(case["count"] * 1_000_003 + case["values"])
    weights = [math.exp(rng.uniform(-1.0, 0.0) - (rng.random() < 0.4) * 7.0) for _ in range(case["count"])]
    total = sum(weights)
    kinds = [rng.choice(["fp32", "bf16"]) if case["types"] == "mixed" else case["types"] for _ in weights]
    return [(int(case["values"] * w / total), k) for w, k in zip(weights, kinds)]


def _views(flat, sizes):
    """Tensors of the given sizes, one behind the other in the flat buffers of their types."""
    at, found = {k: 0 for k in flat}, []
    for n, k in sizes:
        found.append(flat[k][at[k]:at[k] + n])
        at[k] += n
    return found


def _flat(sizes):
    return {k: torch.empty(sum(n for n, t in sizes if t == k), dtype=_TYPES[k], device="cuda")
            for k in sorted({t for _, t in sizes})}


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["op"] == "lookup":
        s["table"] = _normal((case["rows"], case["dim"]), case["type"], g, 0.02)
        s["ids"] = _ids(case, g)
        wide = torch.empty((case["batch"], case["dim"] + case["gap"]), dtype=_TYPES[case["out"]], device="cuda")
        s["rows"] = wide[:, :case["dim"]]
    elif case["op"] == "gradient":
        s["table"] = _normal((case["rows"], case["dim"]), case["out"], g, 0.02)
        s["ids"] = [_ids(case, g) for _ in range(case["micro"])]
        s["grads"] = [_normal((case["batch"], case["dim"]), case["type"], g, 0.05, case["gap"])
                      for _ in range(case["micro"])]
        s["sum"] = torch.empty_like(s["table"])
    else:
        sizes = _sizes(case)
        s["flat"] = _flat(sizes)
        for x in s["flat"].values():
            x.normal_(0.0, 1e-2, generator=g)
        s["grads"] = _views(s["flat"], sizes)
        # every layer has gradients of its own size
        spread = (2.0 ** torch.randint(-3, 4, (len(sizes),), generator=g, device="cuda")).tolist()
        for x, f in zip(s["grads"], spread):
            x.mul_(f)
        typical = 1e-2 * 3.0 * abs(case["scale"]) * math.sqrt(max(1, case["values"]))
        s["max_norm"] = typical * (0.1 if case["clipped"] else 100.0)
        s["clipped"] = None
        if case["op"] == "clip" and case["out"]:
            outs = [(n, k if case["out"] == "same" else case["out"]) for n, k in sizes]
            s["flat_out"] = _flat(outs)
            s["clipped"] = _views(s["flat_out"], outs)
    if own:
        import paper_2206_10581_amd as tt
        if case["op"] in ("lookup", "gradient"):
            s["own"] = tt.DenseEmbedding(s["table"], case["batch"], scale=case["scale"])
        else:
            s["own"] = tt.GradientClip(s["grads"], out=s["clipped"])
    return s


# ---- one pass

def _plain_lookup(s):
    case, table, ids = s["case"], s["table"], s["ids"]
    inside = (ids >= 0) & (ids < table.shape[0])
    rows = table[torch.where(inside, ids, 0)].float() * case["scale"]
    s["rows"].copy_(torch.where(inside[:, None], rows, 0.0))
    return s["rows"]


def _plain_gradient(s):
    case, table = s["case"], s["table"]
    ids, grads = torch.cat(s["ids"]), torch.cat(s["grads"])
    inside = (ids >= 0) & (ids < table.shape[0])
    rows = torch.where(inside[:, None], grads.float() * case["scale"], 0.0)
    total = torch.zeros(table.shape, dtype=torch.float32, device="cuda")
    total.index_add_(0, torch.where(inside, ids, 0), rows)
    s["sum"].copy_(total)
    return s["sum"]


def _plain_norm(s):
    return torch.stack([x.float().square().sum() for x in s["grads"]]).sum().sqrt() * abs(s["case"]["scale"])


def _plain_clip(s):
    norm = _plain_norm(s)
    factor = torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0) * s["case"]["scale"]
    outs = s["clipped"] if s["clipped"] is not None else s["grads"]
    [y.copy_(x.float() * factor) for x, y in zip(s["grads"], outs)]
    return norm


def run(state):
    case = state["case"]
    if case["op"] == "lookup":
        return state["own"].forward(state["ids"], out=state["rows"]) if own else _plain_lookup(state)
    if case["op"] == "gradient":
        if not own:
            return _plain_gradient(state)
        for k, (ids, grads) in enumerate(zip(state["ids"], state["grads"])):
            state["own"].backward(ids, grads, out=state["sum"], add=k > 0)
        return state["sum"]
    if case["op"] == "norm":
        return state["own"].norm(scale=case["scale"]) if own else _plain_norm(state)
    if own:
        norm = state["own"].clip(state["max_norm"], scale=case["scale"])
    else:
        norm = _plain_clip(state)
    return [norm, state["flat_out"] if state["clipped"] is not None else state["flat"]]


# ---- what a pass cannot do without

def _distinct(case):
    """Distinct ids that a batch is expected to hold."""
    held = case["batch"] * (1.0 - case["pad"]) * (1.0 - case["hot"])
    if case["ids"] == "uniform":
        return case["rows"] * -math.expm1(held * math.log1p(-1.0 / case["rows"]))
    k = np.arange(1, case["rows"] + 1, dtype=np.float64)
    return float((-np.expm1(held * np.log1p(-np.log1p(1.0 / k) / math.log(case["rows"] + 1)))).sum())


def work(case):
    if case["op"] in ("lookup", "gradient"):
        rows, dim, batch = case["rows"], case["dim"], case["batch"]
        valid = batch * (1.0 - case["pad"])
        if case["op"] == "lookup":
            moved = 8 * batch + _distinct(case) * dim * _BYTES[case["type"]] + batch * dim * _BYTES[case["out"]]
            return {"bytes": moved, "flops": valid * dim}
        moved = case["micro"] * (8 * batch + valid * dim * _BYTES[case["type"]]) + rows * dim * _BYTES[case["out"]]
        return {"bytes": moved, "flops": 2 * case["micro"] * valid * dim}
    sizes = _sizes(case)
    moved = sum(n * _BYTES[k] for n, k in sizes) + 4
    flops = 2 * sum(n for n, _ in sizes)
    if case["op"] == "clip" and case["clipped"]:
        moved += sum(n * _BYTES[k if case["out"] == "same" else case["out"]] for n, k in sizes)
        flops += sum(n for n, _ in sizes)
    return {"bytes": moved, "flops": flops}


# ---- the definitions in 64 bits

def exact(case, seed):
    global own
    kept, own = own, False  # the inputs alone
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    if case["op"] == "lookup":
        padded = torch.cat([s["table"].double(), torch.zeros(1, case["dim"], dtype=torch.float64, device="cuda")])
        outside = (s["ids"] < 0) | (s["ids"] >= case["rows"])
        return padded.index_select(0, s["ids"].masked_fill(outside, case["rows"])).mul_(case["scale"])
    if case["op"] == "gradient":
        total = torch.zeros(case["rows"], case["dim"], dtype=torch.float64, device="cuda")
        for ids, grads in zip(s["ids"], s["grads"]):
            kept = torch.nonzero((ids >= 0) & (ids < case["rows"]))[:, 0]
            total.index_put_((ids[kept],), grads[kept].double(), accumulate=True)
        return total.mul_(case["scale"])
    squares = torch.zeros((), dtype=torch.float64, device="cuda")
    for x in s["flat"].values():
        for part in x.split(1 << 26):
            part = part.double()
            squares += (part * part).sum()
    norm = squares.sqrt() * abs(case["scale"])
    if case["op"] == "norm":
        return norm
    factor = min(1.0, s["max_norm"] / (float(norm) + 1e-6)) * case["scale"]
    if s["clipped"] is None:
        return [norm, {k: x.double() * factor for k, x in s["flat"].items()}]
    whole = {k: torch.empty(x.shape, dtype=torch.float64, device="cuda") for k, x in s["flat_out"].items()}
    outs = [(y.numel(), next(k for k, t in _TYPES.items() if t == y.dtype)) for y in s["clipped"]]
    for x, y in zip(s["grads"], _views(whole, outs)):
        y.copy_(x.double() * factor)
    return [norm, whole]
