"""Token-embedding lookups, their gradients, and the global norm of gradients with clipping, for timing their calls.

A case is one call as a program makes it: a lookup of token ids in a table that HBM holds (`lookup`), the gradient of a
lookup for the whole table (`dense`) or as its distinct rows (`rows`, of tokens or of pooled bags), the norm of many
gradients and their clipping (`clip`).  Token ids follow a bounded Zipf law over permuted rows, as words of a text or
ids of a feature do.  With `own` false the calls are written out in elementary torch operations, in 32 bits, rounded
once; with `own` true they are the package's.  Inputs come from the seed alone.
"""
import functools
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "i32": 4, "i64": 8}
EPS = 1e-6


def _ids(op, name, **kw):
    """A case over token ids.  `shards`: the table is one of so many parts of the vocabulary (the middle one), other
    parts' tokens lie outside it.  `pad`: share of the ids that fill up short sequences (in runs at their ends);
    `pad_id`: "out" (-1, no row of the table) or "row" (row 0, a row without a gradient).  `bags`: pooled lookups, of
    n / bags ids on average."""
    c = dict(op=op, name=name, n=1, rows=1, dim=1, ids="i64", alpha=1.0, shards=1, pad=0.0, pad_id="out", bags=0, scale=1.0,
             given="bf16", result="bf16", accumulate=False)
    assert set(kw) <= set(c)
    return {**c, **kw}


def _clip(name, **kw):
    """A case over gradients.  `limit`: max_norm over the gradients' norm; `place`: "in" (the gradients themselves) or
    "out" (clipped copies, `result` their type)."""
    c = dict(op="clip", name=name, tensors=1, total=1, given="bf16", result="bf16", place="out", limit=0.5)
    assert set(kw) <= set(c)
    return {**c, **kw}


def listed():
    return [
        # the next token of four running sequences: a serving step waits for it
        _ids("lookup", "decode lookup", n=4, rows=50_000, dim=4096, scale=64.0),
        # a prompt whose length is no round number, scaled by the root of the width
        _ids("lookup", "prompt lookup", n=8_191, rows=100_003, dim=2048, ids="i32", scale=math.sqrt(2048)),
        # a training batch of long sequences
        _ids("lookup", "batch lookup", n=131_072, rows=128_000, dim=4096),
        # one of four parts of a vocabulary, fp32 rows of odd width into bf16 activations
        _ids("lookup", "vocabulary part lookup", n=16_384, rows=25_001, dim=1001, shards=4, given="f32"),
        # a short fine-tuning step on a small fp32 table
        _ids("dense", "short step gradient", n=384, rows=10_000, dim=256, given="f32", result="f32"),
        # a micro-batch of padded sequences into the fp32 gradient that several of them share
        _ids("dense", "micro-batch gradient", n=8_192, rows=100_000, dim=2048, pad=0.2, scale=math.sqrt(2048), result="f32",
             accumulate=True),
        # the gradient of a large batch for a large table, written whole
        _ids("dense", "batch gradient", n=65_536, rows=128_000, dim=4096),
        # pooled lookups of a table that only host memory holds (one table of the eight-table configuration): its rows'
        # gradients go back there
        _ids("rows", "pooled rows gradient", n=81_920, rows=1_000_000, dim=128, ids="i32", alpha=1.1, bags=2048, given="f32",
             result="f32"),
        # rows of a token batch whose short sequences are filled up with a row that has no gradient
        _ids("rows", "token rows gradient", n=4_099, rows=250_007, dim=1024, pad=0.3, pad_id="row", given="f16", result="f32"),
        # a small model's gradients, most of them short
        _clip("small model clipping", tensors=62, total=2_000_000, given="f32", result="f32"),
        # a step whose gradients stay within the limit: their norm is what it costs
        _clip("norm within the limit", tensors=290, total=400_000_000, place="in", limit=2.0),
        # clipped fp32 copies of bf16 gradients, as an optimizer takes them
        _clip("clipping into fp32", tensors=150, total=300_000_000, result="f32"),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["lookup", "lookup", "dense", "dense", "rows", "clip"])
    kinds = ["bf16", "f16", "f32"]
    if op == "clip":
        given = rng.choice(kinds)
        place = rng.choice(["in", "out"])
        return _drawn(_clip("", tensors=size(1, 400), total=size(20_000, 200_000_000), given=given,
                            result=given if place == "in" else rng.choice([given, "f32"]), place=place,
                            limit=2.0 if place == "in" else rng.choice([0.1, 0.5, 2.0])))
    n, dim, rows = size(1, 60_000), size(16, 4096), size(1_000, 120_000)
    if rng.random() < 0.6:
        dim = max(16, dim // 64 * 64)
    c = _ids(op, "", n=n, dim=dim, rows=rows, ids=rng.choice(["i32", "i64"]), alpha=rng.choice([0.8, 1.0, 1.2]),
             scale=rng.choice([1.0, math.sqrt(dim)]), given=rng.choice(kinds), pad=rng.choice([0.0, 0.0, 0.1, 0.5]),
             pad_id=rng.choice(["out", "row"]), shards=rng.choice([1, 1, 2, 8]))
    c["result"] = rng.choice([c["given"], "f32", "bf16"]) if op == "lookup" else rng.choice([c["given"], "f32"])
    if op == "dense":
        c["accumulate"] = c["result"] == "f32" and rng.random() < 0.5
        c["rows"] = size(1_000, 50_000 if c["result"] == "f32" else 100_000)
    if op == "rows":
        c["result"] = "f32"
        c["rows"] = size(1_000, 2_000_000)
        n = c["n"] = min(n, 100_000_000 // dim)
        if rng.random() < 0.5:
            c["bags"] = max(1, n // size(1, 60))
    return _drawn(c)


def _drawn(c):
    del c["name"]
    return c


# ---------------------------------------------------------------------------- inputs


@functools.lru_cache(maxsize=8)
def _zipf(rows, alpha):
    """Cumulative probabilities of a bounded Zipf law."""
    p = np.arange(1, rows + 1, dtype=np.float64) ** -alpha
    return np.cumsum(p / p.sum())


def _sizes(c):
    """Element counts of a model's gradients: from a few to most of the total, few of them round."""
    r = random.Random(c["tensors"] * 1_000_003 + c["total"])
    w = [10.0 ** r.uniform(0, 4) for _ in range(c["tensors"])]
    return [max(1, int(c["total"] * x / sum(w))) for x in w]


def _views(flat, sizes):
    """The tensors of `sizes`, one after another in `flat`, each from a multiple of 64 elements."""
    at, got = 0, []
    for n in sizes:
        got.append(flat[at:at + n])
        at += (n + 63) // 64 * 64
    return got


def prepare(case, seed):
    c = case
    dev = torch.device("cuda", 0)
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    if c["op"] == "clip":
        sizes = _sizes(c)
        room = sum((n + 63) // 64 * 64 for n in sizes)
        flat = torch.zeros(room, dtype=DTYPES[c["given"]], device=dev)
        grads = _views(flat, sizes)
        for g in grads:
            g.normal_(0.0, 1e-3, generator=gen)
        into = flat if c["place"] == "in" else torch.zeros(room, dtype=DTYPES[c["result"]], device=dev)
        s = dict(case=c, grads=grads, outs=_views(into, sizes), into=into,
                 max_norm=c["limit"] * 1e-3 * math.sqrt(sum(sizes)))
        if own:  # the list of gradient tensors that a training program keeps from step to step
            from paper_2511_08568_amd import GradientList
            s["list"] = GradientList(grads) if c["place"] == "in" else GradientList(grads, out=s["outs"])
        return s
    whole = c["rows"] * c["shards"]
    first = c["rows"] * (c["shards"] // 2)
    cum = torch.from_numpy(_zipf(whole, c["alpha"])).to(dev)
    u = torch.rand(c["n"], generator=gen, device=dev, dtype=torch.float64)
    at = torch.searchsorted(cum, u).clamp_(max=whole - 1)
    tokens = torch.randperm(whole, generator=gen, device=dev)[at]
    if c["pad"] > 0:  # sequences of 64 places, each filled up behind its own end
        place = torch.arange(c["n"], device=dev)
        ends = torch.rand(c["n"] // 64 + 1, generator=gen, device=dev) * 2 * c["pad"]
        tokens = torch.where(place % 64 >= 64 * (1 - ends[place // 64]), -1 if c["pad_id"] == "out" else first, tokens)
    tokens = tokens.to(torch.int32 if c["ids"] == "i32" else torch.int64)
    s = dict(case=c, tokens=tokens, first=first, scale=c["scale"],
             padding=first if c["pad"] > 0 and c["pad_id"] == "row" else None,
             partly=c["shards"] > 1 or (c["pad"] > 0 and c["pad_id"] == "out"))
    given, result = DTYPES[c["given"]], DTYPES[c["result"]]
    if c["op"] == "lookup":
        s["table"] = torch.empty(c["rows"], c["dim"], dtype=given, device=dev).normal_(0.0, 0.02, generator=gen)
        return s
    s["offsets"] = None
    m = c["n"]
    if c["bags"]:
        m = c["bags"]
        cuts = torch.randint(0, c["n"] + 1, (m - 1,), generator=gen, device=dev).sort().values
        s["offsets"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), c["n"])])
    s["grad_out"] = torch.empty(m, c["dim"], dtype=given, device=dev).normal_(0.0, 1e-2, generator=gen)
    if c["op"] == "dense":
        s["grad"] = torch.empty(c["rows"], c["dim"], dtype=result, device=dev).normal_(0.0, 1e-2, generator=gen)
    else:
        cap = min(c["n"], c["rows"])
        s["rows"] = torch.full((cap,), -1, dtype=torch.int32, device=dev)
        s["values"] = torch.zeros(cap, c["dim"], dtype=result, device=dev)
        s["count"] = torch.zeros(1, dtype=torch.int64, device=dev)
    return s


# ---------------------------------------------------------------------------- one pass


def run(state):
    s = state
    op = s["case"]["op"]
    if own:
        return _OWN[op](s)
    return _PLAIN[op](s)


def _own_lookup(s):
    from paper_2511_08568_amd import embedding_forward
    return embedding_forward(s["table"], s["tokens"], scale=s["scale"], first_row=s["first"], out_dtype=DTYPES[s["case"]["result"]])


def _own_dense(s):
    from paper_2511_08568_amd import embedding_backward
    c = s["case"]
    return embedding_backward(s["grad_out"], s["tokens"], c["rows"], scale=s["scale"], first_row=s["first"],
                              padding_token=s["padding"], grad=s["grad"], accumulate=c["accumulate"])


def _own_rows(s):
    from paper_2511_08568_amd import embedding_backward_rows
    return embedding_backward_rows(s["grad_out"], s["tokens"], s["case"]["rows"], offsets=s["offsets"], scale=s["scale"],
                                   first_row=s["first"], padding_token=s["padding"], out=(s["rows"], s["values"], s["count"]))


def _own_clip(s):
    from paper_2511_08568_amd import clip_grad_norm
    return clip_grad_norm(s["list"], s["max_norm"], eps=EPS), s["into"]


def _plain_lookup(s):
    t = s["tokens"].long()
    if not s["partly"]:
        return (s["table"].index_select(0, t - s["first"]).float() * s["scale"]).to(DTYPES[s["case"]["result"]])
    t = t - s["first"]
    here = (t >= 0) & (t < s["case"]["rows"])
    x = s["table"].index_select(0, torch.where(here, t, 0)).float() * s["scale"]
    return torch.where(here[:, None], x, 0.0).to(DTYPES[s["case"]["result"]])


def _plain_targets(s):
    """The gradient row of each id, `rows` for ids that have none."""
    t = s["tokens"].long() - s["first"]
    rows = s["case"]["rows"]
    if s["partly"]:
        t = torch.where((t >= 0) & (t < rows), t, rows)
    if s["padding"] is not None:
        t = torch.where(s["tokens"] == s["padding"], rows, t)
    return t


def _plain_per_id(s):
    g = s["grad_out"].float()
    if s["offsets"] is None:
        return g
    lengths = s["offsets"][1:] - s["offsets"][:-1]
    bag = torch.repeat_interleave(torch.arange(lengths.numel(), device=g.device), lengths, output_size=s["case"]["n"])
    return g.index_select(0, bag)


def _plain_dense(s):
    c = s["case"]
    sums = torch.zeros(c["rows"] + 1, c["dim"], device=s["grad"].device)
    sums.index_add_(0, _plain_targets(s), _plain_per_id(s))
    sums = sums[:c["rows"]]
    return s["grad"].add_(sums * s["scale"]) if c["accumulate"] else s["grad"].copy_(sums * s["scale"])


def _plain_rows(s):
    c = s["case"]
    found, at = torch.unique(_plain_targets(s), return_inverse=True)
    sums = torch.zeros(found.numel(), c["dim"], device=s["values"].device)
    sums.index_add_(0, at, _plain_per_id(s))
    there = found < c["rows"]
    k = int(there.sum())
    s["rows"][:k] = found[:k].to(torch.int32)
    s["values"][:k] = sums[:k] * s["scale"]
    s["count"].fill_(k)
    return s["rows"], s["values"], s["count"]


def _plain_clip(s):
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    c = (s["max_norm"] / (norm + EPS)).clamp(max=1.0)
    [o.copy_(g.float() * c) for g, o in zip(s["grads"], s["outs"])]
    return norm, s["into"]


_OWN = {"lookup": _own_lookup, "dense": _own_dense, "rows": _own_rows, "clip": _own_clip}
_PLAIN = {"lookup": _plain_lookup, "dense": _plain_dense, "rows": _plain_rows, "clip": _plain_clip}


# ---------------------------------------------------------------------------- what a pass cannot do without


def _seen(c):
    """(ids that have a row here, distinct rows among them), as expected from the Zipf law."""
    p = np.diff(_zipf(c["rows"] * c["shards"], c["alpha"]), prepend=0.0)
    n = c["n"] * (1 - c["pad"])
    return n / c["shards"], float(-np.expm1(n * np.log1p(-np.minimum(p, 1 - 1e-12))).sum()) / c["shards"]


def work(case):
    c = case
    if c["op"] == "clip":
        n = sum(_sizes(c))
        write = SIZE[c["result"]] if c["place"] == "out" else 0
        return {"bytes": n * (SIZE[c["given"]] + write) + 4, "flops": n * (3 if write else 2)}
    hits, distinct = _seen(c)
    ids = c["n"] * SIZE[c["ids"]]
    row, res = c["dim"] * SIZE[c["given"]], c["dim"] * SIZE[c["result"]]
    if c["op"] == "lookup":
        return {"bytes": ids + distinct * row + c["n"] * res, "flops": hits * c["dim"]}
    given = (c["bags"] or hits) * row + c["bags"] * 8
    if c["op"] == "rows":
        return {"bytes": ids + given + distinct * (4 + res), "flops": hits * c["dim"]}
    return {"bytes": ids + given + (2 * distinct if c["accumulate"] else c["rows"]) * res, "flops": hits * c["dim"]}


# ---------------------------------------------------------------------------- in 64 bits, from the definitions


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "clip":
        squares = sum(float(torch.linalg.vector_norm(g, dtype=torch.float64)) ** 2 for g in s["grads"])
        factor = min(1.0, s["max_norm"] / (math.sqrt(squares) + EPS))
        return torch.tensor(math.sqrt(squares), dtype=torch.float64), _whole(s).mul_(factor)
    ids = s["tokens"].to(torch.int64)
    inside = (ids >= s["first"]) & (ids < s["first"] + c["rows"])
    if c["op"] == "lookup":
        out = torch.zeros(c["n"], c["dim"], dtype=torch.float64, device=ids.device)
        which = inside.nonzero()[:, 0]
        out[which] = s["table"][ids[which] - s["first"]].double() * s["scale"]
        return out
    if s["padding"] is not None:
        inside &= ids != s["padding"]
    which = inside.nonzero()[:, 0]
    source = which if s["offsets"] is None else torch.searchsorted(s["offsets"], which, right=True) - 1
    g = s["grad_out"].double()[source] * s["scale"]
    if c["op"] == "dense":
        total = s["grad"].double() if c["accumulate"] else torch.zeros(c["rows"], c["dim"], dtype=torch.float64, device=ids.device)
        return total.scatter_add_(0, (ids[which] - s["first"])[:, None].expand(-1, c["dim"]), g)
    present = torch.zeros(c["rows"], dtype=torch.int64, device=ids.device)
    present[ids[which] - s["first"]] = 1
    number = present.cumsum(0) - 1
    k = int(present.sum())
    values = torch.zeros(s["values"].shape, dtype=torch.float64, device=ids.device)
    values.scatter_add_(0, number[ids[which] - s["first"]][:, None].expand(-1, c["dim"]), g)
    s["rows"][:k] = present.nonzero()[:, 0].to(torch.int32)
    return s["rows"], values, s["count"].fill_(k)


def _whole(s):
    """The buffer that `into` is, holding the gradients in 64 bits."""
    flat = torch.zeros(s["into"].shape, dtype=torch.float64, device=s["into"].device)
    for g, v in zip(s["grads"], _views(flat, [g.numel() for g in s["grads"]])):
        v.copy_(g)
    return flat
