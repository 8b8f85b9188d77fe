"""Dropout of the replicas' weights and balance of a model's experts: the cases that these operators are measured on.

  hand out  ws_unpack_dropout: the gathered weights go to the tensors of one or several replicas, each with a
            dropout mask of its own that a counter-based generator gives and nothing stores
  sum       ws_reduce_dropout: its adjoint, the replicas' gradients under the same masks, summed into the layout
            that ws_shard_update takes
  counts    ws_router_counts: how often the tokens of all replicas picked each expert, layer by layer
  balance   ws_balance_loss: the load-balancing loss over all replicas' tokens (and the z loss) with the
            gradient of the routers' logits

With `own` the calls are the library's; without, the same functions in elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _drop(name, op, family, lists, **kw):
    c = dict(name=name, op=op, family=family, lists=lists, shards=lists, width=0, layers=0, vocab=0, layout="per_tensor",
             align=32, flat="f32", tensors="f32", p=0.1, step=10, replica=0)
    c.update(kw)
    return c


def _router(name, op, layers, replicas, tokens, experts, topk, **kw):
    c = dict(name=name, op=op, layers=layers, replicas=replicas, tokens=tokens, experts=experts, topk=topk, ragged=False,
             index="i64", logits="f32", score="softmax", z=0.0)
    c.update(kw)
    return c


def listed():
    return [
        # a few tensors, 45 792 parameters, four replicas: latency
        _drop("hand out tiny", "hand out", "tiny", 4, width=128),
        # what one of 16 replicas of the 335 M encoder does after its all-gather of bf16 weights
        _drop("hand out encoder replica", "hand out", "encoder", 1, shards=16, width=1024, layers=24, vocab=30522, flat="bf16",
              tensors="bf16", replica=11),
        # the translation network's fp32 state to eight replicas' bf16 tensors: the ordinary step
        _drop("hand out translation", "hand out", "encdec", 8, width=1024, layers=6, vocab=33708, tensors="bf16"),
        # the gradients of the few tensors: latency
        _drop("sum tiny", "sum", "tiny", 4, width=128),
        # sizes that divide nothing, the concatenated layout, a bf16 sum for the wire
        _drop("sum ragged", "sum", "ragged", 3, width=611, layers=7, vocab=9973, layout="concat", flat="bf16", tensors="bf16", p=0.25),
        # the largest: four replicas' bf16 gradients of the 1.56 G decoder
        _drop("sum decoder", "sum", "decoder", 4, width=1600, layers=48, vocab=50257, tensors="bf16"),
        # one layer, one short batch: latency
        _router("counts small", "counts", 1, 1, 128, 8, 2),
        # a model's layers over eight replicas' batches of unequal length
        _router("counts step", "counts", 24, 8, 4096, 64, 2, ragged=True, index="i32"),
        # long sequences, many experts, eight picks a token: the most indices
        _router("counts long", "counts", 4, 8, 32768, 256, 8),
        # one layer, one short batch: latency
        _router("balance small", "balance", 1, 1, 128, 8, 2),
        # a model's layers over eight replicas' padded batches, bf16 logits, both losses
        _router("balance step", "balance", 24, 8, 4096, 64, 2, ragged=True, logits="bf16", z=1e-3),
        # long sequences, many experts, sigmoid scores: the most logits
        _router("balance long", "balance", 4, 8, 16384, 256, 8, score="sigmoid"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        if rng.random() < 0.5:
            family = rng.choice(["tiny", "encdec", "encoder", "decoder", "ragged"])
            width, layers, vocab = {
                "tiny": lambda: (_log_int(rng, 32, 1024), 0, 0),
                "encdec": lambda: (16 * _log_int(rng, 4, 64), rng.randint(1, 6), _log_int(rng, 1000, 34000)),
                "encoder": lambda: (16 * _log_int(rng, 4, 64), rng.randint(2, 24), _log_int(rng, 1000, 31000)),
                "decoder": lambda: (16 * _log_int(rng, 4, 100), rng.randint(2, 24), _log_int(rng, 1000, 51000)),
                "ragged": lambda: (_log_int(rng, 17, 1200), rng.randint(1, 8), _log_int(rng, 100, 20000)),
            }[family]()
            lists = rng.choice([1, 1, 2, 3, 4, 8, 16])
            c = _drop("", rng.choice(["hand out", "sum"]), family, lists, shards=rng.choice([1, 3, lists, 16, 64]), width=width,
                      layers=layers, vocab=vocab, layout=rng.choice(["per_tensor", "per_tensor", "concat"]), align=rng.choice([32, 32, 8]),
                      flat=rng.choice(["f32", "bf16"]), tensors=rng.choice(["f32", "bf16"]), p=round(rng.uniform(0.01, 0.6), 3),
                      step=rng.randint(0, 1 << 20), replica=rng.choice([0, rng.randint(0, 1000)]))
        else:
            experts, layers = rng.choice([_log_int(rng, 2, 300), 8, 16, 64, 128, 256]), rng.randint(1, 24)
            score = rng.choice(["softmax", "softmax", "sigmoid"])
            c = _router("", rng.choice(["counts", "balance"]), layers, rng.choice([1, 2, 3, 8, 16]), _log_int(rng, 1, 33000), experts,
                        min(experts, rng.choice([1, 2, 2, 4, 8])), ragged=rng.random() < 0.5, index=rng.choice(["i32", "i64"]),
                        logits=rng.choice(["f32", "bf16"]), score=score, z=rng.choice([0.0, 1e-3]) if score == "softmax" else 0.0)
        del c["name"]
        most = {"hand out": 4e9, "sum": 18e9, "counts": 6.8e7, "balance": 1.07e9}[c["op"]]
        if work(c)["bytes"] <= most and (c["op"] in ("counts", "balance") or c["lists"] * sum(_numels(c)) <= 3e9):
            return c


# ------------------------------------------------------------------ tensor lists
def _ragged(d, layers, vocab):
    s = [(vocab, d), (), (0, d)]
    for k in range(layers):
        s += [(d, 3 * d + k), (3 * d + k,), (d + 1, d), (d,), (3, 5, k + 1, d // 4 + 1), (k + 1,)]
    return s + [(d, vocab + 2), (vocab + 2,)]


def _shapes(c):
    d, layers, vocab = c["width"], c["layers"], c["vocab"]
    norm, ffn = [(d,), (d,)], [(d, 4 * d), (4 * d,), (4 * d, d), (d,)]
    attention, biased = [(d, d)] * 4, [(d, d), (d,)] * 4
    return {
        "tiny": lambda: [(64, d), (d,), (3, 3, 16, max(1, d // 4)), (max(1, d // 4),), (4 * d, 64), (64,)],
        "encdec": lambda: ([(vocab, d)] + layers * (attention + norm + ffn + norm) + norm
                           + layers * (attention + norm + attention + norm + ffn + norm) + norm),
        "encoder": lambda: [(vocab, d), (512, d), (2, d)] + norm + layers * (biased + norm + ffn + norm) + [(d, d), (d,)],
        "decoder": lambda: ([(vocab, d), (1024, d)] + layers * (norm + [(d, 3 * d), (3 * d,), (d, d), (d,)] + norm + ffn) + norm),
        "ragged": lambda: _ragged(d, layers, vocab),
    }[c["family"]]()


def _numels(c):
    return [math.prod(s) for s in _shapes(c)]


def _up(n, a):
    return (n + a - 1) // a * a


def _layout(c):
    """Where a tensor list lies: per tensor its start in a replica's arena (every start a multiple of 8 elements), its
    piece and its start in the sharded layout; the arena's length and a shard's."""
    numels, a, r = _numels(c), c["align"], c["shards"]
    concat = c["layout"] == "concat"
    arena, piece, off, at, pos = [], [], [], 0, 0
    for n in numels:
        p = _up(n, a) if concat else _up((n + r - 1) // r, a)
        arena.append(at)
        piece.append(p)
        off.append(pos)
        at, pos = at + _up(n, 8), pos + p
    return numels, arena, piece, off, at, _up((pos + r - 1) // r, a) if concat else pos


# ------------------------------------------------------------------------ inputs
def _gen(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1_000_003 + k * 10_007 + 29) & 0x7FFFFFFF)
    return g


def _normal(shape, std, gen, dtype=torch.float32):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=gen).to(dtype)


def _prepare_drop(c, seed):
    numels, arena, piece, off, length, shard = _layout(c)
    i64 = lambda v: torch.tensor(v, dtype=torch.int64, device="cuda")  # noqa: E731
    s = {"case": c, "numels": i64(numels), "arena": i64(arena), "piece": i64(piece), "off": i64(off), "length": length, "shard": shard,
         "seed": seed * 0x9E3779B1 + 7}
    flat, lists = c["shards"] * shard, c["lists"]
    if c["op"] == "hand out":
        s["flat"] = _normal(flat, 0.02, _gen(seed, 1), _DTYPE[c["flat"]])
        s["lists"] = torch.zeros(lists, length, dtype=_DTYPE[c["tensors"]], device="cuda")
    else:
        s["flat"] = torch.empty(flat, dtype=_DTYPE[c["flat"]], device="cuda")
        s["lists"] = torch.empty(lists, length, dtype=_DTYPE[c["tensors"]], device="cuda")
        for k in range(lists):
            s["lists"][k] = _normal(length, 1e-3, _gen(seed, 10 + k))
    if own:      # what a program makes once: the plan and the table of its tensors
        from paper_2004_13336_b200 import binding as ws
        s["plan"] = ws.Plan(_shapes(c), c["shards"], c["align"], layout=c["layout"], one_launch=False)
        s["table"] = ws.TensorTable(s["plan"], [[t[o:o + n] for o, n in zip(arena, numels)] for t in s["lists"]])
    return s


def _rows(c):
    """Tokens of every replica."""
    n = c["tokens"]
    return [n - (k * n // 3) // c["replicas"] if c["ragged"] else n for k in range(c["replicas"])]


def _prepare_router(c, seed):
    rows, experts, topk = _rows(c), c["experts"], c["topk"]
    total, shape = sum(rows), (c["layers"], sum(rows))
    # every layer's router prefers some experts
    logits = _normal(shape + (experts,), 1.5, _gen(seed, 1)) + _normal((c["layers"], 1, experts), 1.0, _gen(seed, 2))
    picks = torch.topk(logits, topk, dim=-1).indices
    if c["ragged"]:          # a full expert refused some tokens
        picks = torch.where(torch.rand(picks.shape, device="cuda", generator=_gen(seed, 3)) < 0.05, -1, picks)
    s = {"case": c, "picks": picks.to({"i32": torch.int32, "i64": torch.int64}[c["index"]]).contiguous(),
         # the ends of padded sequences are no tokens
         "valid": torch.rand(total, device="cuda", generator=_gen(seed, 4)) < 0.9 if c["ragged"] else None,
         "counts": torch.zeros(c["layers"], experts + 1, dtype=torch.int64, device="cuda")}
    bounds = [0]
    for n in rows:
        bounds.append(bounds[-1] + n)
    cut = lambda t: [[layer[a:b] for a, b in zip(bounds, bounds[1:])] for layer in t]  # noqa: E731
    if c["op"] == "balance":
        s["logits"] = logits.to(_DTYPE[c["logits"]])
        s["dlogits"] = torch.empty_like(s["logits"])
        s["loss"] = torch.empty(c["layers"], 2, device="cuda")
        s["counts"] = _counts(s)
    if own:      # what a program makes once: the set of its routers' tensors and a workspace
        from paper_2004_13336_b200 import binding as ws
        valid = None if s["valid"] is None else [s["valid"][a:b] for a, b in zip(bounds, bounds[1:])]
        more = {} if c["op"] == "counts" else {"logits": cut(s["logits"]), "dlogits": cut(s["dlogits"]), "score": c["score"]}
        s["routers"] = ws.RouterSet(experts, cut(s["picks"]), valid=valid, **more)
        s["workspace"] = torch.empty(s["routers"].workspace_bytes(), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    return _prepare_drop(case, seed) if case["op"] in ("hand out", "sum") else _prepare_router(case, seed)


# -------------------------------------------------------------------- plain forms
def _threshold(p):
    """Of 65536 values of 16 random bits, those below it drop the element."""
    return min(int(math.floor(p * 65536 + 0.5)), 65535)


def _random_words(key, counter):
    """Philox4x32 with 7 rounds (Salmon, Moraes, Dror, Shaw 2011): four 32-bit words in int64 tensors from four counter words."""
    k0, k1 = key & 0xFFFFFFFF, key >> 32 & 0xFFFFFFFF
    c0, c1, c2, c3 = counter
    for _ in range(7):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & 0xFFFFFFFF) ^ c1 ^ k0, b & 0xFFFFFFFF, ((a >> 32) & 0xFFFFFFFF) ^ c3 ^ k1, a & 0xFFFFFFFF
        k0, k1 = k0 + 0x9E3779B9 & 0xFFFFFFFF, k1 + 0xBB67AE85 & 0xFFFFFFFF
    return c0, c1, c2, c3


def _blocks(s):
    """For every run of 8 elements of an arena: its tensor, its number in the tensor and its number in the sharded layout."""
    count = (s["numels"] + 7) // 8
    t = torch.repeat_interleave(torch.arange(len(count), device="cuda"), count, output_size=s["length"] // 8)
    j = torch.arange(s["length"] // 8, device="cuda") - (s["arena"] // 8)[t]
    if s["case"]["layout"] == "concat":
        return t, j, (s["off"] // 8)[t] + j
    per = (s["piece"] // 8)[t]
    return t, j, j // per * (s["shard"] // 8) + (s["off"] // 8)[t] + j % per


def _kept(s, k, t, j):
    """Which of 8 elements replica k keeps, for every run."""
    c = s["case"]
    replica = torch.full_like(j, c["replica"] + k)
    words = _random_words(s["seed"], (j & 0xFFFFFFFF, torch.full_like(j, c["step"]), t, replica + ((j >> 32) << 16)))
    halves = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=-1)
    return halves >= _threshold(c["p"])


def _there(s, t, j):
    """Which of 8 elements exist in the tensor."""
    return j[:, None] * 8 + torch.arange(8, device="cuda") < s["numels"][t][:, None]


def _hand_out(s):
    c = s["case"]
    t, j, at = _blocks(s)
    scaled = s["flat"].view(-1, 8)[at].float() * (65536.0 / (65536 - _threshold(c["p"])))
    scaled = torch.where(_there(s, t, j), scaled, 0.0)
    out = torch.empty_like(s["lists"])
    for k in range(c["lists"]):
        out[k] = torch.where(_kept(s, k, t, j), scaled, 0.0).view(-1)
    return out


def _sum(s):
    c = s["case"]
    t, j, at = _blocks(s)
    total = torch.zeros(len(t), 8, device="cuda")
    for k in range(c["lists"]):
        total += torch.where(_kept(s, k, t, j), s["lists"][k].view(-1, 8).float(), 0.0)
    total *= 65536.0 / (65536 - _threshold(c["p"]))
    flat = torch.zeros_like(s["flat"]).view(-1, 8)
    flat[at] = torch.where(_there(s, t, j), total, 0.0).to(flat.dtype)
    return flat.view(-1)


def _counts(s):
    c = s["case"]
    experts, picks = c["experts"], s["picks"].long()
    real = picks >= 0
    if s["valid"] is not None:
        real = real & s["valid"][:, None]
    counts = torch.zeros(c["layers"], experts + 1, dtype=torch.int64, device="cuda")
    counts.scatter_add_(1, torch.where(real, picks, experts).view(c["layers"], -1), torch.ones_like(picks).view(c["layers"], -1))
    counts[:, experts] = picks.shape[1] if s["valid"] is None else s["valid"].sum()
    return counts


def _balance(s, coef=1e-2):
    c, counts = s["case"], s["counts"]
    experts = c["experts"]
    x = s["logits"].float()
    tokens = counts[:, experts:].float().clamp(min=1)         # (no token at all: no loss)
    share = (counts[:, :experts].float() / (c["topk"] * tokens))[:, None]            # f
    if c["score"] == "softmax":
        top = x.amax(-1, keepdim=True)
        e = (x - top).exp()
        total = e.sum(-1, keepdim=True)
        p, lse = e / total, top + total.log()
    else:
        score = 1 / (1 + (-x).exp())
        p, lse = score / score.sum(-1, keepdim=True), x.new_zeros(x.shape[:-1] + (1,))
    inner = (p * share).sum(-1, keepdim=True)
    d = (coef * experts / tokens)[:, None] * p * (share - inner)
    if c["score"] == "softmax":
        d = d + (2 * c["z"] / tokens)[:, None] * lse * p
    else:
        d = d * (1 - score)
    if s["valid"] is not None:
        live = s["valid"][None, :, None]
        d, inner, lse = torch.where(live, d, 0.0), torch.where(live, inner, 0.0), torch.where(live, lse, 0.0)
    loss = torch.cat([coef * experts * inner.double().sum(1) / tokens, c["z"] * lse.double().square().sum(1) / tokens], 1).float()
    return {"loss": loss, "dlogits": d.to(s["dlogits"].dtype)}


# -------------------------------------------------------------------------- a pass
def run(s):
    c = s["case"]
    if not own:
        return {"hand out": _hand_out, "sum": _sum, "counts": _counts, "balance": _balance}[c["op"]](s)
    from paper_2004_13336_b200 import binding as ws
    if c["op"] == "hand out":
        ws.ws_unpack_dropout(s["plan"], -1, s["flat"], s["table"], ws.make_dropout(c["p"], s["seed"], c["step"], c["replica"]))
        return s["lists"]
    if c["op"] == "sum":
        ws.ws_reduce_dropout(s["plan"], -1, s["table"], ws.make_dropout(c["p"], s["seed"], c["step"], c["replica"]), s["flat"])
        return s["flat"]
    if c["op"] == "counts":
        ws.ws_router_counts(s["routers"], s["counts"])
        return s["counts"]
    ws.ws_balance_loss(s["routers"], s["counts"], s["loss"], 1e-2, z_coef=c["z"], workspace=s["workspace"])
    return {"loss": s["loss"], "dlogits": s["dlogits"]}


def work(case):
    c = case
    if c["op"] in ("hand out", "sum"):
        n, k = sum(_numels(c)), c["lists"]
        f, t = (4 if c["flat"] == "f32" else 2), (4 if c["tensors"] == "f32" else 2)
        return {"bytes": n * (f + k * t), "flops": n * (k + 1) if c["op"] == "sum" else n}
    tokens = c["layers"] * sum(_rows(c))
    valid = sum(_rows(c)) if c["ragged"] else 0
    counts = 8 * c["layers"] * (c["experts"] + 1)
    if c["op"] == "counts":
        return {"bytes": tokens * c["topk"] * (4 if c["index"] == "i32" else 8) + valid + counts, "flops": 0}
    b = 4 if c["logits"] == "f32" else 2
    return {"bytes": 2 * tokens * c["experts"] * b + valid + counts + 8 * c["layers"], "flops": 10 * tokens * c["experts"]}


# ----------------------------------------------------------- the definitions in 64 bits
def _product(a, x):
    """High and low 32 bits of a * x, by 16-bit halves."""
    x0, x1 = x % 65536, x // 65536
    a0, a1 = a % 65536, a // 65536
    mid = a1 * x0 + a0 * x0 // 65536
    mid2 = a0 * x1 + mid % 65536
    return a1 * x1 + mid // 65536 + mid2 // 65536, mid2 % 65536 * 65536 + a0 * x0 % 65536


def _exact_mask(c, seed, t, n, k):
    """1 / (1 - p) where replica k keeps an element of tensor t, else 0."""
    i = torch.arange(_up(n, 8) // 8, device="cuda")
    w = [i % (1 << 32), torch.zeros_like(i) + c["step"], torch.zeros_like(i) + t, c["replica"] + k + (i // (1 << 32)) * 65536]
    key = [seed % (1 << 32), seed // (1 << 32) % (1 << 32)]
    for turn in range(7):
        h0, l0 = _product(0xD2511F53, w[0])
        h2, l2 = _product(0xCD9E8D57, w[2])
        w = [h2 ^ w[1] ^ ((key[0] + turn * 0x9E3779B9) % (1 << 32)), l2, h0 ^ w[3] ^ ((key[1] + turn * 0xBB67AE85) % (1 << 32)), l0]
    bits = torch.stack([w[0] % 65536, w[0] // 65536, w[1] % 65536, w[1] // 65536, w[2] % 65536, w[2] // 65536, w[3] % 65536, w[3] // 65536], 1)
    drop = min(math.floor(c["p"] * 65536 + 0.5), 65535)
    return (bits.reshape(-1)[:n] >= drop).double() * (65536.0 / (65536.0 - drop))


def _exact_places(c, n, piece, off, shard):
    """Where the elements of a tensor lie in the sharded layout."""
    i = torch.arange(n, device="cuda")
    return off + i if c["layout"] == "concat" else i // piece * shard + off + i % piece


def exact(case, seed):
    c = case
    if c["op"] in ("hand out", "sum"):
        s = _prepare_drop(c, seed)
        numels, arena, piece, off, length, shard = _layout(c)
        out = torch.zeros((c["lists"], length) if c["op"] == "hand out" else c["shards"] * shard, dtype=torch.float64, device="cuda")
        for t, n in enumerate(numels):
            if n == 0:
                continue
            at = _exact_places(c, n, piece[t], off[t], shard)
            for k in range(c["lists"]):
                mask = _exact_mask(c, s["seed"], t, n, k)
                if c["op"] == "hand out":
                    out[k, arena[t]:arena[t] + n] = mask * s["flat"][at].double()
                else:
                    out[at] += mask * s["lists"][k, arena[t]:arena[t] + n].double()
        return out
    if c["op"] == "counts":
        return None                       # whole numbers: the plain form is exact
    s = _prepare_router(c, seed)
    dlogits = torch.zeros(s["logits"].shape, dtype=torch.float64, device="cuda")
    loss = torch.zeros(c["layers"], 2, dtype=torch.float64, device="cuda")
    live = s["valid"] if s["valid"] is not None else torch.ones(s["logits"].shape[1], dtype=torch.bool, device="cuda")
    for layer in range(c["layers"]):
        tokens = max(1, int(s["counts"][layer, -1]))
        f = s["counts"][layer, :-1].double() / (c["topk"] * tokens)
        x = s["logits"][layer][live].double().requires_grad_()
        if c["score"] == "softmax":
            p, lse = torch.softmax(x, 1), torch.logsumexp(x, 1)
        else:
            p, lse = torch.sigmoid(x) / torch.sigmoid(x).sum(1, keepdim=True), x.new_zeros(len(x))
        loss[layer, 0] = (balance := 1e-2 * c["experts"] * (f * p.sum(0)).sum() / tokens).detach()
        loss[layer, 1] = (z := c["z"] * lse.square().sum() / tokens).detach()
        dlogits[layer, live] = torch.autograd.grad(balance + z, x)[0]
    return {"loss": loss, "dlogits": dlogits}
