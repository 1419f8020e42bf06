"""Operators of a decoding loop over shared prefixes and a bounded cache: cases, plain forms and the library's calls.

Requests that share a prompt attend over it together (``prefix``); the attention weight that every entry of the cache gets is
added up (``weights``); a request above its budget keeps its heaviest entries, moved together in order (``evict``); and what was
put out is answered with its log probabilities, the entropy and the top alternatives of the row it came from (``logprobs``).

A case is a dict of plain values; ``prepare`` makes its inputs on the GPU, ``run`` makes one pass: through the plain
forms below, or, where ``own`` is true, through the entry points of ``binding``.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

TREE = dict(K=4, L1=2, L2=4, chunk=0)
TOKEN = dict(K=0, L1=0, L2=0, chunk=0)
HEADS = dict(Hq=32, Hkv=8, D=128, dtype="bf16")
PREFIX = dict(op="prefix", B=64, groups=1, shared=8192, L=1024, block=16, **TREE, **HEADS)
WEIGHTS = dict(op="weights", B=8, L=4096, block=16, protected=0, fresh=True, **TREE, **HEADS)
EVICT = dict(op="evict", B=16, L=8192, budget=4096, recent=256, protected=4, caches=16, width=512, dtype="bf16", block=16, **TOKEN)
LOGPROBS = dict(op="logprobs", R=1, V=128256, given=1, top=5, temperature=1.0, dtype="bf16", path=False, **TREE)


def listed():
    return [
        # four answers to one question: a short prompt shared, the answers just begun; latency is all of it
        dict(PREFIX, name="prefix_b4_token", B=4, shared=2048, L=128, **TOKEN),
        # the benchmark's tree in a service with one system prompt of 8192 tokens, conversations of up to 1024 behind it
        dict(PREFIX, name="prefix_b64_tree19"),
        # plain decoding of four groups of 32 requests, a long document each, fp16
        dict(PREFIX, name="prefix_b128_groups4", B=128, groups=4, shared=32768, L=2048, dtype="f16", **TOKEN),
        # one request's token: weights of a moderate context
        dict(WEIGHTS, name="weights_b1_token", B=1, **TOKEN),
        # the benchmark's batch and tree over ragged contexts, a later layer of the step
        dict(WEIGHTS, name="weights_b8_tree19", fresh=False),
        # two prompts come in stretches of 512 tokens over long contexts, a few tokens at the start protected
        dict(WEIGHTS, name="weights_b2_prompt512", B=2, L=16384, protected=64, **dict(TOKEN, chunk=512)),
        # one request a little above its budget, a small draft model's caches
        dict(EVICT, name="evict_b1", B=1, L=1100, budget=1024, recent=64, caches=8, width=128),
        # a serving batch of ragged contexts halved, 8 layers' caches at a time
        dict(EVICT, name="evict_b16"),
        # one row: the answer of one request
        dict(LOGPROBS, name="logprobs_r1"),
        # what a verification of the benchmark's batch put out, rows along the accepted paths
        dict(LOGPROBS, name="logprobs_path_b8", B=8, path=True),
        # scoring a text: 2048 rows of a large vocabulary, 20 alternatives each
        dict(LOGPROBS, name="logprobs_r2048", R=2048, V=151936, top=20),
        # fp32 rows of a vocabulary that leaves them unaligned, several given tokens a row, no alternatives
        dict(LOGPROBS, name="logprobs_f32_r64", R=64, V=50257, given=8, top=0, temperature=0.8, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_CAP = {"prefix": 1.7e11, "weights": 1.4e11, "evict": 2.2e9, "logprobs": 6.2e8}


def draw(rng):
    """One more case: the operator, batch, tree, heads, types and lengths over their ranges."""
    op = rng.choice(["prefix", "prefix", "weights", "evict", "logprobs"])
    c = dict({"prefix": PREFIX, "weights": WEIGHTS, "evict": EVICT, "logprobs": LOGPROBS}[op])
    if op in ("prefix", "weights") or op == "logprobs":
        c["K"], c["L1"], c["L2"] = rng.randint(1, 8), rng.randint(0, 4), rng.randint(1, 6)
        if rng.random() < 0.4:
            c["K"], c["L1"], c["L2"] = 0, 0, 0                  # no draft: one token
    if op == "logprobs":
        c["V"] = _log(rng, 1000, 262144)
        if rng.random() < 0.5:
            c["V"] = max(1024, c["V"] // 64 * 64)
        c["top"], c["temperature"] = rng.choice([0, 1, 5, 20, 32]), rng.choice([1.0, 1.0, round(rng.uniform(0.3, 1.5), 2)])
        c["dtype"], c["path"] = rng.choice(["bf16", "bf16", "f32", "f16"]), rng.random() < 0.3
        if c["path"]:
            c["B"] = _log(rng, 1, 64)
        else:
            c["R"], c["given"] = _log(rng, 1, 2048), rng.choice([1, 1, 3, 16])
    elif op == "evict":
        c["block"] = rng.choice([8, 16, 16, 32, 64, 24])
        c["B"], c["L"] = _log(rng, 1, 64), _log(rng, 64, 32768)
        c["budget"] = max(8, int(c["L"] * rng.uniform(0.1, 1.0)))
        c["protected"], c["recent"] = rng.choice([0, 1, 4, 7]), int(c["budget"] * rng.choice([0.0, 0.1, 0.5]))
        c["caches"], c["width"], c["dtype"] = 2 * rng.randint(1, 16), rng.choice([64, 128, 512, 1024]), rng.choice(["bf16", "f16", "f32"])
        while c["B"] * (c["L"] + 64) * c["caches"] * c["width"] * _size(c) > 4.0e9:             # the cache itself, a few GB
            c["B" if c["B"] > 1 else "caches"] //= 2
    else:
        c["block"] = rng.choice([8, 16, 16, 32, 64, 128, 24])
        c["D"] = rng.choice([64, 128, 128, 256])
        c["Hkv"] = rng.choice([1, 2, 4, 8])
        c["Hq"] = c["Hkv"] * rng.choice([1, 2, 4, 5, 7, 8])
        c["dtype"] = rng.choice(["bf16", "bf16", "f16"])
        if op == "prefix":
            c["B"], c["shared"], c["L"] = _log(rng, 2, 128), _log(rng, 64, 32768), _log(rng, 4, 4096)
            c["groups"] = rng.choice([1, 1, 2, 5])
        else:
            c["B"], c["L"], c["fresh"] = _log(rng, 1, 64), _log(rng, 4, 65536), rng.random() < 0.5
            c["protected"] = rng.choice([0, 0, 4, 100])
            if rng.random() < 0.3:
                c.update(TOKEN, chunk=_log(rng, 8, 512))
    while _cost(c) > _CAP[op]:
        if op == "logprobs" and not c["path"]:
            c["R"] = (c["R"] + 1) // 2
        elif c.get("B", 1) > (2 if op == "prefix" else 1):
            c["B"] = (c["B"] + 1) // 2
        elif op == "prefix" and c["shared"] > c["L"]:
            c["shared"] //= 2
        elif op == "evict":
            c["caches"] //= 2
        else:
            c["L"] = c["L"] // 2
    return c


# ---------------------------------------------------------------------------------------------
# shapes
# ---------------------------------------------------------------------------------------------
def _tree(c):
    """Parents and depths: a trunk of L1 nodes behind the root, then K chains of L2 nodes; or a stretch of a prompt."""
    if c["chunk"]:
        return list(range(-1, c["chunk"] - 1)), list(range(c["chunk"]))
    parent, depth = [-1], [0]
    for i in range(c["L1"]):
        parent.append(i)
        depth.append(i + 1)
    for _ in range(c["K"] if c["L2"] else 0):
        last = c["L1"]
        for j in range(c["L2"]):
            parent.append(last)
            depth.append(c["L1"] + j + 1)
            last = len(parent) - 1
    return parent, depth


def _above(c):
    """[N,N]: whether the column's node is the row's node or above it."""
    parent, _ = _tree(c)
    above = torch.zeros(len(parent), len(parent), dtype=torch.bool)
    for i, p in enumerate(parent):
        if p >= 0:
            above[i] = above[p]
        above[i, i] = True
    return above


def _shared(c):
    """Tokens of each group's prefix, whole blocks: the first group has all, the others down to a half."""
    return [max(1, int(c["shared"] * (1.0 - 0.5 * ((g * 0.6180339887) % 1.0))) // c["block"]) * c["block"] for g in range(c["groups"])]


def _lengths(c):
    """Committed tokens of each request (behind the prefix, where there is one): the first has L, the others between a quarter of it and all."""
    return [max(1, round(c["L"] * (1.0 - 0.75 * ((b * 0.6180339887) % 1.0)))) for b in range(c["B"])]


def _accepted_depths(c):
    most = max(_tree(c)[1])
    return [(most - b) % (most + 1) for b in range(c["B"])]


def _size(c):
    return 4 if c["dtype"] == "f32" else 2


def work(case):
    c, op = case, case["op"]
    depth = _tree(c)[1]
    n = len(depth)
    if op == "logprobs":
        rows = sum(d + 1 for d in _accepted_depths(c)) if c["path"] else c["R"]
        return {"bytes": rows * (c["V"] * _size(c) + 8 * c["given"] + 8 * c["top"] + 8), "flops": 6 * rows * c["V"]}
    if op == "evict":
        cut = [x for x in _lengths(c) if x > c["budget"]]
        # (the first of the heaviest entries may be in place already: a few rows)
        rows = len(cut) * max(0, c["budget"] - c["protected"])
        return {"bytes": 2 * rows * c["caches"] * c["width"] * _size(c) + sum(cut) * 8 + rows * 4, "flops": 40 * sum(cut) + 1}
    own_pairs = sum(n * x + sum(d + 1 for d in depth) for x in _lengths(c))
    own_keys = sum(x + n for x in _lengths(c))
    if op == "weights":
        left_out = sum(min(x, c["protected"]) for x in _lengths(c))
        pairs, keys = own_pairs - n * left_out, own_keys - left_out
        return {"bytes": keys * (c["Hkv"] * c["D"] * _size(c) + 8) + c["B"] * n * c["Hq"] * (c["D"] * _size(c) + 4),
                "flops": (2 * c["D"] + 2) * c["Hq"] * pairs}
    shared = _shared(c)
    pairs = own_pairs + sum(n * shared[b % c["groups"]] for b in range(c["B"]))
    return {"bytes": 2 * (own_keys + sum(shared[:c["B"]])) * c["Hkv"] * c["D"] * _size(c) + 2 * c["B"] * n * c["Hq"] * c["D"] * _size(c),
            "flops": 4 * c["D"] * c["Hq"] * pairs}


def _cost(c):
    """What a drawn case is held to: products for attention and weights, bytes elsewhere."""
    w = work(c)
    if c["op"] in ("prefix", "weights"):                        # (the plain form goes through every pair of request and position)
        n = len(_tree(c)[0])
        top = (c["shared"] if c["op"] == "prefix" else 0) + c["L"] + n
        return max(w["flops"], 4.0 * c["D"] * c["Hq"] * n * c["B"] * top, 4.0 * c["D"] * c["Hkv"] * 8 * c["B"] * top)
    return w["bytes"]


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _paged(c, g, spare=0):
    """Block table, lengths and blocks in use per request, in an order of requests and of blocks made from the seed."""
    n = len(_tree(c)[0])
    order = torch.randperm(c["B"], generator=g, device="cuda")
    lengths = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")[order]
    used = (lengths.long() + n + c["block"] - 1) // c["block"]
    width, total = (c["L"] + n + c["block"] - 1) // c["block"], sum((x + n + c["block"] - 1) // c["block"] for x in _lengths(c))
    ids = torch.randperm(total + spare, generator=g, device="cuda").int()
    at = (torch.cumsum(used, 0) - used)[:, None] + torch.arange(width, device="cuda")
    table = torch.where(torch.arange(width, device="cuda") < used[:, None], ids[at.clamp(max=total - 1)], -1)
    return lengths, table.int().contiguous(), used.int(), ids, total + spare


def prepare(case, seed):
    c, op = dict(case), case["op"]
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dev, dt = dict(device="cuda"), TYPES[c["dtype"]]
    normal = lambda *shape: torch.empty(*shape, dtype=dt, **dev).normal_(generator=g)  # noqa: E731
    parent, depth = _tree(c)
    n = len(parent)
    # a program that works with masks keeps those of its tree, as it keeps the parents
    s = {"case": c, "n": n, "parent": torch.tensor(parent, dtype=torch.int32, **dev), "above": _above(c).to("cuda"),
         "depth": torch.tensor(depth, **dev)}
    if op == "logprobs":
        rows = (c["B"], n) if c["path"] else (c["R"],)
        logits = (3.0 * torch.empty(*rows, c["V"], **dev).normal_(generator=g)).to(dt)
        s["logits"] = logits
        if c["path"]:
            order = torch.randperm(c["B"], generator=g, device="cuda")
            wanted = torch.tensor(_accepted_depths(c), **dev)[order]
            score = torch.rand(c["B"], n, generator=g, **dev) - (torch.tensor(depth, **dev) != wanted[:, None]).float()
            s["accepted"] = score.argmax(-1).int()
            tokens = torch.randint(c["V"], (c["B"], n), generator=g, **dev)
            s["tokens"] = torch.where(torch.arange(n, **dev) <= wanted[:, None], tokens, -1).int()
        else:
            s["tokens"] = torch.randint(c["V"], (c["R"], c["given"]), generator=g, **dev).int()
        return s
    if op == "evict":
        lengths, table, used, ids, total = _paged(c, g, spare=5)
        count = 5
        ring = torch.full((total,), -1, dtype=torch.int32, **dev)
        begin = int(seed) % total
        ring[(begin + torch.arange(count, **dev)) % total] = ids[total - count:]
        # weights as they pile up: few entries have much, many next to nothing, and entries that nobody has looked at are equal
        weights = torch.exp(3.0 * torch.empty(total, c["block"], **dev).normal_(generator=g))
        weights[torch.rand(total, c["block"], generator=g, **dev) < 0.05] = 0.0
        s.update(lengths=lengths, table=table, owned=used, ring=ring, range=torch.tensor([begin, count], dtype=torch.int32, **dev),
                 weights=weights, protected=torch.full((c["B"],), c["protected"], dtype=torch.int32, **dev),
                 cache=torch.empty(c["caches"], total, c["block"], c["width"], dtype=dt, **dev).normal_(generator=g))
        return s
    if op == "weights":
        lengths, table, _, _, blocks = _paged(c, g)
        s.update(lengths=lengths, table=table, q=(2.0 * normal(c["B"], n, c["Hq"], c["D"])).to(dt),
                 k_cache=normal(blocks, c["block"], c["Hkv"], c["D"]), keys=c["L"] + n,
                 weights=torch.rand(blocks, c["block"], generator=g, **dev),
                 protected=torch.full((c["B"],), c["protected"], dtype=torch.int32, **dev) if c["protected"] else None)
        seen, slot = _seen(s, s["keys"])
        s["lse"] = torch.logsumexp(_scores(s, slot, seen), -1).transpose(1, 2).contiguous()
        return s
    # prefix: the requests' own blocks behind those of their group's prefix, in one row of the table
    own_lengths, own_table, _, ids, total = _paged(c, g, spare=sum(_shared(c)) // c["block"])
    shared = [x // c["block"] for x in _shared(c)]
    rest, at = ids[total - sum(shared):], 0
    group = (torch.randperm(c["B"], generator=g, device="cuda") % c["groups"]).int()
    prefix_table = torch.full((c["groups"], max(shared)), -1, dtype=torch.int32, **dev)
    for k, x in enumerate(shared):
        prefix_table[k, :x] = rest[at:at + x]
        at += x
    blocks = torch.tensor(shared, dtype=torch.int32, **dev)
    mine = blocks[group.long()].long()
    column = torch.arange(max(shared) + own_table.shape[1], **dev)
    behind = torch.gather(own_table, 1, (column - mine[:, None]).clamp(0, own_table.shape[1] - 1))
    ahead = torch.gather(prefix_table, 1, column.clamp(max=max(shared) - 1).expand(c["groups"], -1))[group.long()]
    inside = (column >= mine[:, None]) & (column < mine[:, None] + own_table.shape[1])
    table = torch.where(column < mine[:, None], ahead, torch.where(inside, behind, -1)).int().contiguous()
    s.update(lengths=(own_lengths + mine * c["block"]).int(), table=table, group=group, blocks=blocks, prefix_table=prefix_table,
             q=(2.0 * normal(c["B"], n, c["Hq"], c["D"])).to(dt), k_cache=normal(total, c["block"], c["Hkv"], c["D"]),
             v_cache=normal(total, c["block"], c["Hkv"], c["D"]), keys=int(max(shared)) * c["block"] + c["L"] + n)
    # made when the requests come together and kept from step to step: the requests in the order of their groups, where each group's
    # begin, and where each request stands among its group's
    members = torch.sort(group, stable=True).indices
    first = torch.searchsorted(group[members], torch.arange(c["groups"] + 1, dtype=torch.int32, **dev))
    place = torch.empty_like(group)
    place[members] = torch.arange(c["B"], dtype=torch.int32, **dev)
    s["plan"] = (group, members.int(), first.int(), (place - first[group.long()]).int(), blocks, prefix_table)
    return s


# ---------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------
def _seen(s, positions):
    """[B,N,positions]: which keys a node sees; and each key's slot."""
    c, n, lengths, table = s["case"], s["n"], s["lengths"].long(), s["table"].long()
    j = torch.arange(positions, device=table.device)
    node = j - lengths[:, None]
    in_tree = (node >= 0) & (node < n)
    node = node.clamp(0, n - 1)
    seen = torch.where(in_tree[:, None], s["above"].t()[node].transpose(1, 2), (j < lengths[:, None])[:, None])
    slot = torch.gather(table, 1, (j // c["block"]).clamp(max=table.shape[1] - 1).expand(table.shape[0], -1)) * c["block"] + j % c["block"]
    return seen, slot.clamp(min=0)


def _scores(s, slot, seen):
    """[B,Hq,N,keys], -inf where a node does not see a key."""
    c, n = s["case"], s["n"]
    B, Hkv, D, G = c["B"], c["Hkv"], c["D"], c["Hq"] // c["Hkv"]
    k = s["k_cache"].view(-1, Hkv, D)[slot].float().permute(0, 2, 3, 1)
    q = s["q"].float().view(B, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, D)
    return (torch.matmul(q, k).view(B, c["Hq"], n, -1) / math.sqrt(D)).masked_fill_(~seen[:, None], -math.inf)


def _plain_prefix(s):
    c, n = s["case"], s["n"]
    B, Hkv, D = c["B"], c["Hkv"], c["D"]
    seen, slot = _seen(s, s["keys"])
    score = _scores(s, slot, seen)
    p = score.sub_(score.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1, keepdim=True)
    v = s["v_cache"].view(-1, Hkv, D)[slot].float().transpose(1, 2)
    out = torch.matmul(p.view(B, Hkv, -1, p.shape[-1]), v).view(B, c["Hq"], n, D) / total
    return {"out": out.transpose(1, 2).to(s["q"].dtype), "status": torch.zeros(B, dtype=torch.int32, device="cuda")}


def _plain_weights(s):
    c, n = s["case"], s["n"]
    lengths, flat = s["lengths"].long(), s["weights"].view(-1)
    seen, slot = _seen(s, s["keys"])
    j = torch.arange(s["keys"], device="cuda")
    if c["protected"]:
        seen = seen & (j >= s["protected"][:, None])[:, None]
    got = _scores(s, slot, seen).sub_(s["lse"].transpose(1, 2)[..., None]).exp_().sum((1, 2))
    counted = (j < lengths[:, None] + n) & (j >= c["protected"])
    in_tree = j >= lengths[:, None]
    old = flat[slot]
    if c["fresh"]:
        old = torch.where(in_tree, 0.0, old)
    flat[slot[counted]] = (old + got)[counted]
    return {"weights": s["weights"], "status": torch.zeros(c["B"], dtype=torch.int32, device="cuda")}


def _plain_evict(s):
    c, lengths, table, budget = s["case"], s["lengths"].long(), s["table"].long(), s["case"]["budget"]
    B, block, dev = c["B"], c["block"], table.device
    j = torch.arange(c["L"], device=dev)
    live = j < lengths[:, None]
    slot = (torch.gather(table, 1, (j // block).expand(B, -1)) * block + j % block).clamp(min=0)
    first = s["protected"].long().clamp(max=budget)
    recent = torch.minimum(torch.full_like(first, c["recent"]), budget - first)
    sure = (j < first[:, None]) | (j >= (lengths - recent)[:, None])
    score = torch.where(live, torch.where(sure, math.inf, s["weights"].view(-1)[slot]), -math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(1, order, j.expand(B, -1).contiguous())
    keep = live & (rank < budget)
    target = keep.long().cumsum(-1) - 1
    row, entry = keep.nonzero(as_tuple=True)
    source, goal = slot[row, entry], slot[row, target[row, entry]]
    flat = s["cache"].view(c["caches"], -1, c["width"])
    flat[:, goal] = flat[:, source]                              # (all rows are taken before any is put down)
    weights = s["weights"].view(-1)
    weights[goal] = weights[source]
    after = torch.minimum(lengths, torch.full_like(lengths, budget))
    owned = torch.where(lengths > budget, (after + block - 1) // block, s["owned"].long())
    freed = s["owned"].long() - owned
    ring, upto = s["ring"], torch.cumsum(freed, 0)
    column = torch.arange(table.shape[1], device=dev)
    gone = (column >= owned[:, None]) & (column < s["owned"][:, None])
    at = s["range"][0] + s["range"][1] + (upto - freed)[:, None] + column - owned[:, None]
    ring[at[gone] % ring.numel()] = table[gone].int()
    return {"cache": s["cache"], "weights": s["weights"], "lengths": after.int(), "owned": owned.int(), "ring": ring,
            "range": torch.stack([s["range"][0], s["range"][1] + upto[-1]]).int(), "status": torch.zeros(B, dtype=torch.int32, device=dev)}


def _path_rows(s):
    """[B,N]: the accepted path's node at each depth, -1 behind it."""
    step = torch.arange(s["n"], device="cuda")
    on_path = s["above"][s["accepted"].long()][:, None] & (s["depth"] == step[:, None])
    return torch.where(on_path.any(-1), on_path.int().argmax(-1), -1)


def _plain_logprobs(s):
    c, z, tokens = s["case"], s["logits"], s["tokens"].long()
    if c["path"]:
        node = _path_rows(s)
        there = (node >= 0).flatten()
        z = z.flatten(0, 1)[(node.clamp(min=0) + torch.arange(c["B"], device="cuda")[:, None] * s["n"]).flatten()[there]]
        tokens = tokens.flatten()[there][:, None]
    x = z.float() / c["temperature"]
    x = x - x.amax(-1, keepdim=True)
    e = x.exp()
    total = e.sum(-1, keepdim=True)
    log = x - total.log()
    entropy = total.log()[:, 0] - (e * x).sum(-1) / total[:, 0]
    got = {"logprob": torch.gather(log, 1, tokens), "entropy": entropy}
    if c["top"]:
        # of equal logits the lowest index first: the logit's order in the upper bits of a whole number, the index in the lower
        bits = (z.float() + 0.0).view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * 2**20 + (2**20 - 1 - torch.arange(c["V"], device="cuda"))
        got["top_tokens"] = (2**20 - 1 - torch.topk(key, c["top"], -1).values % 2**20).int()
        got["top_logprobs"] = torch.gather(log, 1, got["top_tokens"].long())
    if c["path"]:
        full = {"logprob": 0.0, "entropy": 0.0, "top_tokens": -1, "top_logprobs": 0.0}
        for k, v in got.items():
            v = v[:, 0] if k == "logprob" else v
            spread = torch.full((c["B"] * s["n"],) + v.shape[1:], full[k], dtype=v.dtype, device="cuda")
            spread[there] = v
            got[k] = spread.view(c["B"], s["n"], *v.shape[1:])
    status = torch.zeros(c["B"] * s["n"] if c["path"] else c["R"], dtype=torch.int32, device="cuda")
    return dict(got, status=status.view(c["B"], s["n"]) if c["path"] else status)


# ---------------------------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------------------------
def _own(s):
    from paper_2602_16994_b200 import binding
    c, op = s["case"], s["case"]["op"]
    if op == "prefix":
        o = binding.prefix_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["parent"], s["plan"])
        return {"out": o.out, "status": o.status}
    if op == "weights":
        o = binding.cache_weights(s["weights"], s["q"], s["k_cache"], s["lse"], s["table"], s["lengths"], s["parent"],
                                  protected=s["protected"], fresh=c["fresh"])
        return {"weights": s["weights"], "status": o}
    if op == "evict":
        o = binding.cache_evict(s["cache"], s["weights"], s["lengths"], s["table"], s["owned"], s["ring"], s["range"], c["budget"],
                                recent=c["recent"], protected=s["protected"])
        return {"cache": s["cache"], "weights": s["weights"], "lengths": o.lengths, "owned": o.owned, "ring": s["ring"],
                "range": o.free_range, "status": o.status}
    if c["path"]:
        o = binding.path_logprobs(s["logits"], s["accepted"], s["tokens"], s["parent"], temperature=c["temperature"], top=c["top"])
    else:
        o = binding.token_logprobs(s["logits"], s["tokens"], temperature=c["temperature"], top=c["top"])
    got = {"logprob": o.logprob, "entropy": o.entropy}
    if c["top"]:
        got.update(top_tokens=o.top_tokens, top_logprobs=o.top_logprobs)
    return dict(got, status=o.status)


def run(state):
    if own:
        return _own(state)
    return {"prefix": _plain_prefix, "weights": _plain_weights, "evict": _plain_evict,
            "logprobs": _plain_logprobs}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------
def _exact_rows(s, b):
    """Request by request: keys in order, and [N, keys] of what the nodes see."""
    c, n, length = s["case"], s["n"], int(s["lengths"][b])
    blocks = s["table"][b, :-(-(length + n) // c["block"])].long()
    mask = torch.cat([torch.ones(n, length, dtype=torch.bool, device="cuda"), s["above"]], 1)
    k = s["k_cache"][blocks].flatten(0, 1)[:length + n].double()
    q = s["q"][b].double().view(n, c["Hkv"], c["Hq"] // c["Hkv"], c["D"])
    score = torch.einsum("nhgd,lhd->hngl", q, k) * c["D"] ** -0.5
    return blocks, mask, score, length + n


def _exact_prefix(s):
    c, n = s["case"], s["n"]
    out = torch.empty(c["B"], n, c["Hq"], c["D"], dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        blocks, mask, score, keys = _exact_rows(s, b)
        score = score.masked_fill(~mask[None, :, None], -math.inf)
        weight = (score - torch.logsumexp(score, -1, keepdim=True)).exp()
        v = s["v_cache"][blocks].flatten(0, 1)[:keys].double()
        out[b] = torch.einsum("hngl,lhd->nhgd", weight, v).reshape(n, c["Hq"], c["D"])
    return {"out": out, "status": None}


def _exact_weights(s):
    c, n = s["case"], s["n"]
    weights = s["weights"].double()
    for b in range(c["B"]):
        blocks, mask, score, keys = _exact_rows(s, b)
        lse = s["lse"][b].double().view(n, c["Hkv"], -1).permute(1, 0, 2)[..., None]
        got = torch.where(mask[None, :, None], (score - lse).exp(), 0.0).sum((0, 1, 2))
        at = torch.arange(keys, device="cuda")
        block, place = blocks[at // c["block"]], at % c["block"]
        old = weights[block, place]
        if c["fresh"]:
            old[keys - n:] = 0.0
        counted = at >= c["protected"]
        weights[block[counted], place[counted]] = (old + got)[counted]
    return {"weights": weights, "status": None}


def _exact_logprobs(s):
    c = s["case"]
    names = ["logprob", "entropy"] + (["top_tokens", "top_logprobs"] if c["top"] else [])
    V, flat = c["V"], s["logits"].reshape(-1, c["V"])
    if c["path"]:
        node = _path_rows(s)
        rows = torch.where(node >= 0, node + torch.arange(c["B"], device="cuda")[:, None] * s["n"], -1).flatten().tolist()
        tokens = s["tokens"].reshape(-1, 1)
    else:
        rows, tokens = list(range(c["R"])), s["tokens"]
    logprob = torch.zeros(len(rows), tokens.shape[1], dtype=torch.float64, device="cuda")
    entropy = torch.zeros(len(rows), dtype=torch.float64, device="cuda")
    top = torch.zeros(len(rows), c["top"], dtype=torch.float64, device="cuda")
    for i, r in enumerate(rows):
        if r < 0:
            continue
        z = flat[r].double() / c["temperature"]
        log = z - torch.logsumexp(z, 0)
        logprob[i] = log[tokens[i].long()]
        entropy[i] = -(log.exp() * log).sum()
        if c["top"]:
            top[i] = torch.topk(log, c["top"]).values
    shape = (c["B"], s["n"]) if c["path"] else (c["R"],)
    got = {"logprob": logprob.view(c["B"], s["n"]) if c["path"] else logprob, "entropy": entropy.view(shape), "top_tokens": None,
           "top_logprobs": top.view(*shape, c["top"])}
    return dict({k: got[k] for k in names}, status=None)


def exact(case, seed):
    """An eviction copies and counts: nothing of it is a computed number."""
    if case["op"] == "evict":
        return None
    s = prepare(case, seed)
    return {"prefix": _exact_prefix, "weights": _exact_weights, "logprobs": _exact_logprobs}[case["op"]](s)
