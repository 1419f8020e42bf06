"""The operators around a verification step of a decoding loop: cases, plain forms and the library's calls.

A decoding step with a draft tree gives every request blocks of the paged cache and slots for the tree's nodes
(``slots``), normalises and rotates the projections of the nodes and writes keys and values to the slots (``rope``),
attends from every node over the committed tokens and the node's ancestors (``attend``), verifies the drafted
tokens (``verify``, here from probabilities) and moves the accepted path's entries of the cache behind the committed
tokens (``commit``).

A case is a dict of plain values; ``prepare`` makes its inputs on the GPU, ``run`` makes one pass: through the plain
forms below, or, where ``own`` is true, through the entry points of ``binding``.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

SLOTS = dict(op="slots", B=8, L=4096, K=4, L1=2, L2=4, block=16)
ROPE = dict(op="rope", B=8, K=4, L1=2, L2=4, Hq=32, Hkv=8, D=128, rot=128, pairs="halves", dtype="bf16", norm=True,
            L=8192, block=16)
ATTEND = dict(op="attend", B=8, K=4, L1=2, L2=4, Hq=32, Hkv=8, D=128, dtype="bf16", L=4096, block=16, window=0, sinks=0)
VERIFY = dict(op="verify", B=8, V=128256, most=5, sigma=1.0, dtype="f32", draft=True)
COMMIT = dict(op="commit", B=8, K=4, L1=2, L2=4, caches=64, width=1024, dtype="bf16", L=1024, block=16)


def listed():
    return [
        # slots and positions of the benchmark's batch: the smallest call, latency is all of it
        dict(SLOTS, name="slots_b8_tree19"),
        # a large serving batch of the serving configuration's tree: 2048 requests of up to 32768 tokens
        dict(SLOTS, name="slots_b2048_tree51", B=2048, L=32768, K=8, L2=6),
        # one layer's projections of the benchmark's batch (152 tokens): a small call on the decoding path
        dict(ROPE, name="rope_b8_tree19"),
        # one layer's projections of a serving batch (6528 tokens), half of each head rotated in neighbouring pairs, far positions
        dict(ROPE, name="rope_b128_tree51_pairs", B=128, K=8, L2=6, rot=64, pairs="neighbours", L=131072),
        # plain decoding of one request at a moderate context: a single token, many heads to a key head
        dict(ATTEND, name="attend_b1_token", B=1, K=0, L1=0, L2=0, L=8192),
        # the benchmark's batch and tree over ragged contexts
        dict(ATTEND, name="attend_b8_tree19"),
        # the serving configuration's batch and tree, contexts of a chat service
        dict(ATTEND, name="attend_b128_tree51", B=128, K=8, L2=6, L=4096),
        # long contexts under a sliding window with a few tokens at the start kept visible, fp16, small heads
        dict(ATTEND, name="attend_b16_window", B=16, K=4, L1=0, L2=6, Hq=14, Hkv=2, D=64, dtype="f16", L=65536, block=64,
             window=4096, sinks=4),
        # an interactive batch of drafted chains verified from processed probabilities
        dict(VERIFY, name="verify_b8"),
        # a serving batch with ragged drafts found by lookup (no draft probabilities), the widest listed vocabulary
        dict(VERIFY, name="verify_b128_lookup", B=128, V=151936, most=3, draft=False),
        # the accepted paths of the benchmark's batch moved in 32 layers' caches of keys and values
        dict(COMMIT, name="commit_b8_64caches"),
        # a serving batch, small heads, fewer layers
        dict(COMMIT, name="commit_b128_24caches", B=128, K=8, L2=6, caches=24, width=512, L=1024, block=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_CAP = {"slots": 2.0e6, "rope": 2.5e8, "attend": 4.5e11, "verify": 2.0e8, "commit": 2.5e8}


def draw(rng):
    """One more case: the operator, batch, tree, heads, types and lengths over their ranges."""
    op = rng.choice(["slots", "rope", "attend", "attend", "attend", "verify", "commit"])
    c = dict({"slots": SLOTS, "rope": ROPE, "attend": ATTEND, "verify": VERIFY, "commit": COMMIT}[op])
    c["B"] = _log(rng, 1, 2048 if op == "slots" else 128)
    if op == "verify":
        c["V"] = _log(rng, 1000, 262144)
        if rng.random() < 0.5:
            c["V"] = max(1024, c["V"] // 64 * 64)
        c["most"], c["sigma"] = rng.randint(1, 8), round(rng.uniform(0.5, 1.2), 3)
        c["dtype"], c["draft"] = rng.choice(["f32", "f32", "bf16"]), rng.random() < 0.7
    else:
        c["K"], c["L1"], c["L2"] = rng.randint(1, 8), rng.randint(0, 4), rng.randint(1, 6)
        if rng.random() < 0.2:
            c["K"], c["L1"], c["L2"] = 0, 0, 0                  # no draft: one token
        c["block"] = rng.choice([8, 16, 16, 32, 64, 128, 24])
        c["L"] = _log(rng, 4, 4096 if op == "commit" else 131072)
    if op in ("rope", "attend"):
        c["D"] = rng.choice([64, 128, 128, 256])
        c["Hkv"] = rng.choice([1, 2, 4, 8])
        c["Hq"] = c["Hkv"] * rng.choice([1, 2, 4, 5, 7, 8])
        c["dtype"] = rng.choice(["bf16", "bf16", "f16"])
    if op == "rope":
        c["rot"] = rng.choice([c["D"], c["D"], c["D"] // 2])
        c["pairs"], c["norm"] = rng.choice(["halves", "neighbours"]), rng.random() < 0.8
    if op == "attend" and rng.random() < 0.4:
        c["window"], c["sinks"] = _log(rng, 16, 8192), rng.choice([0, 1, 4, 64])
    if op == "commit":
        c["caches"], c["width"] = 2 * rng.randint(1, 32), rng.choice([64, 128, 512, 1024])
        while c["B"] * (c["L"] + 64) * c["caches"] * c["width"] > 2.0e9:            # the cache itself, a few GB
            c["L" if c["L"] > 64 else "caches"] //= 2
    while _cost(c) > _CAP[op]:
        if op == "verify" and c["most"] > 2:
            c["most"] -= 1
        elif c["B"] > 1:
            c["B"] = (c["B"] + 1) // 2
        else:
            c["L"] = c["L"] // 2
    return c


# ---------------------------------------------------------------------------------------------
# shapes
# ---------------------------------------------------------------------------------------------
def _tree(c):
    """Parents and depths: a trunk of L1 nodes behind the root, then K chains of L2 nodes."""
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


def _paths(c):
    """For every node, the nodes from the root to it."""
    parent, _ = _tree(c)
    paths = []
    for i, p in enumerate(parent):
        paths.append((paths[p] if p >= 0 else []) + [i])
    return paths


def _lengths(c):
    """Committed tokens of each request: the first has L, the others between a quarter of it and all."""
    return [max(1, round(c["L"] * (1.0 - 0.75 * ((b * 0.6180339887) % 1.0)))) for b in range(c["B"])]


def _drafts(c):
    return [(c["most"] - b) % (c["most"] + 1) for b in range(c["B"])]


def _accepted_depths(c):
    most = max(_tree(c)[1])
    return [(most - b) % (most + 1) for b in range(c["B"])]


def _visible(c):
    """(keys that any node of the request sees, pairs of node and key) summed over the batch."""
    _, depth = _tree(c)
    keys = pairs = 0
    for n in _lengths(c):
        w, s = c["window"] or n + len(depth) + 1, min(c["sinks"], n)
        seen = lambda d: min(n, s + max(0, n - max(s, n + d - w + 1)))  # noqa: E731
        keys += seen(0) + len(depth)
        pairs += sum(seen(d) + min(d + 1, w) for d in depth)
    return keys, pairs


def _size(c):
    return 4 if c["dtype"] == "f32" else 2


def work(case):
    c, op = case, case["op"]
    if op == "verify":
        read = c["B"] * c["V"] * _size(c) * (2 if c["draft"] else 1)
        return {"bytes": read + sum(_drafts(c)) * 16 + c["B"] * 24, "flops": 2 * c["B"] * c["V"]}
    n = len(_tree(c)[0])
    if op == "slots":
        return {"bytes": c["B"] * (8 * n + 4 * (n // c["block"] + 1) * 3 + 24), "flops": 4 * c["B"] * n}
    if op == "rope":
        row = (2 * c["Hq"] + 4 * c["Hkv"]) * c["D"] * _size(c)
        return {"bytes": c["B"] * n * (row + 8), "flops": c["B"] * n * (c["Hq"] + c["Hkv"]) * c["D"] * 8}
    if op == "attend":
        keys, pairs = _visible(c)
        io = 2 * c["B"] * n * c["Hq"] * c["D"] * _size(c)
        return {"bytes": io + 2 * keys * c["Hkv"] * c["D"] * _size(c), "flops": 4 * c["D"] * c["Hq"] * pairs}
    moved = sum(_accepted_depths(c)) * c["caches"] * c["width"] * _size(c)
    return {"bytes": 2 * moved + 16 * c["B"], "flops": moved // _size(c)}


def _cost(c):
    """What a drawn case is held to: products for attention, bytes of inputs and outputs elsewhere."""
    w = work(c)
    if c["op"] == "attend":                                     # (the plain form goes through every pair of node and position)
        n = len(_tree(c)[0])
        return max(w["flops"], 4.0 * c["D"] * c["Hq"] * n * c["B"] * (c["L"] + n), 100.0 * w["bytes"])
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
    dev, dt = dict(device="cuda"), TYPES[c.get("dtype", "f32")]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    uniform = lambda *shape: torch.rand(*shape, generator=g, device="cuda")  # noqa: E731
    s = {"case": c}
    if op == "verify":
        drafts = torch.tensor(_drafts(c), **dev)[torch.randperm(c["B"], generator=g, device="cuda")]
        total = sum(_drafts(c))
        cu = torch.zeros(c["B"] + 1, dtype=torch.int32, **dev)
        cu[1:] = torch.cumsum(drafts, 0)
        # rows of the target law: a request's drafts, then one more; rows of the draft law: the drafts alone
        row = torch.arange(total + c["B"], **dev)
        extra = cu[1:].long() + torch.arange(c["B"], **dev)
        is_draft = torch.ones(total + c["B"], dtype=torch.bool, **dev)
        is_draft[extra] = False
        drafted = row[is_draft][:total]
        zq = 3.0 * normal(total + c["B"], c["V"])
        q = torch.softmax(zq[drafted], -1)
        if not c["draft"]:                                      # what a lookup finds carries about half of the law, more or less
            token = torch.randint(c["V"], (total,), generator=g, device="cuda")
            zq[drafted, token] += math.log(c["V"]) + 5.0
        zq += c["sigma"] * normal(total + c["B"], c["V"])
        p = torch.softmax(zq, -1)
        del zq
        if c["draft"]:                                          # tokens drawn from the draft law
            token = (q / torch.empty_like(q).exponential_(generator=g)).argmax(-1) if total else torch.zeros(0, **dev)
        s.update(target=p.to(dt), draft=q.to(dt) if c["draft"] else None, token=token.int(), cu=cu, most=c["most"],
                 u_accept=uniform(total), u_bonus=uniform(total + c["B"]))
        return s
    parent, depth = _tree(c)
    n = len(parent)
    above = torch.zeros(n, n, dtype=torch.bool)                 # whether the column's node is the row's node or above it
    for i, nodes in enumerate(_paths(c)):
        above[i, nodes] = True
    # a program that works with masks keeps those of its tree, as it keeps the parents
    s.update(n=n, parent=torch.tensor(parent, dtype=torch.int32, **dev), above=above.to("cuda"),
             depth=torch.tensor(depth, **dev))
    if op == "slots":
        spare = c["B"] * (n // c["block"] + 2)
        lengths, table, used, ids, total = _paged(c, g, spare)
        owned = (lengths + c["block"] - 1) // c["block"]        # what the committed tokens lie in
        table = torch.where(torch.arange(table.shape[1], **dev) < owned[:, None], table, -1).int().contiguous()
        begin = int(seed) % total
        rest = ids[total - spare:] if spare < total else ids
        ring = torch.full((total,), -1, dtype=torch.int32, **dev)
        ring[(begin + torch.arange(len(rest), **dev)) % total] = rest
        s.update(lengths=lengths, table=table, owned=owned, ring=ring,
                 range=torch.tensor([begin, len(rest)], dtype=torch.int32, **dev))
        return s
    if op == "commit":
        lengths, table, _, _, blocks = _paged(c, g)
        wanted = torch.tensor(_accepted_depths(c), **dev)[torch.randperm(c["B"], generator=g, device="cuda")]
        score = uniform(c["B"], n) - (torch.tensor(depth, **dev) != wanted[:, None]).float()
        cache = torch.empty(c["caches"], blocks, c["block"], c["width"], dtype=dt, **dev).normal_(generator=g)
        s.update(lengths=lengths, table=table, accepted=score.argmax(-1).int(), cache=cache)
        return s
    lengths, table, _, _, blocks = _paged(c, g)
    heads = c["Hq"] + 2 * c["Hkv"]
    if op == "rope":
        tokens = c["B"] * n
        qkv = normal(tokens, heads, c["D"]).to(dt)              # a fused projection's output: q, k and v are views of it
        place = torch.randperm(2 * tokens + c["block"], generator=g, device="cuda")[:tokens]
        shape = (-(-(2 * tokens + c["block"]) // c["block"]), c["block"], c["Hkv"], c["D"])
        s.update(q=qkv[:, :c["Hq"]], k=qkv[:, c["Hq"]:c["Hq"] + c["Hkv"]], v=qkv[:, c["Hq"] + c["Hkv"]:],
                 wq=(1.0 + 0.1 * normal(c["D"])).to(dt) if c["norm"] else None,
                 wk=(1.0 + 0.1 * normal(c["D"])).to(dt) if c["norm"] else None,
                 inv_freq=(500000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, **dev) / c["rot"])).float(),
                 positions=(lengths[:, None] + torch.tensor(depth, dtype=torch.int32, **dev)).int().contiguous(),
                 slots=place.int().view(c["B"], n), k_cache=normal(*shape).to(dt), v_cache=normal(*shape).to(dt))
        return s
    # scores of a few units' spread, as trained heads give them: attention is neither flat nor on one key
    s.update(lengths=lengths, table=table, q=(2.0 * normal(c["B"], n, c["Hq"], c["D"])).to(dt),
             k_cache=torch.empty(blocks, c["block"], c["Hkv"], c["D"], dtype=dt, **dev).normal_(generator=g),
             v_cache=torch.empty(blocks, c["block"], c["Hkv"], c["D"], dtype=dt, **dev).normal_(generator=g),
             keys=c["L"] + n)
    return s


# ---------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------
def _plain_slots(s):
    block, lengths, owned, n = s["case"]["block"], s["lengths"].long(), s["owned"].long(), s["n"]
    table, ring = s["table"], s["ring"].long()
    depth = s["depth"]
    need = (lengths + n + block - 1) // block
    more = (need - owned).clamp(min=0)
    upto = torch.cumsum(more, 0)
    fits = (more == 0) | (upto <= s["range"][1])
    status = torch.where(fits, 0, 6)
    more = torch.where(fits, more, 0)
    column = torch.arange(table.shape[1], device=table.device)
    index = column - owned[:, None]
    fresh = (index >= 0) & (index < more[:, None])
    at = (s["range"][0] + (upto - (need - owned).clamp(min=0))[:, None] + index).clamp(min=0) % ring.numel()
    table = torch.where(fresh, ring[at], table.long())
    place = lengths[:, None] + torch.arange(n, device=table.device)
    slots = torch.gather(table, 1, place // block) * block + place % block
    taken = more.sum()
    after = torch.stack([(s["range"][0] + taken) % ring.numel(), s["range"][1] - taken])
    return {"slots": torch.where(fits[:, None], slots, -1).int(), "positions": (lengths[:, None] + depth).int(),
            "table": table.int(), "owned": (owned + more).int(), "range": after.int(), "status": status.int()}


def _plain_norm(x, w, eps=1e-6):
    x = x.float()
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * w.float()


def _plain_turn(x, cos, sin, pairs):
    r = 2 * cos.shape[-1]
    head, tail = x[..., :r], x[..., r:]
    if pairs == "halves":
        a, b = head[..., :r // 2], head[..., r // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, tail], -1)
    a, b = head[..., 0::2], head[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), tail], -1)


def _plain_rope(s):
    c = s["case"]
    angle = s["positions"].reshape(-1, 1, 1).double() * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _plain_turn(_plain_norm(s["q"], s["wq"]), cos, sin, c["pairs"]).to(s["q"].dtype)
    k = _plain_turn(_plain_norm(s["k"], s["wk"]), cos, sin, c["pairs"]).to(s["q"].dtype)
    slots = s["slots"].reshape(-1).long()
    s["k_cache"].view(-1, c["Hkv"], c["D"])[slots] = k
    s["v_cache"].view(-1, c["Hkv"], c["D"])[slots] = s["v"]
    return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _seen(s, positions):
    """[B,N,positions]: which keys a node sees; and each key's slot."""
    c, n, lengths, table = s["case"], s["n"], s["lengths"].long(), s["table"].long()
    above, depth = s["above"], s["depth"]
    j = torch.arange(positions, device=table.device)
    node = j - lengths[:, None]
    in_tree = (node >= 0) & (node < n)
    node = node.clamp(0, n - 1)
    t = lengths[:, None] + depth
    where = torch.where(in_tree, lengths[:, None] + depth[node], j)
    seen = torch.where(in_tree[:, None], above.t()[node].transpose(1, 2), (j < lengths[:, None])[:, None])
    if c["window"]:
        seen = seen & ((where[:, None] > t[:, :, None] - c["window"]) | (where[:, None] < c["sinks"]))
    slot = torch.gather(table, 1, (j // c["block"]).expand(table.shape[0], -1)) * c["block"] + j % c["block"]
    return seen, slot.clamp(min=0)


def _plain_attend(s):
    c, n = s["case"], s["n"]
    B, Hkv, D, G = c["B"], c["Hkv"], c["D"], c["Hq"] // c["Hkv"]
    seen, slot = _seen(s, s["keys"])
    k = s["k_cache"].view(-1, Hkv, D)[slot].float().permute(0, 2, 3, 1)
    q = s["q"].float().view(B, n, Hkv, G, D).transpose(1, 2).reshape(B, Hkv, n * G, D)
    score = torch.matmul(q, k).view(B, Hkv, n, G, -1) / math.sqrt(D)
    del k
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    p = (score - score.amax(-1, keepdim=True)).exp_()
    del score
    total = p.sum(-1, keepdim=True)
    v = s["v_cache"].view(-1, Hkv, D)[slot].float().transpose(1, 2)
    out = torch.matmul(p.view(B, Hkv, n * G, -1), v).view(B, Hkv, n, G, D) / total
    return {"out": out.transpose(1, 2).reshape(B, n, c["Hq"], D).to(s["q"].dtype),
            "status": torch.zeros(B, dtype=torch.int32, device="cuda")}


def _plain_verify(s):
    c, p, q, token, most = s["case"], s["target"], s["draft"], s["token"].long(), s["most"]
    cu = s["cu"].long()
    first, count = cu[:-1], cu[1:] - cu[:-1]
    B, step = count.numel(), torch.arange(most, device=p.device)
    live = step < count[:, None]
    at = torch.where(live, first[:, None] + step, 0)
    row = at + torch.arange(B, device=p.device)[:, None]
    if token.numel():
        x = token[at]
        px = p[row, x].double()
        qx = q[at, x].double() if q is not None else torch.ones_like(px)
        ratio = torch.where(px > 0, torch.where(qx > 0, px / qx, 1.0), 0.0).clamp(max=1.0)
        accept = live & (s["u_accept"][at].double() < ratio)
    else:
        x, accept = torch.zeros_like(at), live
    length = accept.int().cumprod(-1).sum(-1)
    stop = first + length + torch.arange(B, device=p.device)
    w = p[stop].double()
    rejected = length < count
    if token.numel():
        q_at = torch.where(rejected, first + length, 0)
        x_at = token[q_at]
        if q is not None:
            r = (w - q[q_at].double()).clamp(min=0.0)
        else:
            r = torch.where(torch.arange(c["V"], device=p.device) == x_at[:, None], 0.0, w)
        w = torch.where((rejected & (r.sum(-1) > 0))[:, None], r, w)
    cdf = torch.cumsum(w, -1)
    goal = s["u_bonus"][stop].double() * cdf[:, -1]
    bonus = ((cdf > goal[:, None]) & (w > 0)).int().argmax(-1)
    column = torch.arange(most + 1, device=p.device)
    padded = torch.cat([x, torch.zeros_like(x[:, :1])], 1)
    out = torch.where(column < length[:, None], padded, torch.where(column == length[:, None], bonus[:, None], -1))
    return {"accept_len": length.int(), "out_tokens": out.int(), "bonus_token": bonus.int(),
            "status": torch.zeros(B, dtype=torch.int32, device=p.device)}


def _plain_commit(s):
    c, cache, lengths = s["case"], s["cache"], s["lengths"].long()
    above, depth = s["above"], s["depth"]
    accepted = s["accepted"].long()
    # the path's node at each depth; behind the path every entry stays where it is, and all rows are taken before any is put down
    step = torch.arange(max(_tree(c)[1]) + 1, device=cache.device)
    on_path = above[accepted][:, None] & (depth == step[:, None])
    node = torch.where(on_path.any(-1), on_path.int().argmax(-1), step)
    source, target = lengths[:, None] + node, lengths[:, None] + step
    slot = lambda j: torch.gather(s["table"].long(), 1, j // c["block"]) * c["block"] + j % c["block"]  # noqa: E731
    flat = cache.view(c["caches"], -1, c["width"])
    flat[:, slot(target).flatten()] = flat[:, slot(source).flatten()]
    return {"cache": cache, "lengths": (lengths + depth[accepted] + 1).int(),
            "status": torch.zeros(c["B"], dtype=torch.int32, device="cuda")}


# ---------------------------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------------------------
def _own(s):
    from paper_2602_16994_b200 import binding
    c, op = s["case"], s["case"]["op"]
    if op == "slots":
        o = binding.cache_slots(s["lengths"], s["parent"], s["table"], s["owned"], s["ring"], s["range"], c["block"])
        return {"slots": o.slots, "positions": o.positions, "table": o.block_table, "owned": o.owned, "range": o.free_range,
                "status": o.status}
    if op == "rope":
        q = binding.norm_rope_cache(s["q"], s["k"], s["v"], s["inv_freq"], s["positions"], s["slots"], s["k_cache"],
                                    s["v_cache"], q_weight=s["wq"], k_weight=s["wk"], pairs=c["pairs"])
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if op == "attend":
        o = binding.tree_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["parent"],
                                   window=c["window"], sinks=c["sinks"])
        return {"out": o.out, "status": o.status}
    if op == "verify":
        o = binding.verify_probs(s["target"], s["draft"], s["token"], s["cu"], s["u_accept"], s["u_bonus"], s["most"])
        return {"accept_len": o.accept_len, "out_tokens": o.out_tokens, "bonus_token": o.bonus_token, "status": o.status}
    o = binding.cache_commit(s["cache"], s["accepted"], s["parent"], s["lengths"], s["table"])
    return {"cache": s["cache"], "lengths": o.lengths, "status": o.status}


def run(state):
    if own:
        return _own(state)
    return {"slots": _plain_slots, "rope": _plain_rope, "attend": _plain_attend, "verify": _plain_verify,
            "commit": _plain_commit}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------
def _exact_rope(s):
    c = s["case"]
    theta = s["positions"].reshape(-1, 1).double() * s["inv_freq"].double()
    turn = torch.polar(torch.ones_like(theta), theta)[:, None]  # e^{i t f}: a pair of a head is a complex number
    r = c["rot"]

    def turned(x, w):
        x = x.double()
        if w is not None:
            x = x / ((x * x).sum(-1, keepdim=True) / c["D"] + 1e-6).sqrt() * w.double()
        out = x.clone()
        if c["pairs"] == "halves":
            z = torch.complex(x[..., :r // 2], x[..., r // 2:r]) * turn
            out[..., :r // 2], out[..., r // 2:r] = z.real, z.imag
        else:
            z = torch.complex(x[..., 0:r:2], x[..., 1:r:2]) * turn
            out[..., 0:r:2], out[..., 1:r:2] = z.real, z.imag
        return out

    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    slots = s["slots"].reshape(-1).long()
    block, place = slots // c["block"], slots % c["block"]
    k_cache[block, place] = turned(s["k"], s["wk"])
    v_cache[block, place] = s["v"].double()
    return {"q": turned(s["q"], s["wq"]), "k_cache": k_cache, "v_cache": v_cache}


def _exact_attend(s):
    """Request by request, in chunks of keys: log-sum-exp first, then the weighted sum."""
    c, n, paths = s["case"], s["n"], _paths(s["case"])
    _, depth = _tree(c)
    G, D = c["Hq"] // c["Hkv"], c["D"]
    out = torch.empty(c["B"], n, c["Hq"], D, dtype=torch.float64, device="cuda")
    path_mask = torch.zeros(n, n, dtype=torch.bool)
    for i, nodes in enumerate(paths):
        path_mask[i, nodes] = True
    path_mask, depth = path_mask.cuda(), torch.tensor(depth, device="cuda")
    for b, length in enumerate(s["lengths"].tolist()):
        blocks = s["table"][b, :-(-(length + n) // c["block"])].long()
        k = s["k_cache"][blocks].flatten(0, 1)[:length + n].double()
        v = s["v_cache"][blocks].flatten(0, 1)[:length + n].double()
        at = torch.cat([torch.arange(length, device="cuda"), length + depth])
        mask = torch.cat([torch.ones(n, length, dtype=torch.bool, device="cuda"), path_mask], 1)
        if c["window"]:
            mask &= ((length + depth)[:, None] - at < c["window"]) | (at < c["sinks"])
        q = s["q"][b].double().view(n, c["Hkv"], G, D)
        score = torch.einsum("nhgd,lhd->hngl", q, k) * D ** -0.5
        score = torch.where(mask[None, :, None], score, torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
        weight = (score - torch.logsumexp(score, -1, keepdim=True)).exp()
        out[b] = torch.einsum("hngl,lhd->nhgd", weight, v).reshape(n, c["Hq"], D)
    return {"out": out, "status": None}


def _exact_commit(s):
    c, paths = s["case"], _paths(s["case"])
    cache = s["cache"].double()
    table, slot_of = s["table"].tolist(), lambda row, j: row[j // c["block"]] * c["block"] + j % c["block"]
    source, target = [], []
    for b, (length, node) in enumerate(zip(s["lengths"].tolist(), s["accepted"].tolist())):
        for d, i in enumerate(paths[node]):
            source.append(slot_of(table[b], length + i))
            target.append(slot_of(table[b], length + d))
    flat = cache.view(c["caches"], -1, c["width"])
    flat[:, torch.tensor(target, device="cuda")] = flat[:, torch.tensor(source, device="cuda")]
    return {"cache": cache, "lengths": None, "status": None}


def exact(case, seed):
    """Slots and tokens are whole numbers: they have to be equal, and have no value here."""
    if case["op"] in ("slots", "verify"):
        return None
    s = prepare(case, seed)
    return {"rope": _exact_rope, "attend": _exact_attend, "commit": _exact_commit}[case["op"]](s)
