"""Plain restatements, in Python and 64 bits on the CPU, of log probabilities and of eviction from a paged cache, written from the definitions
in the C header."""
import math

import torch

TOPOLOGY, TOKEN, NONFINITE, PAGE, BLOCKS = 1, 2, 3, 5, 6


def ranked(row, top):
    """Indices of the `top` largest, of equal ones the lower first."""
    return torch.sort(row.double() + 0.0, descending=True, stable=True).indices[:top]


def logprobs(logits, tokens, temperature=1.0, top=0):
    """Rows [R,V] and tokens [R,K]."""
    R, V = logits.shape
    K = tokens.shape[1]
    out = dict(logprob=torch.zeros(R, K, dtype=torch.float64), entropy=torch.zeros(R, dtype=torch.float64),
               top_tokens=torch.full((R, top), -1, dtype=torch.int32), top_logprobs=torch.zeros(R, top, dtype=torch.float64),
               status=torch.zeros(R, dtype=torch.int32))
    for r in range(R):
        z = logits[r].double()
        if not bool((z < math.inf).all()) or float(z.max()) == -math.inf:
            for name in ("logprob", "entropy", "top_logprobs"):
                out[name][r] = math.nan
            out["logprob"][r][tokens[r] == -1] = 0.0
            out["status"][r] = NONFINITE
            continue
        d = (z - z.max()) / temperature
        log = d - d.exp().sum().log()
        p = log.exp()
        out["entropy"][r] = -torch.where(p > 0, p * log, 0.0).sum()
        for k in range(K):
            t = int(tokens[r, k])
            if 0 <= t < V:
                out["logprob"][r, k] = log[t]
            elif t != -1:
                out["logprob"][r, k] = math.nan
                out["status"][r] = TOKEN
        best = ranked(logits[r], top)
        out["top_tokens"][r], out["top_logprobs"][r] = best.int(), log[best]
    return out


def path_of(parent, node):
    """Nodes from the root to `node`, or None."""
    out = []
    while node > 0:
        out.append(node)
        up = int(parent[node])
        if not 0 <= up < node:
            return None
        node = up
    return None if int(parent[0]) != -1 else [0] + out[::-1]


def path_logprobs(logits, accepted, tokens, parent, temperature=1.0, top=0):
    B, N, V = logits.shape
    out = dict(logprob=torch.zeros(B, N, dtype=torch.float64), entropy=torch.zeros(B, N, dtype=torch.float64),
               top_tokens=torch.full((B, N, top), -1, dtype=torch.int32), top_logprobs=torch.zeros(B, N, top, dtype=torch.float64),
               status=torch.zeros(B, N, dtype=torch.int32))
    for b in range(B):
        a = int(accepted[b])
        if a == -1:
            continue
        nodes = path_of(parent[b] if parent.dim() == 2 else parent, a) if -1 <= a < N else None
        if nodes is None:
            out["status"][b] = TOPOLOGY
            continue
        got = logprobs(logits[b, nodes], tokens[b, :len(nodes), None], temperature, top)
        for name, x in got.items():
            out[name][b, :len(nodes)] = x[:, 0] if name == "logprob" else x
    return out


def evict(cache, weights, lengths, table, owned, ring, free_range, budget, recent=0, protected=None):
    """All arrays of a call, after it; and the entries that each request keeps."""
    cache, weights, ring = cache.clone(), weights.clone(), ring.clone()
    B, (blocks, block), width = len(lengths), cache.shape[1:3], table.shape[1]
    lengths_out, owned_out, status = lengths.clone(), owned.clone(), torch.zeros(B, dtype=torch.int32)
    begin, count = (int(x) for x in free_range)
    room = len(ring) - count if 0 <= begin < len(ring) and 0 <= count <= len(ring) else 0
    put, dry, kept = 0, False, []
    for b in range(B):
        n, own, p = int(lengths[b]), int(owned[b]), 0 if protected is None else int(protected[b])
        kept.append(list(range(max(0, n))))
        if n <= budget:
            continue
        ids = table[b, :own].tolist() if 0 <= own <= width else None
        if ids is None or -(-n // block) > own or any(not 0 <= x < blocks for x in ids):
            status[b] = PAGE
            continue
        if not 0 <= p <= budget:
            status[b] = TOPOLOGY
            continue
        r = min(recent, budget - p)
        place = [(ids[j // block], j % block) for j in range(n)]
        w = [float(weights[x]) for x in place]
        w = [-math.inf if math.isnan(x) else x for x in w]
        nan = [math.isnan(float(weights[x])) for x in place]
        middle = sorted(range(p, n - r), key=lambda j: (nan[j], -w[j], j))[:budget - p - r]
        keep = sorted(list(range(p)) + middle + list(range(n - r, n)))
        kept[b] = keep
        rows, old = [cache[:, x[0], x[1]].clone() for x in (place[j] for j in keep)], [weights[place[j]].clone() for j in keep]
        for i, (row, x) in enumerate(zip(rows, old)):
            cache[:, place[i][0], place[i][1]] = row
            weights[place[i]] = x
        lengths_out[b] = budget
        stay = -(-budget // block)
        gone = ids[stay:]
        if gone and (dry or put + len(gone) > room):
            dry = True
            status[b] = BLOCKS
            continue
        for i, x in enumerate(gone):
            ring[(begin + count + put + i) % len(ring)] = x
        put += len(gone)
        owned_out[b] = stay
    range_out = torch.tensor([begin, count + put] if len(ring) else [0, 0], dtype=torch.int32)
    return dict(cache=cache, weights=weights, free_blocks=ring, lengths=lengths_out, owned=owned_out, free_range=range_out, status=status), kept


def weights(w, q, k_cache, lse, table, lengths, parent, n_nodes=None, scale=None, protected=None, fresh=False):
    """weights after the call, status, and per entry the bound's ingredients: what was added, sum e (|score| + |lse|) and sum e sum_d |q_d k_d| scale."""
    B, N, Hq, D = q.shape
    blocks, block, Hkv, _ = k_cache.shape
    G, scale = Hq // Hkv, D ** -0.5 if scale is None else scale
    w = w.double().clone()
    got, size, reach = (torch.zeros_like(w) for _ in range(3))
    status = torch.zeros(B, dtype=torch.int32)
    for b in range(B):
        length, n = int(lengths[b]), N if n_nodes is None else int(n_nodes[b])
        p = 0 if protected is None else max(0, int(protected[b]))
        if length < 0:
            continue
        row = parent[b] if parent.dim() == 2 else parent
        seen_by = [path_of(row, i) for i in range(n)] if 0 <= n <= N else None
        if seen_by is None or any(x is None for x in seen_by):
            status[b] = TOPOLOGY
            continue
        if n == 0:
            continue
        sees = torch.zeros(n, length + n, dtype=torch.bool)
        sees[:, :length] = True
        for i, nodes in enumerate(seen_by):
            sees[i, [length + x for x in nodes]] = True
        j = torch.arange(min(p, length + n), length + n)
        cols = j // block
        ids = torch.where(cols < table.shape[1], table[b, cols.clamp(max=table.shape[1] - 1)], -1).long()
        good = (ids >= 0) & (ids < blocks)
        if not bool(good.all()):
            status[b] = PAGE
        j, ids = j[good], ids[good]
        k = k_cache[ids, j % block].double().repeat_interleave(G, 1)
        x = q[b, :n].double()
        score = torch.einsum("nhd,jhd->nhj", x, k) * scale
        l = lse[b, :n].double()[:, :, None]
        y = score - l
        counts = sees[:, None, j] & l.isfinite() & ~y.isnan()
        e = torch.where(counts, y.exp(), 0.0)
        at = (ids, j % block)
        if fresh:
            tree = j >= length
            w[ids[tree], (j % block)[tree]] = 0.0
        w[at] += e.sum((0, 1))
        got[at] = e.sum((0, 1))
        size[at] = torch.where(counts, e * (score.abs() + l.abs()), 0.0).sum((0, 1))
        reach[at] = torch.where(counts, e * (torch.einsum("nhd,jhd->nhj", x.abs(), k.abs()) * scale), 0.0).sum((0, 1))
    return dict(weights=w, status=status, got=got, size=size, reach=reach)
