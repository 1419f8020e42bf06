"""Plain restatements, in Python and 64 bits on the CPU, of the operators around a verification: what each output has to be, request by
request, written from the definitions in the C header."""
import math

import torch

TOPOLOGY, TOKEN, NONFINITE, PAGE, BLOCKS = 1, 2, 3, 5, 6


def paths(parent):
    """The nodes from the root to each node, or None for a bad tree."""
    out = []
    for i, p in enumerate(parent):
        if (i == 0 and p != -1) or (i > 0 and not 0 <= p < i):
            return None
        out.append((out[p] if i else []) + [i])
    return out


def _row(parent, b):
    return (parent[b] if parent.dim() == 2 else parent).tolist()


def cache_slots(lengths, parent, table, owned, ring, free_range, block, n_nodes=None):
    B, N, width = len(lengths), parent.shape[-1], table.shape[1]
    table = table.clone()
    slots, positions = torch.full((B, N), -1, dtype=torch.int32), torch.full((B, N), -1, dtype=torch.int32)
    status, owned_out = torch.zeros(B, dtype=torch.int32), owned.clone()
    begin, count = (int(x) for x in free_range)
    if not (0 <= begin < len(ring) and 0 <= count <= len(ring)):
        begin, count = 0, 0
    taken, dry = 0, False
    for b in range(B):
        length, n = int(lengths[b]), N if n_nodes is None else int(n_nodes[b])
        if length < 0:
            continue
        good_n = 0 <= n <= N
        n = n if good_n else 0
        need, own = -(-(length + n) // block), int(owned[b])
        fits = 0 <= own <= width and need <= width and length + n < 2**31
        lack = max(0, need - own) if fits else 0
        got = lack > 0 and not dry and taken + lack <= count
        dry |= lack > 0 and not got
        if got:
            for i in range(lack):
                table[b, own + i] = ring[(begin + taken + i) % len(ring)]
            taken += lack
            owned_out[b] = own + lack
        placed, page = fits and (lack == 0 or got), False
        tree = paths(_row(parent, b)[:n])
        for i in range(n):
            if placed:
                at = length + i
                k = int(table[b, at // block])
                s = k * block + at % block
                if k < 0 or s > 2**31 - 1:
                    page = True
                else:
                    slots[b, i] = s
            if placed and tree is not None:
                positions[b, i] = length + len(tree[i]) - 1
        status[b] = TOPOLOGY if not good_n else BLOCKS if not placed else PAGE if page else TOPOLOGY if tree is None else 0
    return dict(slots=slots, positions=positions, block_table=table, owned=owned_out, status=status,
                free_range=torch.tensor([(begin + taken) % max(1, len(ring)), count - taken], dtype=torch.int32))


def norm_rope(x, weight, inv_freq, positions, eps, pairs):
    """(rotated rows, |a| + |b| of each entry's pair) in 64 bits; x [T,H,D]."""
    y = x.double()
    if weight is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    r = 2 * len(inv_freq)
    angle = positions.double().view(-1, 1, 1) * inv_freq.double()
    c, s = angle.cos(), angle.sin()
    out, size = y.clone(), y.abs()
    i = torch.arange(r // 2)
    first, second = (i, i + r // 2) if pairs == "halves" else (2 * i, 2 * i + 1)
    a, b = y[..., first], y[..., second]
    out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    size[..., first] = size[..., second] = a.abs() + b.abs()
    return out, size


def attention(q, k_cache, v_cache, block_table, lengths, parent, n_nodes=None, scale=None, window=0, sinks=0):
    """out, lse, status, and per entry the bound's ingredients: sum_j p_j |v_j| and the largest sum_d |q_d k_d| scale of a row."""
    B, N, Hq, D = q.shape
    P, block, Hkv, _ = k_cache.shape
    G, scale = Hq // Hkv, D ** -0.5 if scale is None else scale
    out, mass = torch.zeros(B, N, Hq, D, dtype=torch.float64), torch.zeros(B, N, Hq, D, dtype=torch.float64)
    lse, reach = torch.full((B, N, Hq), -math.inf, dtype=torch.float64), torch.zeros(B, N, Hq, dtype=torch.float64)
    status, live = torch.zeros(B, dtype=torch.int32), torch.zeros(B, N, dtype=torch.bool)
    for b in range(B):
        length, n = int(lengths[b]), N if n_nodes is None else int(n_nodes[b])
        if length < 0:
            continue
        if not 0 <= n <= N:
            status[b] = TOPOLOGY
            continue
        live[b, :n] = True
        tree = paths(_row(parent, b)[:n])
        keys = length + n
        cols = torch.arange(keys) // block
        ids = torch.where(cols < block_table.shape[1], block_table[b, cols.clamp(max=block_table.shape[1] - 1)], -1).long()
        good = (ids >= 0) & (ids < P)
        seen_by_any = torch.arange(keys) >= length
        at = torch.arange(keys)
        seen_by_any |= (window == 0) | (at < sinks) | (at > length - window)
        if tree is None:
            status[b] = TOPOLOGY
            continue
        if not bool(good[seen_by_any].all()):
            status[b] = PAGE
        depth = torch.tensor([len(t) - 1 for t in tree], dtype=torch.long)
        position = torch.cat([torch.arange(length), length + depth])
        for i in range(n):
            seen = torch.zeros(keys, dtype=torch.bool)
            seen[:length] = True
            seen[[length + x for x in tree[i]]] = True
            if window:
                seen &= (position > length + depth[i] - window) | (position < sinks)
            seen &= good
            j = seen.nonzero().flatten()
            if not len(j):
                continue
            k = k_cache[ids[j], j % block].double().repeat_interleave(G, 1)
            v = v_cache[ids[j], j % block].double().repeat_interleave(G, 1)
            x = q[b, i].double()
            score = torch.einsum("hd,jhd->hj", x, k) * scale
            reach[b, i] = (torch.einsum("hd,jhd->hj", x.abs(), k.abs()) * abs(scale)).amax(-1)
            lse[b, i] = torch.logsumexp(score, -1)
            p = (score - lse[b, i][:, None]).exp()
            out[b, i] = torch.einsum("hj,jhd->hd", p, v)
            mass[b, i] = torch.einsum("hj,jhd->hd", p, v.abs())
    return dict(out=out, lse=lse, status=status, mass=mass, reach=reach, live=live)


def commit(cache, accepted, parent, lengths, table, n_nodes=None):
    cache, lengths_out, status = cache.clone(), lengths.clone(), torch.zeros(len(lengths), dtype=torch.int32)
    block, blocks = cache.shape[2], cache.shape[1]
    for b in range(len(lengths)):
        length, acc = int(lengths[b]), int(accepted[b])
        n = parent.shape[-1] if n_nodes is None else int(n_nodes[b])
        if length < 0 or acc == -1:
            if length >= 0 and (not 0 <= n <= parent.shape[-1] or paths(_row(parent, b)[:n]) is None):
                status[b] = TOPOLOGY
            continue
        tree = paths(_row(parent, b)[:n]) if 0 <= n <= parent.shape[-1] else None
        if tree is None or not 0 <= acc < n:
            status[b] = TOPOLOGY
            continue
        moves = [(i, d) for d, i in enumerate(tree[acc]) if i != d]

        def place(at):
            k = int(table[b, at // block]) if at // block < table.shape[1] else -1
            return (k, at % block) if 0 <= k < blocks else None

        spots = [(place(length + i), place(length + d)) for i, d in moves]
        if any(x is None or y is None for x, y in spots) or any(place(length + d) is None for d in range(len(tree[acc]))):
            status[b] = PAGE
            continue
        rows = [cache[:, x[0], x[1]].clone() for x, _ in spots]
        for r, (_, y) in zip(rows, spots):
            cache[:, y[0], y[1]] = r
        lengths_out[b] = length + len(tree[acc])
    return dict(cache=cache, lengths=lengths_out, status=status)


def verify_probs(target, draft, token, cu, u_accept, u_bonus, most):
    """All in 64 bits; also the smallest distance of a decision's uniform to its threshold."""
    T, B, V = len(token), len(cu) - 1, target.shape[1]
    length, bonus = torch.full((B,), -1, dtype=torch.int32), torch.full((B,), -1, dtype=torch.int32)
    out, status = torch.full((B, most + 1), -1, dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
    margin = math.inf
    for b in range(B):
        first, n = int(cu[b]), int(cu[b + 1]) - int(cu[b])
        if first < 0 or n < 0 or first + n > T or n > most:
            status[b] = TOPOLOGY
            continue
        a, why = 0, 0
        while a < n:
            x = int(token[first + a])
            if not 0 <= x < V:
                why = TOKEN
                break
            p = float(target[first + b + a, x])
            q = 1.0 if draft is None else float(draft[first + a, x])
            if not (0 <= p < math.inf and 0 <= q < math.inf):
                why = NONFINITE
                break
            r = min(1.0, (p / q if q > 0 else 1.0) if p > 0 else 0.0)
            u = float(u_accept[first + a])
            if u > 0 and r < 1:                                   # (0 against a ratio, and any uniform against 1, is exact)
                margin = min(margin, abs(u - r))
            if not u < r:
                break
            a += 1
        if why:
            status[b] = why
            continue
        p = target[first + b + a].double()
        w = p.clone()
        if a < n:
            if draft is None:
                w[int(token[first + a])] = 0
            else:
                w = p - draft[first + a].double()
            w = torch.where(w <= 0, 0.0, w)
            if float(w.sum()) == 0:
                w = p
        w = torch.where(w <= 0, 0.0, w)
        total = float(w.sum())
        if not 0 < total < math.inf:
            status[b] = NONFINITE
            continue
        c = torch.cumsum(w, 0)
        goal = float(u_bonus[first + b + a]) * float(c[-1])
        hit = ((c > goal) & (w > 0)).nonzero().flatten()
        t = int(hit[0]) if len(hit) else int((w > 0).nonzero().flatten()[-1])
        if goal > 0:
            margin = min(margin, abs(float(c[t]) - goal) / total, abs(goal - float(c[t] - w[t])) / total)
        length[b], bonus[b] = a, t
        out[b, :a] = token[first:first + a].int()
        out[b, a] = t
    return dict(accept_len=length, out_tokens=out, bonus_token=bonus, status=status, margin=margin)
