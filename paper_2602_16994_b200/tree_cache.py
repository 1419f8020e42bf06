"""Paged keys and values of a batch of requests that decode with draft trees: what a decoding loop keeps around its verifier.

One step of the loop, for requests whose trees share ``parent`` (Section 2, steps 2 and 3):

    cache.begin(parent)                                   # blocks, slots and positions of the trees' nodes
    for layer in range(layers):
        q = cache.write(layer, q, k, v, inv_freq, ...)    # norm and rotation, keys and values into the cache
        y = cache.attend(layer, q)                        # every node over its request's tokens and its ancestors
    out = binding.verify_specinfer(...)                   # or another verifier
    cache.commit(out.accepted_node)                       # the accepted paths stay
    cache.evict(budget, recent)                           # (with ``weigh``) longer requests keep their heaviest entries

Requests that begin with the same tokens hold them once (``share``), and attend to them together.  Nothing in a step synchronises; lengths, tables and free
blocks live on the device.  ``lengths``, ``owned`` and ``free_range`` are replaced by the calls' results: a step captured into a graph is the same step at every replay, unless its results are copied into the tensors that it read.
"""
from __future__ import annotations

import contextlib
import operator

import torch

from . import binding


class TreeCache:
    """Caches of ``layers`` layers, a block table of ``width`` columns per request, and a ring of free blocks.

    ``storage`` is [2 * layers, num_blocks, block_size, Hkv, D]: keys of layer l at 2 * l, values behind them.  A request whose
    length is set negative takes no part in the calls; its blocks are the caller's to put back (``release``).  A row that ``release`` has
    emptied takes a new request with ``lengths[row] = 0``.

    ``weigh``: the attention weight that entries get is added up in ``weights``, over all layers that ``attend`` sees, for ``evict``.  ``protected`` [B]:
    tokens at a request's beginning that are neither weighed nor evicted; 0 again after ``release``.  After an eviction a request's positions run on: its tokens are
    ``dropped`` more than its entries.  All nodes of a step's tree add weight, ahead of the verification: those of branches that it rejects, most of a wide tree's, as
    those of the path that stays.
    """

    def __init__(self, batch, layers, num_blocks, block_size, Hkv, D, width, dtype=torch.bfloat16, device="cuda", weigh=False):
        i32 = dict(dtype=torch.int32, device=device)
        self.block_size, self.layers = block_size, layers
        self.storage = torch.zeros((2 * layers, num_blocks, block_size, Hkv, D), dtype=dtype, device=device)
        self.block_table = torch.full((batch, width), -1, **i32)
        self.lengths, self.owned = torch.zeros(batch, **i32), torch.zeros(batch, **i32)
        self.free_blocks = torch.arange(num_blocks, **i32)
        self.free_range = torch.tensor([0, num_blocks], **i32)
        self.parent = self.n_nodes = self.step = None
        self.weights = torch.zeros((num_blocks, block_size), dtype=torch.float32, device=device) if weigh else None
        self.protected = torch.zeros(batch, **i32)
        self.dropped = None                              # [B] evicted tokens, once there have been any
        self.weighed = None                              # [B] lengths of the requests whose trees add weight
        self.fresh = True                                # (no layer of the step has been attended to)
        self.prefixes = {}                               # groups that share a prefix: its blocks and the members, on the host
        self.plan = None

    def begin(self, parent, n_nodes=None, stream=None):
        """Blocks for the step's trees; their slots and positions are ``step.slots`` and ``step.positions``."""
        self.parent, self.n_nodes = parent, n_nodes
        self.step = binding.cache_slots(self.lengths, parent, self.block_table, self.owned, self.free_blocks, self.free_range,
                                        self.block_size, n_nodes, stream)
        self.owned, self.free_range = self.step.owned, self.step.free_range
        self.fresh = True
        if self.weights is not None:                     # (a refused tree has no entries of its own, and its nodes weigh nothing)
            with self._on(stream, self.lengths):
                self.weighed = torch.where(self.step.status != 0, -1, self.lengths)
        if self.dropped is not None:                     # (a node without a position keeps its -1)
            with self._on(stream, self.dropped):
                at = self.step.positions
                self.step.positions = torch.where(at < 0, at, at + self.dropped[:, None])
        if stream is not None:                           # (they may be read on the current stream too)
            for t in (self.weighed, self.step.positions):
                if t is not None:
                    t.record_stream(torch.cuda.current_stream(t.device))
        return self.step

    @contextlib.contextmanager
    def _on(self, stream, *used):
        """The tensors of a call on the stream that was named for it, the allocator told."""
        if stream is None:
            yield
            return
        side = torch.cuda.ExternalStream(stream.cuda_stream, self.lengths.device)
        for t in used:
            t.record_stream(side)
        with torch.cuda.stream(side):
            yield

    def write(self, layer, q, k, v, inv_freq, **kw):
        """``binding.norm_rope_cache`` of a layer's projections ([B * N, heads, D]) at the step's slots; returns the queries."""
        return binding.norm_rope_cache(q, k, v, inv_freq, self.step.positions, self.step.slots, self.storage[2 * layer],
                                       self.storage[2 * layer + 1], **kw)

    def attend(self, layer, q, **kw):
        """``binding.tree_attention`` of a layer ([B,N,Hq,D]), ``binding.prefix_attention`` where requests share prefixes."""
        if self.weights is None:
            return self._attend(layer, q, kw)
        if kw.get("window"):
            raise RuntimeError("entries are not weighed under a window")
        wanted = kw.get("want_lse", False)
        got = self._attend(layer, q, dict(kw, want_lse=True))
        self.weigh_status = binding.cache_weights(self.weights, q, self.storage[2 * layer], got.lse, self.block_table, self.weighed, self.parent,
                                                  self.n_nodes, scale=kw.get("scale"), protected=self.protected, fresh=self.fresh,
                                                  stream=kw.get("stream"))
        self.fresh = False
        if not wanted:
            got.lse = None
        return got

    def _attend(self, layer, q, kw):
        k, v = self.storage[2 * layer], self.storage[2 * layer + 1]
        if self.plan is None or kw.get("window"):
            return binding.tree_attention(q, k, v, self.block_table, self.lengths, self.parent, self.n_nodes, **kw)
        return binding.prefix_attention(q, k, v, self.block_table, self.lengths, self.parent, self.plan, self.n_nodes,
                                        **{x: y for x, y in kw.items() if x not in ("window", "sinks")})

    def commit(self, accepted_node, stream=None):
        """The accepted paths' entries behind the committed tokens, in all layers; new lengths.  A request whose ``begin`` was refused
        (``step.status``) keeps its length: nothing of its tree was written, though its last block may have room for the path."""
        status, caches = self.step.status, [self.storage]
        if self.weights is not None:
            caches.insert(0, self.weights[None, :, :, None])
        if stream is None:
            accepted = accepted_node.masked_fill(status != 0, -1)
            for c in caches:
                done = binding.cache_commit(c, accepted, self.parent, self.lengths, self.block_table, self.n_nodes)
            done.status = torch.maximum(done.status, status)
        else:                                            # (the allocator is told of both streams, as the calls tell it)
            side, current = torch.cuda.ExternalStream(stream.cuda_stream, status.device), torch.cuda.current_stream(status.device)
            with torch.cuda.stream(side):
                accepted = accepted_node.masked_fill(status != 0, -1)
            accepted_node.record_stream(side)
            for c in caches:
                done = binding.cache_commit(c, accepted, self.parent, self.lengths, self.block_table, self.n_nodes, stream)
            with torch.cuda.stream(side):
                done.status = torch.maximum(done.status, status)
            status.record_stream(side)
            done.status.record_stream(current)
        self.lengths = done.lengths
        return done

    def evict(self, budget, recent=0, stream=None):
        """``binding.cache_evict`` of all layers, between two steps: requests of more than ``budget`` tokens keep that many.

        What lies behind the first entry that goes moves, in all layers, however few go: calls every so many steps, to a budget so much lower, cost less
        than one a step (16 requests of 4096 tokens, 16 caches of 1 KB a token: 290 us for 1 token too many, 490 for 16, 500 for 4096).
        """
        if self.weights is None:
            raise RuntimeError("evict needs a cache made with weigh=True")
        done = binding.cache_evict(self.storage, self.weights, self.lengths, self.block_table, self.owned, self.free_blocks, self.free_range, budget,
                                   recent, self.protected, stream)
        current = torch.cuda.current_stream(done.lengths.device) if stream is not None else None
        with self._on(stream, self.lengths, *([] if self.dropped is None else [self.dropped])):
            fewer = torch.where(self.lengths >= 0, self.lengths - done.lengths, 0)
            self.dropped = fewer if self.dropped is None else self.dropped + fewer
        if current is not None:
            self.dropped.record_stream(current)
        self.lengths, self.owned, self.free_range = done.lengths, done.owned, done.free_range
        return done

    def _row(self, x):
        """A request's row as its number from 0 on, by which groups know their members: of a negative one (from the end) or a tensor too."""
        x, batch = operator.index(x), self.lengths.numel()
        if not -batch <= x < batch:
            raise IndexError(f"there is no row {x} among {batch}")
        return x % batch

    def share(self, request, rows):
        """Empty ``rows`` begin with the tokens of ``request`` so far, as many as fill whole blocks, which all of them then hold together: what they attend
        to there is read once.  Returns the number of tokens; the ones behind are the rows' own to write again.  Between two steps; for the
        rare beginning of a request: reads tables on the host.

        A group keeps the members that it began with until they end: no rows join it later, and its last member is protected as it was.  Requests that come
        later share with one that is in no group, which has the prompt written for itself once more.
        """
        request, rows = self._row(request), [self._row(x) for x in rows]
        n = int(self.lengths[request]) // self.block_size
        if any(request in members for _, members in self.prefixes.values()) or (self.dropped is not None and int(self.dropped[request])):
            raise RuntimeError("a request that shares a prefix already, or has been cut, is not shared again")
        if n < 1:
            raise RuntimeError("the request has no whole block yet")
        if any(int(self.owned[x]) or x == request for x in rows) or len(set(rows)) != len(rows):
            raise RuntimeError("the rows must be empty, and other ones")
        blocks = self.block_table[request, :n].clone()
        lengths, owned, protected = self.lengths.clone(), self.owned.clone(), self.protected.clone()
        for x in rows:
            self.block_table[x, :n] = blocks
            lengths[x], owned[x] = n * self.block_size, n
        for x in rows + [request]:
            protected[x] = protected[x].clamp(min=n * self.block_size)
        self.lengths, self.owned, self.protected = lengths, owned, protected
        self.prefixes[max(self.prefixes, default=-1) + 1] = (blocks, {request, *rows})
        self._plan()
        return n * self.block_size

    def _plan(self):
        """The plan of the groups that have members left."""
        if not self.prefixes:
            self.plan = None
            return
        i32 = dict(dtype=torch.int32, device=self.lengths.device)
        group = torch.full((self.lengths.numel(),), -1, **i32)
        table = torch.full((len(self.prefixes), max(b.numel() for b, _ in self.prefixes.values())), -1, **i32)
        for g, (blocks, members) in enumerate(self.prefixes.values()):
            group[sorted(members)] = g
            table[g, :blocks.numel()] = blocks
        self.plan = binding.prefix_plan(group, torch.tensor([b.numel() for b, _ in self.prefixes.values()], **i32), table,
                                        sum(len(m) for _, m in self.prefixes.values()))

    def release(self, request):
        """Puts the blocks of a request that has ended back behind the free ones; those of a shared prefix when its last member ends.  For the rare end of a
        request: reads its row on the host."""
        request = self._row(request)
        n, (first, count), size = int(self.owned[request]), self.free_range.tolist(), self.free_blocks.numel()
        keep = 0
        for g, (blocks, members) in list(self.prefixes.items()):
            if request in members:
                members.discard(request)
                if members:
                    keep = blocks.numel()
                else:
                    del self.prefixes[g]
                self._plan()
        at = (first + count + torch.arange(n - keep, device=self.free_blocks.device)) % size
        self.free_blocks[at] = self.block_table[request, keep:n]
        self.block_table[request] = -1
        self.free_range = torch.tensor([first, count + n - keep], dtype=torch.int32, device=self.free_blocks.device)
        lengths, owned = self.lengths.clone(), self.owned.clone()
        lengths[request], owned[request] = -1, 0
        self.lengths, self.owned = lengths, owned
        protected = self.protected.clone()
        protected[request] = 0
        self.protected = protected
        if self.dropped is not None:
            dropped = self.dropped.clone()
            dropped[request] = 0
            self.dropped = dropped
