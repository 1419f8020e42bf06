"""Paged keys and values of a batch of requests that decode with draft trees: what a decoding loop keeps around its verifier.

One step of the loop, for requests whose trees share ``parent`` (Section 2, steps 2 and 3):

    cache.begin(parent)                                   # blocks, slots and positions of the trees' nodes
    for layer in range(layers):
        q = cache.write(layer, q, k, v, inv_freq, ...)    # norm and rotation, keys and values into the cache
        y = cache.attend(layer, q)                        # every node over its request's tokens and its ancestors
    out = binding.verify_specinfer(...)                   # or another verifier
    cache.commit(out.accepted_node)                       # the accepted paths stay

Nothing synchronises; lengths, tables and free blocks live on the device.  ``lengths``, ``owned`` and ``free_range`` are replaced by the
calls' results: a step captured into a graph is the same step at every replay, unless its results are copied into the tensors that it read.
"""
from __future__ import annotations

import torch

from . import binding


class TreeCache:
    """Caches of ``layers`` layers, a block table of ``width`` columns per request, and a ring of free blocks.

    ``storage`` is [2 * layers, num_blocks, block_size, Hkv, D]: keys of layer l at 2 * l, values behind them.  A request whose
    length is set negative takes no part in the calls; its blocks are the caller's to put back (``release``).  A row that ``release`` has
    emptied takes a new request with ``lengths[row] = 0``.
    """

    def __init__(self, batch, layers, num_blocks, block_size, Hkv, D, width, dtype=torch.bfloat16, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.block_size, self.layers = block_size, layers
        self.storage = torch.zeros((2 * layers, num_blocks, block_size, Hkv, D), dtype=dtype, device=device)
        self.block_table = torch.full((batch, width), -1, **i32)
        self.lengths, self.owned = torch.zeros(batch, **i32), torch.zeros(batch, **i32)
        self.free_blocks = torch.arange(num_blocks, **i32)
        self.free_range = torch.tensor([0, num_blocks], **i32)
        self.parent = self.n_nodes = self.step = None

    def begin(self, parent, n_nodes=None, stream=None):
        """Blocks for the step's trees; their slots and positions are ``step.slots`` and ``step.positions``."""
        self.parent, self.n_nodes = parent, n_nodes
        self.step = binding.cache_slots(self.lengths, parent, self.block_table, self.owned, self.free_blocks, self.free_range,
                                        self.block_size, n_nodes, stream)
        self.owned, self.free_range = self.step.owned, self.step.free_range
        return self.step

    def write(self, layer, q, k, v, inv_freq, **kw):
        """``binding.norm_rope_cache`` of a layer's projections ([B * N, heads, D]) at the step's slots; returns the queries."""
        return binding.norm_rope_cache(q, k, v, inv_freq, self.step.positions, self.step.slots, self.storage[2 * layer],
                                       self.storage[2 * layer + 1], **kw)

    def attend(self, layer, q, **kw):
        """``binding.tree_attention`` of a layer ([B,N,Hq,D])."""
        return binding.tree_attention(q, self.storage[2 * layer], self.storage[2 * layer + 1], self.block_table, self.lengths, self.parent,
                                      self.n_nodes, **kw)

    def commit(self, accepted_node, stream=None):
        """The accepted paths' entries behind the committed tokens, in all layers; new lengths.  A request whose ``begin`` was refused
        (``step.status``) keeps its length: nothing of its tree was written, though its last block may have room for the path."""
        status = self.step.status
        if stream is None:
            accepted = accepted_node.masked_fill(status != 0, -1)
            done = binding.cache_commit(self.storage, accepted, self.parent, self.lengths, self.block_table, self.n_nodes)
            done.status = torch.maximum(done.status, status)
        else:                                            # (the allocator is told of both streams, as the calls tell it)
            side, current = torch.cuda.ExternalStream(stream.cuda_stream, status.device), torch.cuda.current_stream(status.device)
            with torch.cuda.stream(side):
                accepted = accepted_node.masked_fill(status != 0, -1)
            accepted_node.record_stream(side)
            done = binding.cache_commit(self.storage, accepted, self.parent, self.lengths, self.block_table, self.n_nodes, stream)
            with torch.cuda.stream(side):
                done.status = torch.maximum(done.status, status)
            status.record_stream(side)
            done.status.record_stream(current)
        self.lengths = done.lengths
        return done

    def release(self, request):
        """Puts the blocks of a request that has ended back behind the free ones.  For the rare end of a request: reads its row on the host."""
        n, (first, count), size = int(self.owned[request]), self.free_range.tolist(), self.free_blocks.numel()
        at = (first + count + torch.arange(n, device=self.free_blocks.device)) % size
        self.free_blocks[at] = self.block_table[request, :n]
        self.block_table[request] = -1
        self.free_range = torch.tensor([first, count + n], dtype=torch.int32, device=self.free_blocks.device)
        lengths, owned = self.lengths.clone(), self.owned.clone()
        lengths[request], owned[request] = -1, 0
        self.lengths, self.owned = lengths, owned
