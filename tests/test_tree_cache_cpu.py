"""TreeCache's own part of a step, on the CPU: the calls on the device are stood in for by their restatements in 64 bits."""
from types import SimpleNamespace

import pytest
import torch

from . import step_ref as ref
from paper_2602_16994_b200 import tree_cache

I32 = torch.int32


@pytest.fixture
def calls(monkeypatch):
    def cache_slots(lengths, parent, table, owned, ring, free_range, block, n_nodes=None, stream=None):
        r = ref.cache_slots(lengths, parent, table, owned, ring, free_range, block, n_nodes)
        table.copy_(r["block_table"])
        return SimpleNamespace(**r)

    def cache_commit(cache, accepted, parent, lengths, table, n_nodes=None, stream=None):
        r = ref.commit(cache, accepted, parent, lengths, table, n_nodes)
        cache.copy_(r["cache"])
        return SimpleNamespace(lengths=r["lengths"], status=r["status"])

    monkeypatch.setattr(tree_cache, "binding", SimpleNamespace(cache_slots=cache_slots, cache_commit=cache_commit))


def put(cache, marks):
    """What write() does with a step's rows: entries with a slot get their mark."""
    flat = cache.storage.flatten(1, 2)
    for slot, mark in zip(cache.step.slots.flatten().tolist(), marks.flatten().tolist()):
        if slot >= 0:
            flat[:, slot] = mark


def committed(cache, b):
    at = torch.arange(int(cache.lengths[b]))
    return cache.storage[0].flatten(0, 1)[cache.block_table[b, at // cache.block_size].long() * cache.block_size + at % cache.block_size, 0, 0]


def test_a_refused_step_is_not_committed(calls):
    """14 tokens in a block of 16 and no free block: the tree of 10 nodes is written nowhere, though its root and first child have room."""
    cache = tree_cache.TreeCache(1, 1, 1, 16, 1, 1, width=4, dtype=torch.float32, device="cpu")
    parent = torch.tensor([-1, 0, 1, 2, 0, 4, 5, 0, 7, 8], dtype=I32)
    cache.begin(torch.arange(-1, 13, dtype=I32))                 # a prompt of 14 tokens
    cache.commit(torch.tensor([13], dtype=I32))
    assert cache.lengths.tolist() == [14]
    for node in (0, 1, 3, -1):
        step = cache.begin(parent)
        assert step.status.tolist() == [ref.BLOCKS] and bool((step.slots == -1).all())
        done = cache.commit(torch.tensor([node], dtype=I32))
        assert cache.lengths.tolist() == [14] and done.lengths.tolist() == [14]
        assert done.status.tolist() == [ref.BLOCKS]


def test_a_pool_that_runs_dry_and_is_filled_again(calls):
    """Every committed entry is one that was written, in each request, before, while and after the pool is dry."""
    g = torch.Generator().manual_seed(0)
    B, block, blocks = 3, 8, 9
    parent = torch.tensor([-1, 0, 1, 2, 0, 4, 5, 0, 7, 8], dtype=I32)
    tree_paths = ref.paths(parent.tolist())
    cache = tree_cache.TreeCache(B, 1, blocks, block, 1, 1, width=8, dtype=torch.float32, device="cpu")
    kept, refused, mark = [[] for _ in range(B)], 0, 1.0
    for step in range(14):
        if step == 9:
            cache.release(2)
            kept[2] = []
        s = cache.begin(parent)
        marks = mark + torch.arange(B * 10, dtype=torch.float32).view(B, 10)
        mark += B * 10
        put(cache, marks)
        node = torch.randint(0, 10, (B,), generator=g).int()
        done = cache.commit(node)
        for b in range(B):
            if s.status[b]:
                refused += 1
                assert done.status[b] == s.status[b]
            elif cache.lengths[b] >= 0:
                kept[b] += [float(marks[b, i]) for i in tree_paths[int(node[b])]]
            if cache.lengths[b] >= 0:
                assert committed(cache, b).tolist() == kept[b]
    assert refused > 3 and int((cache.lengths >= 0).sum()) == 2


def test_a_bad_tree_is_not_committed(calls):
    cache = tree_cache.TreeCache(2, 1, 4, 8, 1, 1, width=2, dtype=torch.float32, device="cpu")
    parent = torch.tensor([[-1, 0, 1], [-1, 1, 0]], dtype=I32)
    assert cache.begin(parent).status.tolist() == [0, ref.TOPOLOGY]
    done = cache.commit(torch.tensor([2, 2], dtype=I32))
    assert done.lengths.tolist() == [3, 0] and done.status.tolist() == [0, ref.TOPOLOGY]
