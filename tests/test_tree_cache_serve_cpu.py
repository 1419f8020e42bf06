"""TreeCache's own part of shared prefixes and evictions, on the CPU: the calls on the device are stood in for by their restatements in 64 bits."""
from types import SimpleNamespace

import pytest
import torch

from . import serve_ref, step_ref as ref
from .test_tree_cache_cpu import committed, put
from paper_2602_16994_b200 import binding, tree_cache

I32 = torch.int32


@pytest.fixture
def calls(monkeypatch):
    seen = SimpleNamespace(plans=0)

    def cache_slots(lengths, parent, table, owned, ring, free_range, block, n_nodes=None, stream=None):
        r = ref.cache_slots(lengths, parent, table, owned, ring, free_range, block, n_nodes)
        table.copy_(r["block_table"])
        return SimpleNamespace(**r)

    def cache_commit(cache, accepted, parent, lengths, table, n_nodes=None, stream=None):
        r = ref.commit(cache, accepted, parent, lengths, table, n_nodes)
        cache.copy_(r["cache"])
        return SimpleNamespace(lengths=r["lengths"], status=r["status"])

    def cache_evict(cache, weights, lengths, table, owned, ring, free_range, budget, recent=0, protected=None, stream=None):
        r, _ = serve_ref.evict(cache, weights, lengths, table, owned, ring, free_range, budget, recent, protected)
        cache.copy_(r["cache"])
        weights.copy_(r["weights"])
        ring.copy_(r["free_blocks"])
        return SimpleNamespace(**r)

    def prefix_plan(*args):
        seen.plans += 1
        return binding.prefix_plan(*args)

    monkeypatch.setattr(tree_cache, "binding", SimpleNamespace(cache_slots=cache_slots, cache_commit=cache_commit, cache_evict=cache_evict,
                                                               prefix_plan=prefix_plan))
    return seen


def step(cache, parent, mark, node):
    s = cache.begin(parent)
    marks = mark + torch.arange(s.slots.numel(), dtype=torch.float32).view(s.slots.shape)
    put(cache, marks)
    if cache.weights is not None:                                # (what attention would have added)
        flat = cache.weights.view(-1)
        for slot, x in zip(s.slots.flatten().tolist(), marks.flatten().tolist()):
            if slot >= 0:
                flat[slot] = x % 13
    cache.commit(torch.tensor(node, dtype=I32))
    return s, marks


def test_evictions_between_steps(calls):
    """What is committed is what was kept and then written; positions run on; freed blocks come back."""
    cache = tree_cache.TreeCache(2, 1, 12, 4, 1, 1, width=10, dtype=torch.float32, device="cpu", weigh=True)
    cache.protected[:] = torch.tensor([2, 0], dtype=I32)
    kept, position = [[], []], [0, 0]
    parent = torch.arange(-1, 4, dtype=I32)
    for i in range(12):
        s, marks = step(cache, parent, 100.0 * i, [4, 2])
        assert s.status.tolist() == [0, 0]
        for b, n in enumerate((5, 3)):
            assert s.positions[b].tolist() == list(range(position[b], position[b] + 5))
            position[b] += n
            kept[b] += marks[b, :n].tolist()
            assert committed(cache, b).tolist() == kept[b]
        before = [list(x) for x in kept]
        w = [serve_weights(cache, b) for b in range(2)]
        cache.evict(9, recent=3)
        for b, p in enumerate((2, 0)):
            n = len(kept[b])
            if n > 9:
                middle = sorted(range(p, n - 3), key=lambda j: (-w[b][j], j))[:6 - p]
                kept[b] = [before[b][j] for j in sorted(list(range(p)) + middle + list(range(n - 3, n)))]
            assert committed(cache, b).tolist() == kept[b]
        assert int(cache.free_range[1]) + int(cache.owned.sum()) == 12
    assert cache.dropped.tolist() == [60 - 9, 36 - 9]


def serve_weights(cache, b):
    at = torch.arange(int(cache.lengths[b]))
    return cache.weights.view(-1)[cache.block_table[b, at // cache.block_size].long() * cache.block_size + at % cache.block_size].tolist()


def test_a_prefix_is_shared_and_comes_back_with_its_last_member(calls):
    cache = tree_cache.TreeCache(4, 1, 12, 4, 1, 1, width=6, dtype=torch.float32, device="cpu", weigh=True)
    cache.lengths = torch.tensor([0, -1, -1, -1], dtype=I32)
    with pytest.raises(RuntimeError, match="whole block"):
        cache.share(0, [1])
    _, marks = step(cache, torch.arange(-1, 9, dtype=I32), 0.0, [9, -1, -1, -1])
    for rows in ([0], [1, 1]):
        with pytest.raises(RuntimeError, match="empty"):
            cache.share(0, rows)
    assert cache.share(0, [1, 3]) == 8
    assert cache.lengths.tolist() == [10, 8, -1, 8] and cache.owned.tolist() == [3, 2, 0, 2] and cache.protected.tolist() == [8, 8, 0, 8]
    assert cache.plan.group.tolist() == [0, 0, -1, 0] and cache.plan.blocks.tolist() == [2]
    assert torch.equal(cache.plan.table[0], cache.block_table[0, :2])
    with pytest.raises(RuntimeError, match="already"):
        cache.share(1, [2])
    _, more = step(cache, torch.arange(-1, 3, dtype=I32), 1000.0, [3, 1, -1, 2])
    assert committed(cache, 1).tolist() == marks[0, :8].tolist() + more[1, :2].tolist()
    assert committed(cache, 3).tolist() == marks[0, :8].tolist() + more[3, :3].tolist()
    cache.evict(9, recent=1)                                     # what is shared stays
    for b in (0, 1, 3):
        assert committed(cache, b).tolist()[:8] == marks[0, :8].tolist() and int(cache.lengths[b]) == 9
    held = 2 + 3 * 1
    assert int(cache.free_range[1]) == 12 - held
    cache.release(0)
    assert cache.plan.group.tolist() == [-1, 0, -1, 0] and int(cache.free_range[1]) == 12 - held + 1
    cache.release(3)
    cache.release(1)
    assert cache.plan is None and int(cache.free_range[1]) == 12
    free = cache.free_blocks[(int(cache.free_range[0]) + torch.arange(12)) % 12]
    assert sorted(free.tolist()) == list(range(12)) and cache.protected.tolist() == [0, 0, 0, 0] and cache.dropped.tolist() == [0, 0, 0, 0]


def holdings(cache):
    """Blocks that are free, in the ring's order, and those that requests hold."""
    first, count = cache.free_range.tolist()
    free = cache.free_blocks[(first + torch.arange(count)) % cache.free_blocks.numel()].tolist()
    return free, {x for b in range(cache.owned.numel()) for x in cache.block_table[b, :int(cache.owned[b])].tolist()}


def shared_by_four(weigh=True):
    cache = tree_cache.TreeCache(4, 1, 12, 4, 1, 1, width=6, dtype=torch.float32, device="cpu", weigh=weigh)
    cache.lengths = torch.tensor([0, -1, -1, -1], dtype=I32)
    step(cache, torch.arange(-1, 9, dtype=I32), 0.0, [9, -1, -1, -1])
    return cache


@pytest.mark.parametrize("shared,ended", [([-1], [3, 0]), ([-1], [-1, 0]), ([3], [-1, -4]), ([3], [-4, 3]), ([torch.tensor(-1), 1], [1, 0, 3]),
                                          (torch.tensor([1, 3]), [torch.tensor(-3), 0, torch.tensor(3)])])
def test_rows_are_the_same_by_any_name(calls, shared, ended):
    """Rows from the end, and rows in tensors: no block that a request still holds comes back, and none twice."""
    cache = shared_by_four()
    assert cache.share(torch.tensor(0), shared) == 8
    for x in ended:
        cache.release(x)
        free, held = holdings(cache)
        assert len(set(free)) == len(free) and not held & set(free) and len(free) + len(held) == 12
    assert cache.plan is None and cache.prefixes == {} and cache.protected.tolist() == [0, 0, 0, 0]


def test_a_plan_lists_those_that_share_alone(calls):
    cache = shared_by_four()
    cache.share(0, [3])
    assert cache.plan.members.tolist() == [0, 3] and cache.plan.first.tolist() == [0, 2]
    cache.release(0)
    assert cache.plan.members.tolist() == [3] and cache.plan.first.tolist() == [0, 1] and int(cache.plan.place[3]) == 0


def test_a_member_is_not_shared_again_by_another_name(calls):
    cache = shared_by_four()
    assert cache.share(-4, [1]) == 8
    for request in (0, -4, torch.tensor(0), torch.tensor(-4), 1, -3):
        with pytest.raises(RuntimeError, match="already"):
            cache.share(request, [2])
    other = shared_by_four()
    for rows in ([0], [-4], [torch.tensor(0)], [1, -3], [torch.tensor(1), 1]):
        with pytest.raises(RuntimeError, match="empty"):
            other.share(0, rows)
    for request, rows in ((4, [1]), (-5, [1]), (0, [4]), (0, [1, -5])):
        with pytest.raises(IndexError):
            other.share(request, rows)
    for request in (4, -5):
        with pytest.raises(IndexError):
            other.release(request)
    assert other.prefixes == {} and other.share(0, []) == 8


def test_without_weights_nothing_is_evicted(calls):
    cache = tree_cache.TreeCache(1, 1, 2, 4, 1, 1, width=2, dtype=torch.float32, device="cpu")
    with pytest.raises(RuntimeError, match="weigh"):
        cache.evict(1)
