"""Shared prefixes, weights, eviction and log probabilities at the ends of their ranges: offsets beyond 32 bits, the most nodes, heads, tokens and
requests, temperatures at their limits, two calls at once."""
import math

import pytest
import torch

from . import serve_ref, step_ref as ref
from .test_gpu_prefix import check as check_prefix, prefix_case
from .test_gpu_serve import check_logprobs, check_path, evict_case, rows
from .test_gpu_step import chain, cuda, random_tree, tree
from .test_gpu_weights import case as weights_case, check as check_weights
from paper_2602_16994_b200 import binding, tree_cache

pytestmark = pytest.mark.gpu

I32 = torch.int32


def far(cache, blocks):
    """The same blocks at the end of a cache of `blocks` (on the device), and what is added to their numbers."""
    big = torch.zeros(blocks, *cache.shape[1:], dtype=cache.dtype, device="cuda")
    shift = blocks - cache.shape[0]
    big[shift:] = cache.cuda()
    return big, shift


def shifted(table, shift):
    return torch.where(table >= 0, table + shift, table)


def test_offsets_beyond_32_bits_in_prefixes_and_weights():
    blocks = 2**31 // (16 * 2 * 128) + 2000                       # entries of a cache: above 2^31
    case = prefix_case([0, 0, 1], [9, 2], [100, 3, 50], tree(4, 2, 4), 8, 2, 128, seed=1)
    c, (group, shared, table), skip = case
    want = ref.attention(**c)
    k, shift = far(c["k_cache"], blocks)
    v, _ = far(c["v_cache"], blocks)
    assert k.numel() > 2**31
    plan = binding.prefix_plan(group.cuda(), shared.cuda(), shifted(table, shift).cuda())
    check_prefix(case, want, hide=False, k_cache=k, v_cache=v, block_table=shifted(c["block_table"], shift).cuda(), plan=plan)
    del v
    w = weights_case([300, 40], tree(4, 2, 4), 8, 2, 128, 16, seed=2)
    want = serve_ref.weights(w["weights"], w["q"], w["k_cache"], w["lse"], w["table"], w["lengths"], w["parent"])
    k.zero_()
    k[blocks - w["k_cache"].shape[0]:] = w["k_cache"].cuda()
    shift = blocks - w["k_cache"].shape[0]
    got = torch.zeros(blocks, 16, device="cuda")
    got[shift:] = w["weights"].cuda()
    d = cuda(w)
    binding.cache_weights(got, d["q"], k, d["lse"], shifted(w["table"], shift).cuda(), d["lengths"], d["parent"])
    assert bool((got[:shift] == 0).all())
    assert float((got[shift:].cpu().double() - want["weights"]).abs().max()) < 1e-4


def test_offsets_beyond_32_bits_in_an_eviction():
    c = evict_case(3, 300, 16, 2, (8, 128), seed=3)
    blocks = 2**31 // (16 * 8 * 128) + 3000
    want, _ = serve_ref.evict(c["cache"], c["weights"], c["lengths"], c["block_table"], c["owned"], c["free_blocks"], c["free_range"], 100, 20)
    n = c["cache"].shape[1]
    shift = blocks - n
    big = torch.zeros(2, blocks, 16, 8, 128, dtype=torch.bfloat16, device="cuda")
    big[:, shift:] = c["cache"].cuda()
    w = torch.zeros(blocks, 16, device="cuda")
    w[shift:] = c["weights"].cuda()
    d = cuda(c)
    got = binding.cache_evict(big, w, d["lengths"], shifted(c["block_table"], shift).cuda(), d["owned"], d["free_blocks"], d["free_range"], 100, recent=20)
    assert torch.equal(big[:, shift:].cpu(), want["cache"]) and not bool(big[:, :shift].any())
    assert torch.equal(w[shift:].cpu(), want["weights"]) and torch.equal(got.lengths.cpu(), want["lengths"])


def test_weights_of_lengths_at_the_end_of_32_bits():
    """Tables with room for 2^31 entries, few of whose columns name a block: those get their weight, and the requests beside them theirs."""
    block, width, D = 2**16, 2**15, 64
    g = torch.Generator().manual_seed(26)
    k = torch.randn(4, block, 1, D, generator=g).bfloat16()
    q = torch.randn(3, 1, 1, D, generator=g).bfloat16()
    table = torch.full((3, width), -1, dtype=I32)
    table[0, 0], table[0, width - 1], table[1, 5], table[2, 0] = 0, 1, 2, 3
    lengths, lse = torch.tensor([2**31 - 1, 2**31 - 60, 1000], dtype=I32), torch.tensor([1.0, 2.0, 3.0]).view(3, 1, 1)
    w = torch.zeros(4, block, device="cuda")
    status = binding.cache_weights(w, q.cuda(), k.cuda(), lse.cuda(), table.cuda(), lengths.cuda(), torch.tensor([-1], dtype=I32).cuda())
    assert status.tolist() == [5, 5, 0]
    for b, (owner, upto) in enumerate(((0, block), (0, block - 1), (1, block), (2, 1001))):
        # (the table ends where 2^31 entries do: its last entry, 2^31 - 1, lies behind the last that counts)
        score = (k[b, :, 0].double() @ q[owner, 0, 0].double()) / 8
        want = (score - float(lse[owner])).exp()
        want[upto:] = 0.0
        # an exponential is off by 2^-22, its argument by three roundings and by a product of 64 entries summed in fp32
        reach = (k[b, :, 0].double().abs() @ q[owner, 0, 0].double().abs()) / 8
        bound = want * ((score.abs() + 3) * 3 * 2.0**-24 + reach * 5 * 2.0**-22 + 2.0**-21)
        assert bool(((w[b].cpu().double() - want).abs() <= bound).all()), b


def test_an_eviction_of_lengths_at_the_end_of_32_bits():
    """A length that the table's columns have room for and the cache has not: nothing moves.  (Blocks that the table names again and again.)"""
    block, width = 2**20, 2048
    g = torch.Generator().manual_seed(24)
    cache, weights = torch.randint(0, 256, (1, 1, block, 1), generator=g).byte().cuda(), torch.rand(1, block, generator=g).cuda()
    before, w = cache.clone(), weights.clone()
    lengths = torch.tensor([2**31 - 1, 2**31 - 65537, block + 1, -2**31], dtype=I32, device="cuda")
    table, owned = torch.zeros(4, width, dtype=I32, device="cuda"), torch.full((4,), width, dtype=I32, device="cuda")
    ring, free = torch.full((9,), -1, dtype=I32, device="cuda"), torch.tensor([0, 0], dtype=I32, device="cuda")
    for budget in (100, 2**20):
        got = binding.cache_evict(cache, weights, lengths, table, owned, ring, free, budget)
        assert got.status.tolist() == [5, 5, 5, 0] and torch.equal(got.lengths, lengths) and torch.equal(got.owned, owned)
        assert torch.equal(cache, before) and torch.equal(weights, w) and got.free_range.tolist() == [0, 0]


def test_an_eviction_in_one_block_of_almost_all_slots():
    """A budget and a block that 32 bits do not hold together: the same as in a block of just the request's size."""
    n, budget, most = 70100, 70000, 2**31 - 65600
    g = torch.Generator().manual_seed(25)
    rows, w = torch.randint(0, 256, (n,), generator=g).byte(), torch.rand(n, generator=g)
    got = []
    for block in (n, most):
        cache, weights = torch.zeros(1, 1, block, 1, dtype=torch.uint8, device="cuda"), torch.zeros(1, block, device="cuda")
        cache[0, 0, :n, 0], weights[0, :n] = rows.cuda(), w.cuda()
        one = torch.zeros(1, dtype=I32, device="cuda")
        done = binding.cache_evict(cache, weights, one + n, one[None], one + 1, torch.full((3,), -1, dtype=I32, device="cuda"),
                                   torch.zeros(2, dtype=I32, device="cuda"), budget, recent=9)
        assert done.status.tolist() == [0] and done.lengths.tolist() == [budget] and done.owned.tolist() == [1] and done.free_range.tolist() == [0, 0]
        got.append((cache[0, 0, :n, 0].cpu(), weights[0, :n].cpu()))
        del cache, weights
    keep = sorted(torch.sort(w[:n - 9], descending=True, stable=True).indices[:budget - 9].tolist()) + list(range(n - 9, n))
    assert torch.equal(got[0][0][:budget], rows[keep]) and torch.equal(got[0][1][:budget], w[keep])
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_offsets_beyond_32_bits_in_logits():
    R, V = 17000, 131072
    z = torch.zeros(R, V, dtype=torch.bfloat16, device="cuda")
    some, t = rows(3, V, 1, torch.bfloat16, 4)
    at = torch.tensor([0, 9000, R - 1])
    z[at.cuda()] = some.cuda()
    tokens = torch.zeros(R, 1, dtype=I32)
    tokens[at] = t
    got = binding.token_logprobs(z, tokens.cuda(), top=4)
    want = serve_ref.logprobs(some, t, 1.0, 4)
    assert torch.equal(got.top_tokens[at.cuda()].cpu(), want["top_tokens"])
    assert float((got.logprob[at.cuda()].cpu() - want["logprob"]).abs().max()) < 1e-4
    flat = got.logprob[1:9000]                                   # rows of one value: log V each, and the first tokens
    assert float((flat + math.log(V)).abs().max()) < 1e-4 and got.top_tokens[5].tolist() == [0, 1, 2, 3]


def test_prefixes_without_groups_and_with_empty_ones():
    case = prefix_case([-1, -2, -1], [], [100, 0, 50], tree(4, 2, 4), 8, 2, 128, seed=5)
    none = binding.prefix_plan(case[1][0].cuda(), torch.zeros(0, dtype=I32, device="cuda"), torch.zeros(0, 1, dtype=I32, device="cuda"))
    check_prefix(case, plan=none)
    check_prefix(prefix_case([1, 1, -1], [4, 0, 7], [100, 0, 50], tree(4, 2, 4), 8, 2, 128, seed=6))


def test_the_most_nodes_and_heads():
    g = torch.Generator().manual_seed(7)
    check_prefix(prefix_case([0, 0], [3], [5, 60], random_tree(1024, g), 2, 1, 64, seed=7))
    check_prefix(prefix_case([0, 0, 0], [3], [5, 60, 200], chain(3), 128, 1, 64, seed=8))
    check_weights(weights_case([5, 300], random_tree(1024, g), 2, 1, 64, 16, seed=9))
    check_weights(weights_case([5, 300], chain(1024), 1, 1, 64, 16, seed=10, fresh=True))
    check_weights(weights_case([5, 300, 40], chain(3), 200, 1, 64, 16, seed=11))
    check_weights(weights_case([64, 300], random_tree(33, g), 6, 3, 128, 16, seed=12))
    check_weights(weights_case([64, 300], random_tree(34, g), 6, 3, 128, 16, seed=13))


@pytest.mark.parametrize("temperature", [1e-30, 1e30])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_temperatures_at_their_limits(temperature, dtype):
    z, t = rows(2, 3000, 2, dtype, 14)
    z[0, ::2] = -math.inf
    z[1, 5] = torch.finfo(dtype).min
    t[:, 0] = z.argmax(-1).int()
    check_logprobs(z, t, temperature, 5)


def test_many_given_tokens():
    check_logprobs(*rows(2, 9000, 700, torch.bfloat16, 15), top=2)


def test_masks_that_come_late_in_a_row():
    """Masked stretches ahead of, between and behind the others, of sizes around a batch of loads."""
    for R in (1, 300):
        for first in (1, 8191, 8192, 8193, 20000):
            z, t = rows(R, 40000, 1, torch.bfloat16, 16)
            z[:, :first] = -math.inf
            z[:, 30000:39000] = -math.inf
            t[:] = 39999
            check_logprobs(z, t, 1.0, 3)


def test_two_calls_at_once():
    """The same calls on two streams at the same time, each with tensors of its own to write."""
    w = cuda(weights_case([900, 40, 333], tree(4, 2, 4), 8, 2, 128, 16, seed=17))
    c = evict_case(4, 2000, 16, 3, (2, 64), seed=18)
    p = prefix_case([0, 1, 0, -1], [40, 7], [100, 60, 30, 200], tree(4, 2, 4), 8, 2, 128, seed=19)
    plan, d = binding.prefix_plan(*(x.cuda() for x in p[1])), cuda(p[0])
    streams, out = [torch.cuda.Stream() for _ in range(3)], []
    torch.cuda.synchronize()
    for _ in range(8):
        for s in streams:
            e = cuda(c)
            weights = w["weights"].clone()
            s.wait_stream(torch.cuda.current_stream())
            status = binding.cache_weights(weights, w["q"], w["k_cache"], w["lse"], w["table"], w["lengths"], w["parent"], stream=s)
            a = binding.prefix_attention(d["q"], d["k_cache"], d["v_cache"], d["block_table"], d["lengths"], d["parent"], plan, stream=s)
            cut = binding.cache_evict(e["cache"], e["weights"], e["lengths"], e["block_table"], e["owned"], e["free_blocks"], e["free_range"], 300,
                                      recent=7, stream=s)
            out.append((weights, status, a.out, a.status, e["cache"], e["weights"], cut.lengths, cut.free_range, e["free_blocks"]))
    torch.cuda.synchronize()
    for x in out[1:]:
        for a, b in zip(x, out[0]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("N,V", [(33, 500), (70, 70001), (1024, 300)])
@pytest.mark.parametrize("B", [1, 3])
def test_paths_of_many_nodes(B, N, V):
    """Chains longer than the places that are gone through at once, accepted to their ends or not; rows by one CTA and by several."""
    g = torch.Generator().manual_seed(N + B)
    z = (3 * torch.randn(B, N, V, generator=g)).bfloat16()
    parent = torch.arange(-1, N - 1, dtype=I32)
    accepted = torch.tensor([N - 1, 32, 31][:B], dtype=I32)
    check_path(z, accepted, torch.randint(0, V, (B, N), generator=g).int(), parent, 0.9, 2)


@pytest.mark.parametrize("V", [16385, 32768, 32769, 65537, 131073, 262151])
@pytest.mark.parametrize("R", [1, 12, 13, 37, 75])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_by_any_number_of_ctas(R, V, dtype):
    """Sizes on both sides of where a row goes to one CTA more."""
    z, t = rows(R, V, 1, dtype, R + V)
    z[R // 2, : V // 2] = -math.inf
    check_logprobs(z, t, 1.0, 32)


@pytest.mark.parametrize("groups", [[0] * 3, [0] * 4, [0] * 6 + [1] * 2, [0, 1, 1, 2, 2, 2, 2, 2, 2]])
def test_prefix_rows_around_two_blocks(groups):
    """Averages of rows of a prefix below, at and above two blocks, groups of unequal sizes among them."""
    n = max(groups) + 1
    check_prefix(prefix_case(groups, [20, 9, 30][:n], [50 + 37 * i for i in range(len(groups))], tree(4, 2, 4), 8, 2, 128, seed=len(groups)))


def test_more_alternatives_than_there_may_be_take_no_memory():
    z, t = rows(1, 100, 1, torch.float32, 21)
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.max_memory_allocated()
    with pytest.raises(RuntimeError):
        binding.token_logprobs(z.cuda(), t.cuda(), top=2**31 - 1)
    assert torch.cuda.max_memory_allocated() < before + 2**20


def test_an_eviction_on_a_stream_tells_the_allocator_of_what_it_reads(monkeypatch):
    """``dropped`` of an earlier eviction, which another stream may have made, is read on the stream of the next one and let go of."""
    cache = tree_cache.TreeCache(2, 1, 16, 4, 1, 64, width=8, weigh=True)
    cache.block_table.copy_(torch.arange(16, dtype=I32).view(2, 8))
    cache.lengths, cache.owned = torch.full((2,), 30, dtype=I32, device="cuda"), torch.full((2,), 8, dtype=I32, device="cuda")
    cache.free_range = torch.tensor([0, 0], dtype=I32, device="cuda")
    cache.evict(20)
    before, told, real = cache.dropped, [], cache._on

    def on(stream, *used):
        told.extend(used)
        return real(stream, *used)

    monkeypatch.setattr(cache, "_on", on)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cache.evict(10, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert any(x is before for x in told)
    assert cache.dropped.tolist() == [20, 20] and cache.lengths.tolist() == [10, 10] and cache.free_range.tolist() == [0, 10]


def test_a_refused_tree_adds_no_weight():
    """Two requests, blocks for one of them: the other's entries keep the weights that they had, and its lengths."""
    g = torch.Generator().manual_seed(23)
    cache = tree_cache.TreeCache(2, 1, 9, 16, 2, 64, width=5, weigh=True)
    cache.storage.copy_(torch.randn(cache.storage.shape, generator=g))
    cache.weights.copy_(torch.rand(cache.weights.shape, generator=g))
    cache.block_table[:, :4] = torch.arange(8, dtype=I32).view(2, 4)
    cache.lengths, cache.owned = torch.full((2,), 64, dtype=I32, device="cuda"), torch.full((2,), 4, dtype=I32, device="cuda")
    cache.free_range = torch.tensor([8, 1], dtype=I32, device="cuda")
    before = cache.weights.cpu()
    parent = torch.arange(-1, 2, dtype=I32).cuda()
    done = cache.begin(parent)
    refused = (done.status != 0).nonzero().flatten().tolist()
    assert refused == [1]
    q = torch.randn(2, 3, 4, 64, generator=g).bfloat16().cuda()
    cache.attend(0, q)
    after = cache.weights.cpu()
    assert torch.equal(after[4:8], before[4:8]) and bool((after[:4] > before[:4]).all())
    added = after[:4].double() - before[:4].double()
    assert float(added.sum() + after[8, :3].double().sum()) == pytest.approx(12, rel=1e-3)          # (three nodes of four heads)
