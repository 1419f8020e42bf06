"""Attention weights of cache entries against their restatement in 64 bits, and their way through a step with an eviction."""
import math

import pytest
import torch

from . import serve_ref as ref, step_ref
from .test_gpu_step import chain, cuda, pages, random_tree, tree
from paper_2602_16994_b200 import binding

pytestmark = pytest.mark.gpu

I32 = torch.int32


def case(lengths, parent, Hq, Hkv, D, block, dtype=torch.bfloat16, seed=0, n_nodes=None, protected=None, fresh=False):
    g = torch.Generator().manual_seed(seed)
    B, N = len(lengths), parent.shape[-1]
    lengths = torch.as_tensor(lengths, dtype=I32)
    table, blocks = pages(lengths.clamp(min=0), N, block, g)
    q = (1.5 * torch.randn(B, N, Hq, D, generator=g)).to(dtype)
    k = torch.randn(blocks, block, Hkv, D, generator=g).to(dtype)
    r = step_ref.attention(q, k, k, table, lengths, parent, n_nodes)
    return dict(weights=torch.rand(blocks, block, generator=g), q=q, k_cache=k, lse=r["lse"].float(), table=table, lengths=lengths, parent=parent,
                n_nodes=n_nodes, protected=protected, fresh=fresh)


def check(c, scale=None, **moved):
    """An exponential is off by 2^-22 and by its argument's errors: three roundings of |score| and |lse| (the factor, the product with log2 e, the
    difference), a product of D entries summed in fp32 (in steps of 16, each off by 2^-22 of the entries' products at most); a thread adds its terms one by one."""
    want = ref.weights(c["weights"], c["q"], c["k_cache"], c["lse"], c["table"], c["lengths"], c["parent"], c["n_nodes"], scale, c["protected"],
                       c["fresh"])
    d = dict({k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}, **moved)
    args = lambda: (d["q"], d["k_cache"], d["lse"], d["table"], d["lengths"], d["parent"])  # noqa: E731
    status = binding.cache_weights(d["weights"], *args(), n_nodes=d["n_nodes"], scale=scale, protected=d["protected"], fresh=c["fresh"])
    assert torch.equal(status.cpu(), want["status"])
    D, terms = c["q"].shape[-1], c["q"].shape[1] * c["q"].shape[2]
    bound = want["size"] * 3 * 2.0**-24 + want["reach"] * (D // 16 + 1) * 2.0**-22 + want["got"] * (2.0**-22 + terms * 2.0**-24) + want["weights"].abs() * 2.0**-23
    off = (d["weights"].cpu().double() - want["weights"]).abs()
    assert bool((off <= bound).all()), (float((off - bound).max()), int((off > bound).sum()))
    untouched = want["got"] == 0
    if not c["fresh"]:
        assert torch.equal(d["weights"].cpu()[untouched], c["weights"][untouched])
    again = c["weights"].cuda()
    binding.cache_weights(again, *args(), n_nodes=d["n_nodes"], scale=scale, protected=d["protected"], fresh=c["fresh"])
    assert torch.equal(again, d["weights"])                      # the same bits
    return d["weights"]


@pytest.mark.parametrize("lengths,parent,Hq,Hkv,D,block", [
    ([0], tree(0, 0, 0), 1, 1, 64, 16), ([1], tree(0, 0, 0), 4, 2, 128, 16), ([300], tree(0, 0, 0), 32, 8, 128, 16),
    ([127, 128, 129, 0, 255, 256], tree(3, 1, 2), 4, 2, 64, 8), ([1000, 3, 700], tree(4, 2, 4), 8, 2, 128, 24), ([500, 900], tree(8, 2, 6), 14, 2, 64, 64),
    ([260, 20], tree(2, 0, 3), 6, 3, 256, 16), ([700, 384], chain(150), 4, 2, 128, 16), ([130], chain(600), 2, 1, 64, 7), ([40, 90], chain(33), 71, 1, 128, 1),
    ([129, 640], chain(40), 8, 1, 256, 32)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("fresh", [False, True])
def test_weights(lengths, parent, Hq, Hkv, D, block, dtype, fresh):
    check(case(lengths, parent, Hq, Hkv, D, block, dtype, sum(lengths) + D, fresh=fresh))


def test_weights_of_random_trees_idle_ragged_and_protected():
    g = torch.Generator().manual_seed(1)
    for seed in range(4):
        B, N = 9, 45 + 100 * seed
        parent = torch.stack([random_tree(N, g) for _ in range(B)])
        lengths = torch.randint(0, 500, (B,), generator=g).int()
        n_nodes = torch.randint(0, N + 1, (B,), generator=g).int()
        protected = torch.randint(0, 300, (B,), generator=g).int()
        lengths[3], n_nodes[0], protected[5], protected[6] = -4, N, 10000, -1
        check(case(lengths, parent, 4, 2, 64, 16, seed=seed, n_nodes=n_nodes, protected=protected, fresh=seed % 2 == 0))


def test_weights_over_many_requests():
    """More requests than CTAs, and runs that go through several of them."""
    g = torch.Generator().manual_seed(2)
    check(case(torch.randint(0, 400, (333,), generator=g), tree(2, 0, 2), 2, 1, 64, 16, seed=2))
    check(case([5000, 3, 2000], tree(2, 0, 2), 2, 2, 64, 16, seed=3, protected=torch.tensor([129, 0, 1900], dtype=I32)))


@pytest.mark.parametrize("requests", [641, 700, 768, 769, 1600])
def test_weights_of_as_many_requests_as_a_cta_has_threads_and_more(requests):
    """One request to a thread, in all of its warps, and several."""
    g = torch.Generator().manual_seed(requests)
    lengths = torch.randint(0, 150, (requests,), generator=g)
    lengths[::7], lengths[-1] = -1, 300
    check(case(lengths, tree(2, 0, 1), 2, 1, 64, 16, seed=requests))


def test_weights_are_the_same_bits_in_many_calls():
    c = cuda(case([900, 40, 333, 2000, 7], tree(4, 2, 4), 8, 2, 128, 16, seed=14))
    want = None
    for _ in range(200):
        w = c["weights"].clone()
        status = binding.cache_weights(w, c["q"], c["k_cache"], c["lse"], c["table"], c["lengths"], c["parent"])
        want = w if want is None else want
        assert torch.equal(w, want) and not bool(status.any())


def test_weights_beside_what_is_no_number():
    """Keys, queries and lse that are not finite reach nothing that they are no part of; rows of infinite lse add nothing."""
    c = case([300, 200, 260], tree(4, 2, 4), 8, 2, 128, 16, seed=5)
    at = lambda b, j: (int(c["table"][b, j // 16]), j % 16)  # noqa: E731
    c["k_cache"][at(0, 17)] = math.nan
    c["k_cache"][at(1, 200 + 18)] = math.inf                     # a leaf's own key
    c["q"][2, 3] = math.nan
    c["q"][2, 4, 1] = math.inf
    c["lse"][0, :, :] = torch.where(torch.arange(8) < 3, math.nan, c["lse"][0])
    c["lse"][1, 18], c["lse"][2, 3], c["lse"][2, 4, 1], c["lse"][2, 6] = math.nan, math.nan, math.inf, -math.inf
    out = check(c)
    assert bool(out.isfinite().all())


def test_weights_of_bad_blocks_and_trees():
    parent = tree(4, 2, 4).repeat(6, 1)
    parent[1, 4], parent[2, 0] = 5, 0
    c = case([300, 300, 300, 300, 300, 300], parent, 4, 2, 128, 16, seed=6, n_nodes=torch.tensor([19, 19, 19, 20, 19, 19], dtype=I32))
    c["table"][4, 3], c["table"][4, 19] = -1, c["k_cache"].shape[0]
    c["table"] = c["table"][:, :19].contiguous()                 # 304 entries of 319
    c["table"][5, 1] = 2**31 - 1
    check(c)


def test_weights_of_views_and_scales():
    c = case([300, 77], tree(4, 2, 4), 8, 2, 128, 16, seed=7)
    wide_q = torch.zeros(2, 19, 12, 128, dtype=torch.bfloat16, device="cuda")
    wide_q[:, :, 2:10] = c["q"].cuda()
    wide_k = torch.zeros(c["k_cache"].shape[0], 16, 5, 136, dtype=torch.bfloat16, device="cuda")
    wide_k[:, :, 1:3, 8:] = c["k_cache"].cuda()
    check(c, q=wide_q[:, :, 2:10], k_cache=wide_k[:, :, 1:3, 8:])
    c["lse"] = step_ref.attention(c["q"], c["k_cache"], c["k_cache"], c["table"], c["lengths"], c["parent"], scale=0.3)["lse"].float()
    check(c, 0.3)
    c["lse"] = step_ref.attention(c["q"], c["k_cache"], c["k_cache"], c["table"], c["lengths"], c["parent"], scale=0.0)["lse"].float()
    check(c, 0.0)


def test_weights_add_up_to_the_rows():
    """All weights of a step, together, are the number of its rows: each row's weights sum to 1."""
    c = case([900, 40, 333], tree(4, 2, 4), 8, 2, 128, 16, seed=8)
    d = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    a = binding.tree_attention(d["q"], d["k_cache"], d["k_cache"], d["table"], d["lengths"], d["parent"], want_lse=True)
    w = torch.zeros_like(d["weights"])
    binding.cache_weights(w, d["q"], d["k_cache"], a.lse, d["table"], d["lengths"], d["parent"])
    assert abs(float(w.double().sum()) / (3 * 19 * 8) - 1) < 1e-5


def test_weights_on_streams_and_in_graphs():
    c = case([900, 40, 333], tree(4, 2, 4), 8, 2, 128, 16, seed=9)
    d = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    call = lambda w, s=None: binding.cache_weights(w, d["q"], d["k_cache"], d["lse"], d["table"], d["lengths"], d["parent"], stream=s)  # noqa: E731
    want = d["weights"].clone()
    call(want)
    side = torch.cuda.Stream()
    w = d["weights"].clone()
    side.wait_stream(torch.cuda.current_stream())
    call(w, side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(w, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        status = call(w)
    for _ in range(3):
        w.copy_(d["weights"])
        graph.replay()
        assert torch.equal(w, want) and status.tolist() == [0, 0, 0]


def test_weights_whose_waits_run_out():
    c = case([900, 40, 333], tree(4, 2, 4), 8, 2, 128, 16, seed=9)
    d = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    call = lambda w: binding.cache_weights(w, d["q"], d["k_cache"], d["lse"], d["table"], d["lengths"], d["parent"])  # noqa: E731
    want, w = d["weights"].clone(), d["weights"].clone()
    call(want)
    torch.cuda.synchronize()
    try:
        binding.set_test_hooks(wait_cycles=2_000_000, hold_slot=1 * 19 + 3)
        status = call(w)
        torch.cuda.synchronize()
    finally:
        binding.set_test_hooks()
    assert status[1] == 4
    w.copy_(d["weights"])
    assert call(w).tolist() == [0, 0, 0] and torch.equal(w, want)


def test_weights_refusals():
    c = case([100], tree(1, 0, 1), 4, 2, 64, 16, seed=10)
    d = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}

    def call(**kw):
        e = dict(d, **kw)
        return binding.cache_weights(e["weights"], e["q"], e["k_cache"], e["lse"], e["table"], e["lengths"], e["parent"], scale=kw.get("scale"))

    for bad in (dict(q=d["q"].float()), dict(k_cache=d["k_cache"].half()), dict(weights=d["weights"].bfloat16()), dict(weights=d["weights"][:1]),
                dict(lse=d["lse"].double()), dict(lse=d["lse"][:, :1]), dict(parent=d["parent"][:1]), dict(q=d["q"][..., :32]), dict(scale=-1.0),
                dict(scale=math.nan), dict(q=d["q"].clone().requires_grad_()), dict(lse=d["lse"].clone().requires_grad_())):
        with pytest.raises(RuntimeError):
            call(**bad)
