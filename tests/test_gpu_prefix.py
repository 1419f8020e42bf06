"""Attention of requests that share prefixes against the attention of each by itself, in 64 bits."""
import math

import pytest
import torch

from . import step_ref as ref
from .test_gpu_step import chain, check_attention, cuda, pages, random_tree, tree
from paper_2602_16994_b200 import binding

pytestmark = pytest.mark.gpu

I32 = torch.int32


def prefix_case(group, blocks, own, parent, Hq, Hkv, D, dtype=torch.bfloat16, block=16, seed=0, n_nodes=None, spread=2.0, scale=None, spare=2):
    """Requests of `own` tokens behind the prefix of their group (negative: idle; group negative: no prefix); the whole table for the restatement, the plan for
    the call."""
    g = torch.Generator().manual_seed(seed)
    N, B = parent.shape[-1], len(group)
    group, shared = torch.tensor(group, dtype=I32), torch.tensor(blocks, dtype=I32)
    own = torch.as_tensor(own, dtype=I32)
    table, count = pages(own.clamp(min=0), N, block, g)
    total = count + int(shared.sum())
    ids = torch.randperm(total, generator=g).int()
    table = torch.where(table >= 0, ids[table.clamp(min=0).long()], -1)
    prefix = torch.full((len(blocks), max([1] + blocks) + spare), -1, dtype=I32)
    at = count
    for k, x in enumerate(blocks):
        prefix[k, :x] = ids[at:at + x]
        at += x
    skip = torch.tensor([blocks[x] if 0 <= x < len(blocks) else 0 for x in group.tolist()], dtype=I32)
    rows = torch.full((B, int(skip.max()) + table.shape[1]), -1, dtype=I32)
    for b in range(B):
        if skip[b]:
            rows[b, :skip[b]] = prefix[group[b], :skip[b]]
        rows[b, skip[b]:skip[b] + table.shape[1]] = table[b]
    lengths = torch.where(own >= 0, own + skip * block, own)
    normal = lambda *s: torch.randn(*s, generator=g).to(dtype)  # noqa: E731
    c = dict(q=(spread * torch.randn(B, N, Hq, D, generator=g)).to(dtype), k_cache=normal(total, block, Hkv, D), v_cache=normal(total, block, Hkv, D),
             block_table=rows, lengths=lengths, parent=parent, n_nodes=None if n_nodes is None else torch.tensor(n_nodes, dtype=I32), scale=scale)
    return c, (group, shared, prefix), skip


def check(case, want=None, status=None, hide=True, **moved):
    c, plan, skip = case
    want = want or ref.attention(**c)
    dtype, D = c["q"].dtype, c["q"].shape[-1]
    d = dict(cuda(c), **moved)
    if hide:                                                     # (the prefix's columns of the requests' rows are not read)
        for b, x in enumerate(skip.tolist()):
            d["block_table"][b, :x] = -7
    out = d.pop("out", None)
    if out is None:
        out = torch.full_like(c["q"], 7.0, device="cuda")
    made = moved.get("plan") or binding.prefix_plan(*(x.cuda() for x in plan))
    d.pop("plan", None)
    got = binding.prefix_attention(d.pop("q"), d.pop("k_cache"), d.pop("v_cache"), d.pop("block_table"), d.pop("lengths"), d.pop("parent"), made,
                                   out=out, want_lse=True, **d)
    torch.cuda.synchronize()
    assert got.status.tolist() == (want["status"].tolist() if status is None else status)
    x, lse, live = got.out.cpu().double(), got.lse.cpu().double(), want["live"]
    half = torch.finfo(dtype).eps / 2
    # the bound of the attention of one request by itself: scores of D products and sums in fp32, exponentials and sums, weights rounded to the values'
    # type, the result's own rounding; joining two units' parts is two more factors of 2^-22
    score = want["reach"][..., None] * (D + 4) * 2.0**-24
    bound = want["mass"] * (2 * score + half + 2.0**-20 + 2.0**-21) + want["out"].abs() * half
    if dtype == torch.float16:                                   # (weights below 2^-14 lie in steps of 2^-24: half of one for each key, of values up to 6)
        bound = bound + int(c["lengths"].max() + c["q"].shape[1]) * 2.0**-25 * 6 * 2.0**-8 + 2.0**-25
    off = (x - want["out"]).abs()
    same = (x == want["out"]) | (x.isnan() & want["out"].isnan())
    assert bool(((off <= bound) | same)[live].all()), float((off - bound)[live].max())
    assert bool((x[~live] == 7.0).all())
    off = (lse - want["lse"]).abs()
    same = (lse == want["lse"]) | (lse.isnan() & want["lse"].isnan())
    assert bool(((off <= score[..., 0] * 2 + 2.0**-18 + want["lse"].abs() * 2.0**-22) | same)[live].all())
    return got


TREES = {"token": chain(1), "d2k4": tree(4, 2, 4), "k8": tree(8, 2, 6)}


@pytest.mark.parametrize("group,blocks,own", [
    ([0], [1], [0]), ([0, 0], [8], [0, 1]), ([0] * 5, [20], [130, 0, 7, 128, 300]), ([0, 1, 0, -1, 1], [3, 17], [5, 200, 100, 77, 0]),
    ([2, 2, 0, 2], [9, 5, 0], [10, 20, 30, 40]), ([-1, -1], [4], [50, 60]), ([0] * 40, [33], [3 * i for i in range(40)])])
@pytest.mark.parametrize("shape", ["token", "d2k4", "k8"])
@pytest.mark.parametrize("Hq,Hkv,D,dtype,block", [(4, 1, 128, torch.bfloat16, 16), (6, 2, 64, torch.float16, 7), (8, 8, 128, torch.float16, 32),
                                                  (4, 2, 256, torch.bfloat16, 16), (16, 2, 64, torch.bfloat16, 24)])
def test_prefix_attention(group, blocks, own, shape, Hq, Hkv, D, dtype, block):
    if len(group) * TREES[shape].shape[0] * Hq > 12000:
        group, own = group[:12], own[:12]
    check(prefix_case(group, blocks, own, TREES[shape], Hq, Hkv, D, dtype, block, len(group) + D + sum(own)))


def test_prefix_attention_of_requests_that_share_nothing():
    """The same function as the tree attention's, within the bounds of both (its rows may go by other blocks: not the same bits)."""
    case = prefix_case([-1, -1, -1], [2], [300, 0, 1000], tree(4, 2, 4), 8, 2, 128, seed=3)
    want = ref.attention(**case[0])
    check_attention(case[0], want)
    check(case, want)


def test_prefix_attention_over_long_prefixes_and_many_requests():
    for D, dtype in ((128, torch.bfloat16), (64, torch.float16)):
        check(prefix_case([i % 3 for i in range(30)], [200, 10, 129], [(37 * i) % 90 for i in range(30)], chain(1), 8, 2, D, dtype, seed=D))
    check(prefix_case([0] * 3, [700], [10, 2000, 500], chain(1), 4, 1, 128, seed=1))
    check(prefix_case([i // 2 - 1 for i in range(300)], [1 + i % 5 for i in range(149)], [i % 40 for i in range(300)], chain(2), 2, 1, 64, block=8,
                      seed=2))


def test_prefix_attention_of_random_trees_idle_and_ragged():
    g = torch.Generator().manual_seed(1)
    for seed in range(3):
        B, N = 9, 21 + 70 * seed
        parent = torch.stack([random_tree(N, g) for _ in range(B)])
        own = torch.randint(0, 300, (B,), generator=g).tolist()
        own[3] = -1
        n_nodes = torch.randint(0, N + 1, (B,), generator=g).tolist()
        n_nodes[0], n_nodes[5] = N, 0
        check(prefix_case([0, 1, 0, 0, -1, 1, 0, 1, 0], [12, 3], own, parent, 4, 2, 128, seed=seed, n_nodes=n_nodes))


def test_prefix_attention_beside_what_is_no_number():
    """What is not finite in keys and values of a prefix reaches its members alone, in a request's own blocks that request; of bad blocks nothing is read."""
    case = prefix_case([0, 1, 0, -1], [9, 7], [100, 60, 30, 200], tree(4, 2, 4), 8, 2, 128, seed=4)
    c = case[0]
    c["v_cache"][c["block_table"][1, 6], 3, 1, 5] = math.inf     # in group 1's prefix
    c["v_cache"][c["block_table"][0, 9], 2, 0, 7] = math.nan     # request 0's own
    c["k_cache"][c["block_table"][3, 0], 0, 0, 0] = math.nan
    check(case)


def test_prefix_attention_with_bad_blocks():
    case = prefix_case([0, 1, 0, 1], [9, 7], [100, 60, 30, 20], tree(4, 2, 4), 8, 2, 128, seed=5)
    c, (group, shared, prefix), skip = case
    P = c["k_cache"].shape[0]
    for k, x, bad in ((0, 3, -1), (0, 8, P)):
        prefix[k, x] = bad
        c["block_table"][group == k, x] = bad
    c["block_table"][3, 8] = -1                                  # of its own
    got = check(case)
    assert got.status.tolist() == [5, 0, 5, 5]
    # a prefix without any good block: its members see what is theirs
    prefix[1, :7] = -1
    c["block_table"][group == 1, :7] = -1
    check(case)


def test_prefix_attention_of_plans_that_do_not_fit():
    case = prefix_case([0, 1, 0, 1, -1, 0], [9, 7], [100, 60, 30, 20, 50, 10], tree(4, 2, 4), 8, 2, 128, seed=6)
    c, plan, skip = case
    want = ref.attention(**c)
    good = binding.prefix_plan(*(x.cuda() for x in plan))

    def bad(rows, **kw):
        w = {k: v.clone() for k, v in want.items()}
        for b in rows:
            w["out"][b], w["lse"][b], w["status"][b] = 0, -math.inf, 1
        check(case, w, plan=good._replace(**{k: torch.tensor(v, dtype=I32, device="cuda") for k, v in kw.items()}))

    bad([0, 1, 2, 3, 4, 5], first=[4, 1, 6])
    bad([0, 1, 2, 3, 4, 5], first=[-1, 3, 6])
    bad([0, 1, 2, 3, 4, 5], first=[1, 4, 7])
    bad([2], place=[0, 0, -1, 1, 0, 2])
    bad([2, 5], place=[0, 0, 2, 1, 0, 1])
    bad([4], group=[0, 1, 0, 1, 2, 0])
    c["parent"] = c["parent"].repeat(6, 1)
    c["parent"][5, 3] = 3
    c["lengths"][3] = 7 * 16 - 1                                 # shorter than its prefix
    w = {k: v.clone() for k, v in want.items()}
    for b in (3, 5):
        w["out"][b], w["lse"][b], w["status"][b] = 0, -math.inf, 1
    check(case, w)
    w = {k: v.clone() for k, v in want.items()}
    for b in (0, 2, 3, 5):                                       # (more blocks than the table has)
        w["out"][b], w["lse"][b], w["status"][b] = 0, -math.inf, 1
    members = good._replace(blocks=torch.tensor([12, 7], dtype=I32, device="cuda"))
    check(case, w, plan=members)


def test_prefix_attention_of_views_scales_and_masked_rows():
    case = prefix_case([0, 0, 1], [9, 2], [100, 3, 50], tree(4, 2, 4), 8, 2, 128, seed=7, scale=0.3)
    c = case[0]
    wide = torch.zeros(3, 19, 12, 128, dtype=torch.bfloat16, device="cuda")
    wide[:, :, 2:10] = c["q"].cuda()
    out = torch.full((3, 19, 12, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros(c["k_cache"].shape[0], 16, 2, 2, 128, dtype=torch.bfloat16, device="cuda")
    kv[:, :, 0], kv[:, :, 1] = c["k_cache"].cuda(), c["v_cache"].cuda()
    check(case, q=wide[:, :, 2:10], k_cache=kv[:, :, 0], v_cache=kv[:, :, 1], out=out[:, :, 1:9, 8:])
    assert bool((out[:, :, 9:] == 7.0).all()) and bool((out[..., :8] == 7.0).all())
    case = prefix_case([0, 0], [9], [100, 3], chain(1), 8, 2, 128, seed=8, scale=0.0)
    check(case)
    case[0]["k_cache"][:, :, 0, 0], case[0]["q"][:, :, :4, 0] = -math.inf, 1.0               # all scores of a head are -inf
    case[0]["scale"] = None
    check(case)


def test_prefix_attention_on_streams_and_in_graphs():
    case = prefix_case([0, 1, 0, -1], [40, 7], [100, 60, 30, 200], tree(4, 2, 4), 8, 2, 128, seed=9)
    d = cuda(case[0])
    plan = binding.prefix_plan(*(x.cuda() for x in case[1]))
    call = lambda s=None: binding.prefix_attention(d["q"], d["k_cache"], d["v_cache"], d["block_table"], d["lengths"], d["parent"], plan, stream=s)  # noqa: E731
    want = call().out
    for _ in range(20):
        assert torch.equal(call().out, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [call(side), call()]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0].out, want) and torch.equal(got[1].out, want)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, call()))
    d["q"].neg_()
    want = call().out
    for graph, o in graphs * 2:
        graph.replay()
        assert torch.equal(o.out, want)


def test_prefix_attention_whose_waits_run_out():
    case = prefix_case([0, 1, 0, -1], [40, 7], [100, 60, 30, 200], tree(4, 2, 4), 8, 2, 128, seed=9)
    try:
        binding.set_test_hooks(wait_cycles=2_000_000, hold_slot=1 * 19)
        d = cuda(case[0])
        got = binding.prefix_attention(d["q"], d["k_cache"], d["v_cache"], d["block_table"], d["lengths"], d["parent"],
                                       binding.prefix_plan(*(x.cuda() for x in case[1])))
        torch.cuda.synchronize()
    finally:
        binding.set_test_hooks()
    assert got.status.tolist() == [4, 4, 4, 4]
    check(case)


def test_prefix_attention_refusals():
    case = prefix_case([0, 0], [2], [10, 3], chain(1), 4, 2, 64, seed=10)
    d = cuda(case[0])
    plan = binding.prefix_plan(*(x.cuda() for x in case[1]))

    def call(p=plan, **kw):
        e = dict(d, **kw)
        return binding.prefix_attention(e["q"], e["k_cache"], e["v_cache"], e["block_table"], e["lengths"], e["parent"], p, scale=e["scale"])

    assert call().status.tolist() == [0, 0]
    for p in (None, plan[:5], [*plan], plan._replace(group=plan.group[:1]), plan._replace(first=plan.first[:1]), plan._replace(place=plan.place.long()),
              plan._replace(table=plan.table[0]), plan._replace(table=plan.table.repeat(2, 1)), plan._replace(members=plan.members.cpu())):
        with pytest.raises(RuntimeError):
            call(tuple(p) if isinstance(p, binding.PrefixPlan) else p)
    for bad in (dict(q=d["q"].float()), dict(scale=-1.0), dict(v_cache=d["v_cache"][..., :32]), dict(q=d["q"].clone().requires_grad_())):
        with pytest.raises(RuntimeError):
            call(**bad)
    with pytest.raises(RuntimeError):
        binding.prefix_plan(plan.group.long(), plan.blocks, plan.table)


@pytest.mark.parametrize("groups", [[-1] * 126 + [0, 0], [0, -1, 1, -1, 0, 1, -1], [-1, -1, 0], [0, 1, 1, 0]])
def test_prefix_attention_of_plans_that_list_those_that_share(groups):
    """The members alone in the plan, few of many requests or all; scratch for them alone; a plan told a wrong number fits nobody."""
    case = prefix_case(groups, [9, 20][:max(groups) + 1], [(29 * i) % 200 for i in range(len(groups))], chain(1), 16, 4, 128, seed=len(groups))
    parts, sharing = [x.cuda() for x in case[1]], sum(g >= 0 for g in groups)
    plan = binding.prefix_plan(*parts, sharing)
    assert plan.members.numel() == sharing
    check(case, plan=plan)
    if sharing < len(groups):
        w = {k: v.clone() for k, v in ref.attention(**case[0]).items()}
        w["out"][:], w["lse"][:], w["status"][:] = 0, -math.inf, 1
        check(case, w, plan=binding.prefix_plan(*parts, sharing - 1))
