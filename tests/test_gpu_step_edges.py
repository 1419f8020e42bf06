"""The operators around a verification where two of their threads, calls or results could be at odds: one writer to a row, flags that
travel with their data, waits that run out, scores and probabilities at the ends of their range, steps that were refused."""
import math

import pytest
import torch

from . import step_ref as ref
from .test_gpu_step import (I32, attention_case, chain, chains_case, check_attention, check_chains, commit_case, cuda, rope_case, slots_case,
                            tree)
from paper_2602_16994_b200 import binding
from paper_2602_16994_b200.tree_cache import TreeCache

pytestmark = pytest.mark.gpu

TIMEOUT = 4


# ---------------------------------------------------------------------------------------------
# tree_attention: rows of a bad tree have one writer
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape,Hq,Hkv,D", [((0, 0, 0), 8, 2, 128), ((4, 2, 4), 8, 2, 128), ((8, 2, 6), 32, 8, 128), ((8, 2, 6), 8, 1, 64),
                                            ((4, 2, 4), 4, 2, 256)])
@pytest.mark.parametrize("lengths", [[3000], [20000], [2500, 300, 4000, 0]])
def test_rows_of_a_bad_tree_are_zeros_where_units_are_cut(shape, Hq, Hkv, D, lengths):
    """Some thousand keys to a unit are cut into runs and joined; the joined rows of a bad tree must not come on top of its zeros."""
    parent = (tree(*shape) if shape[2] else chain(1)).repeat(len(lengths), 1)
    c = attention_case(lengths, parent, Hq, Hkv, D, torch.bfloat16, 16, seed=21)
    bad = [b for b, n in enumerate(lengths) if n >= 2500]
    for b in bad:
        c["parent"][b, -1] = parent.shape[1]                      # (of one node: a root with a parent)
    want = ref.attention(**c)
    assert [b for b, s in enumerate(want["status"].tolist()) if s == ref.TOPOLOGY] == bad
    for _ in range(10):
        got = check_attention(c, want)
        assert bool((got.out[bad] == 0).all()) and bool((got.lse[bad] == -math.inf).all())


def test_a_bad_tree_for_all_requests():
    c = attention_case([5000, 900, 40], tree(4, 2, 4), 8, 2, 128, torch.bfloat16, 16, seed=22)
    c["parent"][7] = 7
    for _ in range(10):
        got = check_attention(c)
        assert got.status.tolist() == [1, 1, 1] and bool((got.out == 0).all()) and bool((got.lse == -math.inf).all())


def test_a_bad_tree_before_and_behind_good_ones_of_a_run():
    """Requests of a few tiles, several to a run: what is known of one request's tree is not taken for the next one's."""
    g = torch.Generator().manual_seed(23)
    lengths = torch.randint(0, 700, (70,), generator=g).tolist()
    parent = tree(4, 2, 4).repeat(70, 1)
    c = attention_case(lengths, parent, 8, 2, 128, torch.bfloat16, 16, seed=24, n_nodes=torch.randint(3, 20, (70,), generator=g).tolist())
    c["parent"][torch.rand(70, generator=g) < 0.4, 2] = 2
    want = ref.attention(**c)
    assert 10 < int((want["status"] == ref.TOPOLOGY).sum()) < 60
    for _ in range(5):
        check_attention(c, want)


# ---------------------------------------------------------------------------------------------
# tree_attention: what is noted of a tile arrives with it
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("D,heads,parent", [(128, (8, 2), tree(4, 2, 4)), (64, (6, 1), tree(8, 2, 6)), (128, (32, 8), tree(8, 2, 6)),
                                            (256, (4, 2), chain(1)), (64, (7, 1), chain(1))])
@pytest.mark.parametrize("block", [16, 24, 7])
def test_bad_blocks_in_many_tiles(D, heads, parent, block):
    """Tiles that hold bad blocks between tiles that do not, more of them than the notes of tiles under way have places: the keys that count as seen,
    and the copies that have to be told to the tensor cores, are those of the tile at hand, every time."""
    g = torch.Generator().manual_seed(D + block)
    c = attention_case([2600, 4100, 900], parent, *heads, D, torch.bfloat16, block, seed=D)
    used = -(-c["lengths"] // block)
    for b in range(3):
        hit = (torch.rand(int(used[b]) - 1, generator=g) < 0.05).nonzero().flatten()
        c["block_table"][b, hit] = torch.where(torch.rand(len(hit), generator=g) < 0.5, -1, 2**31 - 1).int()
    want = ref.attention(**c)
    assert want["status"].tolist()[:2] == [ref.PAGE] * 2          # (the short one may have drawn none)
    first = check_attention(c, want)
    for _ in range(10):
        again = check_attention(c, want)
        assert torch.equal(first.out, again.out) and torch.equal(first.lse, again.lse)


# ---------------------------------------------------------------------------------------------
# tree_attention: a wait that runs out
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("D,heads,parent", [(128, (8, 2), tree(4, 2, 4)), (128, (32, 8), tree(8, 2, 6)), (64, (7, 1), chain(1)),
                                            (256, (4, 2), tree(4, 2, 4))])
@pytest.mark.parametrize("block", [16, 7])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right(D, heads, parent, block):
    """One request's queries are never fetched (the library's test hook) and every wait gives up after 2e6 cycles, about a millisecond: the call
    comes back with SPEC_DEV_TIMEOUT, and what follows is as if nothing had been."""
    c = attention_case([2000, 300, -1, 40], parent.repeat(4, 1), *heads, D, torch.bfloat16, block, seed=D)
    c["parent"][3, -1] = parent.shape[0]
    want, d = ref.attention(**c), cuda(c)
    out = torch.full_like(d["q"], 7.0)
    try:
        binding.set_test_hooks(wait_cycles=2_000_000, hold_slot=1 * parent.shape[0])
        t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        t0.record()
        got = binding.tree_attention(**d, out=out, want_lse=True)
        t1.record()
        torch.cuda.synchronize()
        assert t0.elapsed_time(t1) < 500.0                        # milliseconds: bounded
        assert got.status.tolist() == [TIMEOUT, TIMEOUT, 0, ref.TOPOLOGY]
        assert bool((out[2] == 7.0).all()) and bool((out[3] == 0).all())
    finally:
        binding.set_test_hooks(0, -1)
    for _ in range(3):
        check_attention(c, want)


# ---------------------------------------------------------------------------------------------
# TreeCache: a pool that runs dry
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("side", [False, True])
def test_a_pool_that_runs_dry_in_mid_loop(side):
    """Refused steps are not committed, and the steps behind a release are right: entries and attention are those of a program that keeps every
    request's tokens in a list."""
    g = torch.Generator().manual_seed(3)
    B, block, blocks, Hq, Hkv, D = 3, 8, 9, 4, 2, 64
    parent = tree(3, 0, 3)
    N, tree_paths = len(parent), ref.paths(parent.tolist())
    cache = TreeCache(B, 1, blocks, block, Hkv, D, width=8)
    cache.storage.normal_()
    kept, refused, parent_d = [[] for _ in range(B)], 0, parent.cuda()
    stream = torch.cuda.Stream() if side else None
    torch.cuda.synchronize()
    for step in range(14):
        if step == 9:
            cache.release(2)
            kept[2] = []
        if step == 11:
            cache.lengths[2] = 0                                 # a new request
        torch.cuda.synchronize()
        s = cache.begin(parent_d, stream=stream)
        qkv = torch.randn(B * N, Hq + 2 * Hkv, D, generator=g).to(torch.bfloat16).cuda()
        torch.cuda.synchronize()
        q = cache.write(0, qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], torch.full((D // 2,), 0.01, device="cuda"), stream=stream)
        out = cache.attend(0, q.view(B, N, Hq, D), stream=stream)
        torch.cuda.synchronize()
        lengths, written = cache.lengths.tolist(), {}
        for b in range(B):
            if lengths[b] < 0 or s.status[b]:
                continue
            k, v = (cache.storage[i].flatten(0, 1)[s.slots[b].long()].cpu() for i in (0, 1))
            old, written[b] = kept[b], (k, v)
            c = dict(q=q.view(B, N, Hq, D)[b:b + 1].cpu(), k_cache=torch.stack([x for x, _ in old] + list(k))[None],
                     v_cache=torch.stack([x for _, x in old] + list(v))[None], parent=parent, block_table=torch.zeros(1, 1, dtype=I32),
                     lengths=torch.tensor([len(old)], dtype=I32))
            want = ref.attention(**c)
            bound = want["mass"] * (2.0**-8 + 2.0**-10) + want["out"].abs() * 2.0**-8
            assert out.status[b] == 0 and bool(((out.out[b:b + 1].cpu().double() - want["out"]).abs() <= bound).all())
        node = torch.randint(0, N, (B,), generator=g).int()
        accepted = node.cuda()
        torch.cuda.synchronize()
        done = cache.commit(accepted, stream=stream)
        torch.cuda.synchronize()
        for b in range(B):
            if s.status[b]:
                refused += 1
                assert int(done.status[b]) == int(s.status[b]) != 0 and int(done.lengths[b]) == lengths[b]
            elif lengths[b] >= 0:
                kept[b] += [(written[b][0][i], written[b][1][i]) for i in tree_paths[int(node[b])]]
                assert int(done.status[b]) == 0 and int(done.lengths[b]) == len(kept[b])
    assert refused > 3


# ---------------------------------------------------------------------------------------------
# tree_attention: exponentials
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("parent,heads", [(chain(1), (1, 1)), (tree(8, 2, 6), (4, 1))])
def test_every_exponential_is_as_good_as_the_sums(parent, heads):
    """Requests that each see one weight, 2^-(j / 64), at 16 keys of every place of a run of 16 (others far below), beside two weights of 1: the
    sum shows how far the weight is off."""
    B, N, length = 161, parent.shape[-1], 128
    for place in range(0, 16, 2):
        c = attention_case([length] * B, parent, *heads, 64, torch.bfloat16, 16, seed=1, scale=math.log(2.0))
        c["q"].zero_()
        c["q"][..., 0] = 1.0
        c["k_cache"].zero_()
        y = torch.arange(B) / 64.0
        at = torch.arange(length)
        for b in range(B):
            here = (at % 16 == place) | (at % 16 == place + 1)
            score = torch.where(here, -y[b], -120.0)
            score[(place + 8) % 16] = 0.0                         # (the reference of this tile, whoever else works on others)
            c["k_cache"][c["block_table"][b, at // 16].long(), at % 16, 0, 0] = score.to(torch.bfloat16)
            c["k_cache"][c["block_table"][b, length // 16:(length + N + 15) // 16].long()] = 0.0
        lse = binding.tree_attention(**cuda(c), want_lse=True).lse[:, 0, 0].cpu().double()
        scale = float(torch.tensor(math.log(2.0)).float())
        want = torch.log(2.0 + 16.0 * torch.exp(-y.double() * scale))
        # eleven sums of one rounding each, 2^-22 for an exponential, the exponent (scale, its product with log2 e, a score of y) and the
        # logarithm with its product by ln 2 to two roundings
        bound = 11 * 2.0**-24 + 2.0**-22 + y.double() * 2.0**-23 + want.abs() * 2.0**-23
        assert bool(((lse - want).abs() <= bound).all()), (place, float(((lse - want).abs() - bound).max()))


# ---------------------------------------------------------------------------------------------
# verify_probs: infinities that are not at a drafted token
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [7, 1000, 4097, 128256])
def test_chains_with_infinities_beside_the_drafted_token(dtype, V):
    inf, nan = math.inf, math.nan
    c = chains_case([2] * 8, V, dtype, seed=V)
    c["u_accept"][:] = 1.0 - 2**-24
    first = torch.arange(8) * 2
    c["target_probs"][first + torch.arange(8), c["token"][first].long()] *= 0.25        # every first draft is rejected
    other = (c["token"][first].long() + 3) % V
    for b, (p, q) in enumerate([(inf, inf), (inf, None), (None, inf), (nan, inf), (None, nan), (inf, nan), (torch.finfo(dtype).max, inf), (-inf, -inf)]):
        if p is not None:
            c["target_probs"][3 * b, other[b]] = p
        if q is not None:
            c["draft_probs"][2 * b, other[b]] = q
    want = check_chains(c)
    assert want["status"].tolist() == [3, 3, 0, 3, 3, 3, 0, 3]
    lookup = dict(c, draft_probs=None)
    lookup["target_probs"] = c["target_probs"].clone()
    lookup["target_probs"][6 * 3, other[6]] = 0.5
    assert check_chains(lookup)["status"].tolist() == [3, 3, 0, 3, 0, 3, 0, 0]


# ---------------------------------------------------------------------------------------------
# tree_attention: scores of -inf
# ---------------------------------------------------------------------------------------------
def attended(c, hidden=None):
    """One request's rows in 64 bits, straight from the definition."""
    N, Hq, D = c["q"].shape[1:]
    block, G, length = c["k_cache"].shape[1], Hq // c["k_cache"].shape[2], int(c["lengths"][0])
    at = torch.arange(length + N)
    k = c["k_cache"][c["block_table"][0, at // block].long(), at % block].double().repeat_interleave(G, 1)
    v = c["v_cache"][c["block_table"][0, at // block].long(), at % block].double().repeat_interleave(G, 1)
    seen = torch.zeros(N, length + N, dtype=torch.bool)
    seen[:, :length] = True
    for i, p in enumerate(ref.paths(c["parent"].tolist())):
        seen[i, [length + x for x in p]] = True
    score = (c["q"][0].double()[:, :, None] * k.transpose(0, 1)[None]).sum(-1) * D ** -0.5
    if hidden is not None:
        seen[:, hidden] = False
    score = torch.where(seen[:, None], score, -math.inf)
    return torch.softmax(score, -1), v, torch.logsumexp(score, -1)


@pytest.mark.parametrize("length", [0, 40, 300, 3000])
@pytest.mark.parametrize("parent,heads", [(chain(1), (4, 1)), (tree(4, 2, 4), (4, 2)), (tree(8, 2, 6), (8, 2))])
def test_scores_of_minus_infinity(length, parent, heads):
    """A row whose only scores are -inf is 0 / 0, no number; one that has others besides takes no notice of them; the log of the sum is that of 0."""
    N = parent.shape[-1]
    c = attention_case([length], parent, *heads, 128, torch.bfloat16, 16, seed=length + N)
    c["q"] = c["q"].abs() + 0.125
    c["k_cache"][..., 3] = -math.inf
    got = binding.tree_attention(**cuda(c), want_lse=True)
    assert got.status.tolist() == [0] and bool(got.out.isnan().all()) and bool((got.lse == -math.inf).all())
    # one tree node with a finite key: its own row and those below it are its value
    node = N // 2
    c["k_cache"][c["block_table"][0, (length + node) // 16].long(), (length + node) % 16, :, 3] = 1.0
    got = binding.tree_attention(**cuda(c), want_lse=True)
    below = torch.tensor([node in p for p in ref.paths(parent.tolist())])
    v = c["v_cache"][c["block_table"][0, (length + node) // 16].long(), (length + node) % 16].repeat_interleave(heads[0] // heads[1], 0)
    assert bool((got.out[0, below].cpu() == v).all()) and bool(got.lse[0, below].isfinite().all())
    assert bool(got.out[0, ~below].isnan().all()) and bool((got.lse[0, ~below] == -math.inf).all())
    # all keys of the context finite but for one in three: rows are what the others give
    c["k_cache"][..., 3] = 1.0
    at = torch.arange(0, length + N, 3)
    c["k_cache"][c["block_table"][0, at // 16].long(), at % 16, :, 3] = -math.inf
    got = binding.tree_attention(**cuda(c), want_lse=True)
    p, v, lse = attended(c, at)
    some = lse.isfinite()
    bound = torch.einsum("nhj,jhd->nhd", p, v.abs()) * (2.0**-8 + 2.0**-10) + 2.0**-8 * torch.einsum("nhj,jhd->nhd", p, v).abs()
    off = (got.out[0].cpu().double() - torch.einsum("nhj,jhd->nhd", p, v)).abs()
    assert bool((off <= bound)[some].all()) and bool(got.out[0].cpu()[~some].isnan().all())
    assert bool(((got.lse[0].cpu().double() - lse).abs() <= 2.0**-16 * (1 + lse.abs()))[some].all())


def test_scores_of_minus_infinity_beside_bad_blocks_and_windows():
    """A row that sees nothing is 0; one that sees keys, all at -inf, is no number, also where the rest is hidden or left behind by the window."""
    parent = tree(4, 2, 4)
    for window, sinks in ((0, 0), (30, 3), (1, 0)):
        c = attention_case([700, 700], parent, 8, 2, 128, torch.bfloat16, 16, seed=31, window=window, sinks=sinks)
        c["q"] = c["q"].abs() + 0.125
        c["k_cache"][..., 3] = -math.inf
        c["block_table"][0] = -1                                  # sees nothing
        c["block_table"][1, :20] = -1                             # sees the rest
        got = binding.tree_attention(**cuda(c), want_lse=True)
        assert bool((got.out[0] == 0).all()) and bool(got.out[1].isnan().all()) and bool((got.lse == -math.inf).all())


# ---------------------------------------------------------------------------------------------
# what autograd knows of the calls
# ---------------------------------------------------------------------------------------------
def small_calls():
    r = cuda(rope_case(3, 2, 1, 64, 64, torch.bfloat16))
    a = cuda(attention_case([10], tree(1, 0, 1), 2, 1, 64, torch.bfloat16, 16))
    m = cuda(commit_case([5], tree(1, 0, 1), [1], 2, (16,), torch.float32, 16))
    return [(binding.norm_rope_cache, r, ("q", "k", "v", "inv_freq", "q_weight", "k_weight", "k_cache", "v_cache")),
            (binding.tree_attention, a, ("q", "k_cache", "v_cache")), (binding.cache_commit, m, ("cache",))]


def test_tangents_and_gradients_are_not_dropped():
    for call, args, names in small_calls():
        for name in names:
            with pytest.raises(RuntimeError, match="backward"):
                call(**dict(args, **{name: args[name].clone().requires_grad_()}))
            with torch.no_grad():
                call(**dict(args, **{name: args[name].clone().requires_grad_()}))
            with torch.autograd.forward_ad.dual_level():
                dual = torch.autograd.forward_ad.make_dual(args[name].clone(), torch.ones_like(args[name]))
                with pytest.raises(RuntimeError, match="tangent"):
                    call(**dict(args, **{name: dual}))


def test_writes_in_place_are_known_to_autograd():
    for call, args, _ in small_calls():
        written = {"norm_rope_cache": ("k_cache", "v_cache", "q_out"), "tree_attention": ("out",), "cache_commit": ("cache",)}[call.__name__]
        args = dict(args)
        for name in ("q_out", "out"):
            if name in written:
                args[name] = torch.empty_like(args["q"])
        for name in written:
            w = torch.ones_like(args[name]).requires_grad_()
            y = (w * args[name]).sum()                            # keeps what it multiplies by for its backward pass
            call(**args)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                y.backward()
    c = slots_case(2, 3, 8, 1)
    d = cuda(c)
    before = d["block_table"]._version
    binding.cache_slots(**d)
    assert d["block_table"]._version == before + 1


def test_tensors_of_inference_mode_are_taken():
    for call, args, _ in small_calls():
        with torch.inference_mode():
            frozen = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in args.items()}
            call(**frozen)
        call(**frozen)


# ---------------------------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------------------------
def test_written_tensors_whose_entries_share_memory_are_refused():
    r, a, m = (args for _, args, _ in small_calls())
    for call, args, names in ((binding.norm_rope_cache, dict(r, q_out=r["q"].clone()), ("k_cache", "v_cache", "q_out")),
                              (binding.tree_attention, dict(a, out=a["q"].clone()), ("out",)), (binding.cache_commit, m, ("cache",))):
        call(**args)
        for name in names:
            for dim in range(args[name].dim() - 1):
                if args[name].size(dim) > 1:
                    with pytest.raises(RuntimeError, match="share memory"):
                        call(**dict(args, **{name: args[name].narrow(dim, 0, 1).expand_as(args[name])}))
    call(**dict(m, cache=m["cache"][:1]))


# ---------------------------------------------------------------------------------------------
# tree_attention: many short units, many times
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("heads,D,window,shape", [((32, 8), 128, 0, (8, 2, 6)), ((8, 1), 64, 60, (8, 2, 6)), ((4, 2), 256, 0, (8, 2, 6)),
                                                  ((8, 2), 128, 0, (8, 2, 6)), ((32, 8), 128, 500, None), ((14, 2), 64, 0, None),
                                                  ((8, 4), 256, 0, None), ((16, 4), 64, 0, (4, 2, 4))])
def test_calls_with_many_short_units(heads, D, window, shape):
    """Warps come to a unit's end, and to the next one's beginning, at different times, some with nothing to do: whoever comes late finds the others'
    work done, or not, and goes on alike."""
    g = torch.Generator().manual_seed(4)
    parent = tree(*shape) if shape else chain(1)
    lengths = torch.randint(0, 300, (60,), generator=g).tolist()
    nodes = torch.randint(0, parent.shape[-1] + 1, (60,), generator=g).tolist() if shape else None
    c = attention_case(lengths, parent, *heads, D, torch.bfloat16, 16, seed=6, n_nodes=nodes, window=window, sinks=2)
    want, d = ref.attention(**c), cuda(c)
    first = check_attention(c, want)
    live = want["live"].cuda()
    wrong = torch.zeros((), dtype=torch.int32, device="cuda")
    for _ in range(3000):
        again = binding.tree_attention(**d)
        wrong += (again.status != first.status).any() | (again.out[live] != first.out[live]).any()
    assert int(wrong) == 0


def test_a_flag_that_is_no_truth_value_is_refused():
    d = cuda(attention_case([10], tree(1, 0, 1), 2, 1, 64, torch.bfloat16, 16))
    with pytest.raises(RuntimeError, match="ambiguous"):
        binding.tree_attention(**d, want_lse=torch.ones(2))


# ---------------------------------------------------------------------------------------------
# tree_attention: what belongs to nodes beyond n_nodes, and lengths beyond the table
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("heads", [(8, 2), (6, 2), (32, 8)])
@pytest.mark.parametrize("shape", [(4, 2, 4), (8, 2, 6)])
def test_what_belongs_to_nodes_beyond_a_tree_reaches_no_row(heads, shape):
    parent = tree(*shape)
    N = parent.shape[-1]
    nodes = [1, N, 0, N // 2, 7]
    c = attention_case([50, 300, 7, 0, 900], parent.repeat(5, 1), *heads, 128, torch.bfloat16, 16, seed=41, n_nodes=nodes)
    want = ref.attention(**c)
    for b, n in enumerate(nodes):
        c["q"][b, n:] = float("nan")
        c["parent"][b, n:] = 2**31 - 1
        at = torch.arange(int(c["lengths"][b]) + n, int(c["lengths"][b]) + N)
        for name in ("k_cache", "v_cache"):
            c[name][c["block_table"][b, at // 16].long(), at % 16] = float("nan")
    check_attention(c, want)


@pytest.mark.parametrize("window", [0, 50])
def test_rows_of_lengths_beyond_the_table_are_those_of_its_keys(window):
    c = attention_case([100], tree(4, 2, 4), 4, 2, 128, torch.bfloat16, 16, seed=14, window=window, sinks=3)
    held = int((c["block_table"][0] >= 0).sum()) * 16             # (the tree itself lies beyond)
    c["lengths"][0] = 2**31 - 1 - 19
    got = binding.tree_attention(**cuda(c), want_lse=True)
    assert got.status.tolist() == [ref.PAGE]
    at = torch.arange(3 if window else held)
    k = c["k_cache"][c["block_table"][0, at // 16].long(), at % 16].double().repeat_interleave(2, 1)
    v = c["v_cache"][c["block_table"][0, at // 16].long(), at % 16].double().repeat_interleave(2, 1)
    score = torch.einsum("nhd,jhd->nhj", c["q"][0].double(), k) * 128 ** -0.5
    p = torch.softmax(score, -1)
    want = torch.einsum("nhj,jhd->nhd", p, v)
    bound = torch.einsum("nhj,jhd->nhd", p, v.abs()) * (2.0**-8 + 2.0**-10) + want.abs() * 2.0**-8
    assert bool(((got.out[0].cpu().double() - want).abs() <= bound).all())
    assert bool(((got.lse[0].cpu().double() - torch.logsumexp(score, -1)).abs() <= 2.0**-16).all())
