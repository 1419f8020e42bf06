"""The operators around a verification against their restatements in 64 bits, at sizes, trees, masks and layouts where they can go wrong."""
import math

import numpy as np
import pytest
import torch

from . import step_ref as ref
from paper_2602_16994_b200 import binding, synth
from paper_2602_16994_b200.tree_cache import TreeCache

pytestmark = pytest.mark.gpu

I32 = torch.int32


def tree(K, L1, L2):
    return torch.tensor(synth.delayed_tree(K, L1, L2)[0], dtype=I32)


def random_tree(n, g):
    return torch.tensor([-1] + [int(torch.randint(0, i, (1,), generator=g)) for i in range(1, n)], dtype=I32)


def chain(n):
    return torch.arange(-1, n - 1, dtype=I32)


def cuda(x):
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in x.items()}


def pages(lengths, n, block, g, spare=3):
    """A block table of distinct, shuffled blocks for lengths + n entries per request, and the number of blocks."""
    used = [max(0, -(-(max(0, int(x)) + n) // block)) for x in lengths]
    ids = torch.randperm(sum(used) + spare, generator=g).int()
    table = torch.full((len(lengths), max(1, max(used)) + 1), -1, dtype=I32)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = ids[at:at + u]
        at += u
    return table, sum(used) + spare


# ---------------------------------------------------------------------------------------------
# cache_slots
# ---------------------------------------------------------------------------------------------
def slots_case(B, N, block, seed, most=300, per_request=False, ragged=False, short_ring=None):
    g = torch.Generator().manual_seed(seed)
    lengths = torch.randint(0, most, (B,), generator=g).int()
    owned = -(-lengths // block)
    width = -(-(most + N) // block)
    ids = torch.randperm(B * width + 64, generator=g).int()
    table = torch.full((B, width), -1, dtype=I32)
    for b in range(B):
        table[b, :owned[b]] = ids[b * width:b * width + int(owned[b])]
    free = ids[B * width:]
    size = B * (N // block + 2) + 5
    ring = torch.full((size,), -7, dtype=I32)
    count = size - 3 if short_ring is None else short_ring
    begin = int(torch.randint(0, size, (1,), generator=g))
    fresh = torch.arange(100000, 100000 + count).int()
    ring[(begin + torch.arange(count)) % size] = fresh
    parent = torch.stack([random_tree(N, g) for _ in range(B)]) if per_request else random_tree(N, g)
    n_nodes = torch.randint(0, N + 1, (B,), generator=g).int() if ragged else None
    return dict(lengths=lengths, parent=parent, block_table=table, owned=owned.int(), free_blocks=ring,
                free_range=torch.tensor([begin, count], dtype=I32), block_size=block, n_nodes=n_nodes)


def check_slots(c):
    want = ref.cache_slots(c["lengths"], c["parent"], c["block_table"], c["owned"], c["free_blocks"], c["free_range"],
                           c["block_size"], c["n_nodes"])
    d = cuda(c)
    for _ in range(2):                                           # (the call can be repeated)
        got = binding.cache_slots(**d)
        for name in ("status", "owned", "free_range", "block_table", "slots", "positions"):
            assert torch.equal(getattr(got, name).cpu(), want[name]), name
        assert got.block_table is d["block_table"] or got.block_table.data_ptr() == d["block_table"].data_ptr()
    return want


@pytest.mark.parametrize("B,N,block", [(1, 1, 1), (1, 1, 16), (8, 19, 16), (9, 51, 7), (3, 1024, 64), (257, 5, 16), (2500, 3, 24)])
@pytest.mark.parametrize("per_request,ragged", [(False, False), (True, True)])
def test_slots(B, N, block, per_request, ragged):
    if per_request and B * N > 10000:
        B = 300
    check_slots(slots_case(B, N, block, B + N, per_request=per_request, ragged=ragged))


@pytest.mark.parametrize("ring", [0, 1, 5, 17])
def test_slots_of_a_ring_that_runs_dry(ring):
    want = check_slots(slots_case(40, 19, 16, ring, short_ring=ring))
    assert (want["status"] == ref.BLOCKS).any()


def test_slots_idle_bad_and_full_rows():
    c = slots_case(12, 9, 8, 3, per_request=True, ragged=True)
    c["lengths"][1] = -1                                         # idle
    c["lengths"][2] = 2**31 - 1                                  # longer than any table
    c["owned"][3] = c["block_table"].shape[1] + 1
    c["owned"][4] = -1
    c["n_nodes"][5], c["n_nodes"][6], c["n_nodes"][7], c["n_nodes"][8] = 10, -1, 9, 9
    c["parent"][7, 4] = 4                                        # its own parent
    c["parent"][8, 0] = 0
    c["n_nodes"][9] = 9
    c["lengths"][9], c["owned"][9] = 20, 3
    c["block_table"][9, 2] = -1                                  # a block that it says it owns
    want = check_slots(c)
    assert want["status"].tolist()[1:10] == [0, 6, 6, 6, 1, 1, 1, 1, 5]


def test_slots_from_a_range_outside_the_ring():
    c = slots_case(4, 9, 8, 5)
    c["free_range"] = torch.tensor([len(c["free_blocks"]), 3], dtype=I32)
    check_slots(c)
    c["free_blocks"] = torch.zeros(0, dtype=I32)
    c["free_range"] = torch.zeros(2, dtype=I32)
    check_slots(c)


# ---------------------------------------------------------------------------------------------
# norm_rope_cache
# ---------------------------------------------------------------------------------------------
def rope_case(T, Hq, Hkv, D, rot, dtype, block=16, seed=0, norm=True, fused=True, top=100000):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(T, Hq + 2 * Hkv, D, generator=g).to(dtype)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    blocks = -(-(T + 5) // block) + 1
    w = [(1 + 0.2 * torch.randn(D, generator=g)).to(dtype) if norm else None for _ in range(2)]
    return dict(q=q, k=k, v=v, inv_freq=(10000.0 ** (-torch.arange(0, rot, 2).double() / max(1, rot))).float(),
                positions=torch.randint(0, top, (T,), generator=g).int(), slots=torch.randperm(blocks * block, generator=g)[:T].int(),
                k_cache=torch.randn(blocks, block, Hkv, D, generator=g).to(dtype),
                v_cache=torch.randn(blocks, block, Hkv, D, generator=g).to(dtype), q_weight=w[0], k_weight=w[1])


def check_rope(c, pairs, q_out=None, eps=1e-6, **moved):
    dtype, half = c["q"].dtype, torch.finfo(c["q"].dtype).eps / 2
    block, n_slots = c["k_cache"].shape[1], c["k_cache"].shape[0] * c["k_cache"].shape[1]
    d = dict(cuda(c), **moved)
    before = d["q"].clone() if q_out is None else None
    got = binding.norm_rope_cache(**d, pairs=pairs, q_out=q_out, eps=eps)
    live = (c["slots"] >= 0) & (c["slots"] < n_slots)

    def near(x, want, size):
        # fp32 up to the end: 12 roundings of the norm (half of the sum's own 13, root, quotient, products), a cosine and a sine to 2^-22,
        # two products and a sum: below 2^-21 of |a| + |b|; then one rounding, of at most half a step (a step of denormals: below 2^-24)
        bound = size * 2.0**-21 + want.abs() * half + (2.0**-25 if dtype == torch.float16 else 0)
        assert bool(((x.cpu().double() - want).abs() <= bound).all()), float(((x.cpu().double() - want).abs() - bound).max())

    want, size = ref.norm_rope(c["q"], c["q_weight"], c["inv_freq"], c["positions"], eps, pairs)
    near(got[live], want[live], size[live])
    want, size = ref.norm_rope(c["k"], c["k_weight"], c["inv_freq"], c["positions"], eps, pairs)
    at = c["slots"][live].long()
    near(d["k_cache"][at // block, at % block], want[live], size[live])
    assert torch.equal(d["v_cache"][at // block, at % block].cpu(), c["v"][live])
    rest = torch.ones(n_slots, dtype=torch.bool)
    rest[at] = False
    for name in ("k_cache", "v_cache"):
        assert torch.equal(d[name].flatten(0, 1).cpu()[rest], c[name].flatten(0, 1)[rest])
    if before is not None:
        assert torch.equal(d["q"], before)
    return got


@pytest.mark.parametrize("T,Hq,Hkv,D,rot", [(1, 1, 1, 64, 64), (19, 32, 8, 128, 128), (7, 14, 2, 64, 32), (33, 4, 4, 256, 256),
                                            (5, 3, 1, 80, 80), (6, 6, 2, 96, 48), (4, 2, 1, 8, 0), (3, 5, 5, 16, 16),
                                            (2, 71, 1, 128, 96), (300, 8, 8, 128, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
def test_norm_rope(T, Hq, Hkv, D, rot, dtype, pairs):
    check_rope(rope_case(T, Hq, Hkv, D, rot, dtype, seed=T + D), pairs)


def test_norm_rope_without_norms_far_positions_and_odd_blocks():
    c = rope_case(40, 4, 2, 128, 128, torch.float32, block=7, norm=False, top=2**31 - 1)
    check_rope(c, "halves")


def test_norm_rope_skips_padding():
    c = rope_case(40, 4, 2, 128, 64, torch.bfloat16, seed=3)
    c["slots"][[0, 7, 39]] = torch.tensor([-1, -5, c["k_cache"].shape[0] * 16], dtype=I32)
    c["q"][[0, 7, 39]] = float("nan")
    out = torch.full((40, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    check_rope(c, "neighbours", q_out=out)
    assert bool((out[[0, 7, 39]] == 3.0).all())


@pytest.mark.parametrize("D", [128, 64])
def test_norm_rope_skips_padding_between_the_tokens_of_a_cta(D):
    # far more tokens than CTAs, half of them left out at random: a CTA's next token may come right behind the last, or several places on
    c = rope_case(5000, 6, 2, D, D, torch.bfloat16, seed=6)
    c["slots"][torch.rand(5000, generator=torch.Generator().manual_seed(7)) < 0.5] = -1
    for pairs in ("halves", "neighbours"):
        check_rope(c, pairs)


def test_norm_rope_in_place_and_unaligned():
    c = rope_case(21, 6, 2, 64, 64, torch.bfloat16, seed=4)
    wide = torch.zeros(21, 10, 67, dtype=torch.bfloat16, device="cuda")           # rows that start on no 16 bytes
    q, k, v = wide[:, :6, 3:], wide[:, 6:8, 3:], wide[:, 8:, 3:]
    q.copy_(c["q"]), k.copy_(c["k"]), v.copy_(c["v"])
    check_rope(c, "halves", q_out=q, q=q, k=k, v=v)


def test_norm_rope_of_zero_rows_and_no_tokens():
    c = rope_case(3, 2, 1, 64, 64, torch.float16, seed=5)
    c["q"].zero_(), c["k"].zero_()
    check_rope(c, "halves")
    e = rope_case(1, 2, 1, 64, 64, torch.float16)
    for name in ("q", "k", "v", "positions", "slots"):
        e[name] = e[name][:0]
    assert binding.norm_rope_cache(**cuda(e)).shape == (0, 2, 64)


# ---------------------------------------------------------------------------------------------
# tree_attention
# ---------------------------------------------------------------------------------------------
def attention_case(lengths, parent, Hq, Hkv, D, dtype, block, seed=0, n_nodes=None, spread=2.0, **kw):
    g = torch.Generator().manual_seed(seed)
    lengths, N = torch.tensor(lengths, dtype=I32), parent.shape[-1]
    table, blocks = pages(lengths, N, block, g)
    return dict(q=(spread * torch.randn(len(lengths), N, Hq, D, generator=g)).to(dtype),
                k_cache=torch.randn(blocks, block, Hkv, D, generator=g).to(dtype),
                v_cache=torch.randn(blocks, block, Hkv, D, generator=g).to(dtype), block_table=table, lengths=lengths, parent=parent,
                n_nodes=None if n_nodes is None else torch.tensor(n_nodes, dtype=I32), **kw)


def check_attention(c, want=None, stream=None, **moved):
    want = want or ref.attention(**c)
    dtype = c["q"].dtype
    B, N, Hq, D = c["q"].shape
    d = dict(cuda(c), **moved)
    out = d.pop("out", None)
    if out is None:
        out = torch.full((B, N, Hq, D), 7.0, dtype=dtype, device="cuda")
    got = binding.tree_attention(**d, out=out, want_lse=True, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(got.status.cpu(), want["status"])
    x, lse, live = got.out.cpu().double(), got.lse.cpu().double(), want["live"]
    half = torch.finfo(dtype).eps / 2
    # a score: D products and sums in fp32, each within 2^-24 of the sum of their sizes, and the product with the scale; a weight
    # from it: twice that (its own exponent and the sum's), 2^-20 for exponentials and sums, half a step of its rounding to the
    # type of the values; fp16 weights below 2^-14 are rounded to steps of 2^-24, which 2^-12 of the largest weight bounds over 4096 keys;
    # the result's own rounding
    score = want["reach"][..., None] * (D + 4) * 2.0**-24
    bound = want["mass"] * (2 * score + half + 2.0**-20) + want["out"].abs() * half
    if dtype == torch.float16:
        bound = bound + 2.0**-12 * half * 4 + 2.0**-25
    off = (x - want["out"]).abs()
    same = (x == want["out"]) | (x.isnan() & want["out"].isnan())
    assert bool(((off <= bound) | same)[live].all()), float((off - bound)[live & ~same.all(-1).all(-1)].max())
    assert bool((x[~live] == 7.0).all())
    off = (lse - want["lse"]).abs()
    same = (lse == want["lse"]) | (lse.isnan() & want["lse"].isnan())
    assert bool(((off <= score[..., 0] * 2 + 2.0**-18 + want["lse"].abs() * 2.0**-22) | same)[live].all())
    return got


TREES = {"token": chain(1), "d2k4": tree(4, 2, 4), "k8": tree(8, 2, 6), "pair": tree(1, 0, 1)}


@pytest.mark.parametrize("lengths", [[0], [1], [15, 16, 17], [127, 128, 129, 0], [300, 5, 1000]])
@pytest.mark.parametrize("shape", ["token", "d2k4", "k8"])
@pytest.mark.parametrize("Hq,Hkv,D,dtype,block", [(4, 1, 128, torch.bfloat16, 16), (6, 2, 64, torch.float16, 7), (8, 8, 128, torch.float16, 32),
                                                  (4, 2, 256, torch.bfloat16, 16), (16, 2, 64, torch.bfloat16, 1),
                                                  (4, 1, 64, torch.bfloat16, 24), (4, 1, 128, torch.bfloat16, 256),
                                                  (5, 1, 256, torch.float16, 8)])
def test_attention(lengths, shape, Hq, Hkv, D, dtype, block):
    check_attention(attention_case(lengths, TREES[shape], Hq, Hkv, D, dtype, block, seed=sum(lengths) + D))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 0), (16, 4), (100, 0), (128, 130), (129, 3), (400, 64), (5000, 4)])
@pytest.mark.parametrize("D,dtype", [(128, torch.bfloat16), (64, torch.float16)])
def test_attention_with_a_window(window, sinks, D, dtype):
    c = attention_case([700, 3, 260, 0], tree(3, 1, 5), 4, 2, D, dtype, 16, seed=window, window=window, sinks=sinks)
    check_attention(c)


@pytest.mark.parametrize("n,heads", [(33, 4), (64, 2), (65, 4), (129, 1), (200, 7)])
def test_attention_of_random_trees(n, heads):
    g = torch.Generator().manual_seed(n)
    parent = torch.stack([random_tree(n, g), chain(n), torch.tensor([-1] + [0] * (n - 1), dtype=I32)])
    check_attention(attention_case([40, 129, 0], parent, heads, 1, 128, torch.bfloat16, 16, seed=n))


def test_attention_of_a_stretch_of_a_prompt():
    check_attention(attention_case([77], chain(1024), 2, 1, 64, torch.bfloat16, 16, seed=9))
    check_attention(attention_case([77], chain(700), 2, 1, 128, torch.float16, 64, seed=10, window=90, sinks=2))


def test_attention_of_ragged_trees_and_idle_requests():
    c = attention_case([50, -1, 200, 0, 31, 64], tree(4, 2, 4), 8, 2, 128, torch.bfloat16, 16, n_nodes=[1, 19, 0, 7, 20, 19])
    want = ref.attention(**c)
    assert want["status"].tolist() == [0, 0, 0, 0, 1, 0]
    check_attention(c, want)


def test_attention_of_ragged_trees_in_two_blocks_of_rows():
    """Requests of which the second block of 128 rows, or half of it, has nothing to do, beside ones that fill it; several to a CTA."""
    g = torch.Generator().manual_seed(4)
    lengths = torch.randint(0, 300, (40,), generator=g).tolist()
    nodes = torch.randint(0, 52, (40,), generator=g).tolist()
    lengths[5] = -1
    check_attention(attention_case(lengths, tree(8, 2, 6), 32, 8, 128, torch.bfloat16, 16, seed=6, n_nodes=nodes))
    check_attention(attention_case(lengths, tree(8, 2, 6), 8, 1, 64, torch.float16, 16, seed=7, n_nodes=nodes, window=60, sinks=2))


def test_attention_of_nobody():
    c = attention_case([-1, -5], tree(4, 2, 4), 4, 2, 128, torch.bfloat16, 16)
    assert check_attention(c).status.tolist() == [0, 0]
    c = attention_case([9, 0], tree(4, 2, 4), 4, 2, 128, torch.bfloat16, 16, n_nodes=[0, 0])
    assert check_attention(c).status.tolist() == [0, 0]


@pytest.mark.parametrize("window", [0, 50])
def test_attention_of_lengths_beyond_the_table(window):
    """Whatever a length says, only the table's blocks are gone through; rows that see some of them are what those give."""
    c = attention_case([100, 40], tree(4, 2, 4), 4, 2, 128, torch.bfloat16, 16, seed=14, window=window, sinks=3)
    want = ref.attention(**c)
    c["lengths"][0] = 2**31 - 1 - 19
    got = binding.tree_attention(**cuda(c))
    assert got.status.tolist() == [5, 0]
    assert bool(got.out[0].isfinite().all())
    assert torch.equal(got.out[1], binding.tree_attention(**cuda(dict(c, q=c["q"][1:], block_table=c["block_table"][1:], lengths=c["lengths"][1:]))).out[0])
    assert bool(((got.out[1].cpu().double() - want["out"][1]).abs() <= want["mass"][1] * 2.0**-7).all())


def test_attention_of_many_requests():
    g = torch.Generator().manual_seed(1)
    lengths = torch.randint(0, 40, (300,), generator=g).tolist()
    check_attention(attention_case(lengths, tree(2, 1, 2), 4, 2, 64, torch.bfloat16, 16, seed=2))


@pytest.mark.parametrize("lengths", [[20000], [9000, 3, 5000, 700]])
def test_attention_over_long_contexts(lengths):
    """Long axes are split over the chip and joined."""
    check_attention(attention_case(lengths, tree(2, 1, 2), 4, 1, 128, torch.bfloat16, 16, seed=5))


@pytest.mark.parametrize("spread", [0.0, 30.0])
def test_attention_flat_and_sharp(spread):
    check_attention(attention_case([500, 129], tree(4, 2, 4), 4, 2, 128, torch.bfloat16, 16, spread=spread))


def test_attention_whose_scores_rise_along_the_context():
    """Every tile raises the running maximum by far."""
    for sign in (1.0, -1.0):
        c = attention_case([900], tree(4, 2, 4), 4, 1, 128, torch.bfloat16, 16, seed=3)
        c["q"] = torch.ones_like(c["q"])
        for j in range(900 + 19):
            c["k_cache"][c["block_table"][0, j // 16], j % 16] = sign * (j - 450) / 64.0
        check_attention(c)


@pytest.mark.parametrize("scale", [0.0, 0.01, 1.0])
def test_attention_scale(scale):
    check_attention(attention_case([200], tree(4, 2, 4), 4, 1, 64, torch.bfloat16, 16, scale=scale))


def test_attention_keeps_what_a_row_does_not_see_out_of_it():
    """NaN and infinities in unseen places: unused slots, other branches, beyond the window's edge, unlisted blocks."""
    parent = tree(4, 2, 4)
    for fill in (float("nan"), float("inf"), -float("inf")):
        c = attention_case([301, 40], parent, 8, 2, 128, torch.bfloat16, 16, seed=11, window=64, sinks=3)
        want = ref.attention(**c)
        bad = {k: c[k].clone() for k in ("k_cache", "v_cache")}
        for b, length in enumerate([301, 40]):
            seen = torch.zeros(c["block_table"].shape[1] * 16, dtype=torch.bool)
            seen[length:length + 19] = True
            at = torch.arange(len(seen))
            seen |= (at < length) & ((at < 3) | (at > length - 64))
            for j in (~seen).nonzero().flatten().tolist():
                if c["block_table"][b, j // 16] >= 0:
                    for name in bad:
                        bad[name][c["block_table"][b, j // 16], j % 16] = fill
        check_attention(dict(c, **bad), want)
        # one branch's node, and the context's oldest key that the root sees: rows that see them may be anything, the others may not
        for b, j, hit in ((0, 301 + 7, [7, 8, 9, 10]), (0, 301 - 63, [0]), (1, 40 + 18, [18])):
            bad = {k: c[k].clone() for k in ("k_cache", "v_cache")}
            for name in bad:
                bad[name][c["block_table"][b, j // 16], j % 16] = fill
            got = binding.tree_attention(**dict(cuda(c), **cuda(bad)))
            clean = binding.tree_attention(**cuda(c))
            rows = torch.ones(2, 19, dtype=torch.bool)
            tree_paths = ref.paths(parent.tolist())
            if j >= [301, 40][b]:
                hit = [i for i in range(19) if j - [301, 40][b] in tree_paths[i]]
            rows[b, hit] = False
            # (a sum over other tiles' order is the same sum: the rows agree to the bit)
            assert torch.equal(got.out.cpu()[rows], clean.out.cpu()[rows])
            assert not bool(got.out.cpu()[~rows].isfinite().all())


def test_attention_passes_on_what_a_row_sees():
    """A NaN in a seen value's entry reaches that entry of the rows that see it, and only it."""
    parent = tree(4, 2, 4)
    c = attention_case([301], parent, 4, 1, 128, torch.bfloat16, 16, seed=12)
    c["v_cache"][c["block_table"][0, 308 // 16], 308 % 16, 0, 5] = float("nan")
    c["v_cache"][c["block_table"][0, 302 // 16], 302 % 16, 0, 9] = float("inf")
    c["v_cache"][c["block_table"][0, 17 // 16], 17 % 16, 0, 77] = float("nan")
    got = binding.tree_attention(**cuda(c)).out.cpu()[0]
    tree_paths = ref.paths(parent.tolist())
    want = torch.zeros(19, 128, dtype=torch.bool)
    want[:, 77] = True
    for i in range(19):
        want[i, 5] |= 7 in tree_paths[i]
        want[i, 9] |= 1 in tree_paths[i]
    assert torch.equal(~got.isfinite(), want[:, None].expand_as(got))
    assert bool((got[1:, :, 9] == float("inf")).all())


@pytest.mark.parametrize("length", [40, 301, 700])
@pytest.mark.parametrize("fill", [float("nan"), float("inf")])
def test_attention_of_keys_that_are_no_numbers(length, fill):
    """Rows that see such a key are NaN in every entry, wherever in the sequence it lies; the others are as without it."""
    parent = tree(4, 2, 4)
    c = attention_case([length], parent, 4, 2, 128, torch.bfloat16, 16, seed=13)
    clean = binding.tree_attention(**cuda(c))
    tree_paths = ref.paths(parent.tolist())
    for j in (0, 31, 33, 100, 130, length - 1, length + 7):
        if j >= length and j != length + 7 or j < 0:
            continue
        d = cuda(c)
        d["k_cache"][c["block_table"][0, j // 16].item(), j % 16] = fill
        got = binding.tree_attention(**d).out[0].cpu()
        hit = torch.tensor([j < length or j - length in p for p in tree_paths])
        assert bool(got[hit].isnan().all()) and torch.equal(got[~hit], clean.out[0].cpu()[~hit])


def test_attention_with_bad_blocks_and_bad_trees():
    parent = tree(4, 2, 4).repeat(5, 1)
    c = attention_case([100, 100, 100, 10, 33], parent, 4, 2, 128, torch.bfloat16, 16, seed=13)
    c["block_table"][0, 2] = -1
    c["block_table"][1, 6] = c["k_cache"].shape[0]                # holds nodes: rows lose themselves
    c["parent"][2, 5] = 5
    c["block_table"][3] = -1                                      # rows that see nothing
    want = ref.attention(**c)
    assert want["status"].tolist() == [5, 5, 1, 5, 0]
    got = check_attention(c, want)
    assert bool((got.out[3] == 0).all()) and bool((got.lse[3] == -math.inf).all())
    assert bool((got.out[2] == 0).all())
    c = attention_case([100], tree(4, 2, 4), 4, 2, 128, torch.bfloat16, 16, seed=14)
    c["block_table"] = c["block_table"][:, :7].contiguous()       # a table that ends before the tree does
    check_attention(c)
    c = attention_case([100], tree(4, 2, 4), 4, 2, 128, torch.bfloat16, 16, seed=14, window=20)
    c["block_table"][0, :4] = 2**31 - 1                           # blocks that no node sees any more
    assert check_attention(c).status.tolist() == [0]


def test_attention_strides():
    c = attention_case([100, 37], tree(4, 2, 4), 4, 2, 128, torch.bfloat16, 16, seed=15)
    P = c["k_cache"].shape[0]
    both = torch.randn(P, 2, 2, 16, 128).to(torch.bfloat16).cuda()                # [block, k or v, head, slot, D]
    k, v = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    k.copy_(c["k_cache"]), v.copy_(c["v_cache"])
    q = torch.zeros(19, 2, 7, 136, dtype=torch.bfloat16, device="cuda")[:, :, 2:6, :128].transpose(0, 1)
    q.copy_(c["q"])
    out = torch.full((2, 4, 19, 128), 7.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    table = torch.full((2, 50), -1, dtype=I32, device="cuda")[:, :c["block_table"].shape[1]]
    table.copy_(c["block_table"])
    check_attention(c, q=q, k_cache=k, v_cache=v, out=out, block_table=table)


def test_attention_beyond_32_bit_offsets():
    """Caches of more than 2^31 entries each: blocks at their ends."""
    blocks, block = 2**31 // (128 * 2 * 64) + 50, 64
    g = torch.Generator().manual_seed(0)
    k = torch.zeros(blocks, block, 2, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(blocks, block, 2, 128, dtype=torch.bfloat16, device="cuda")
    c = attention_case([200], tree(4, 2, 4), 4, 2, 128, torch.bfloat16, block, seed=16)
    ids = torch.tensor([blocks - 1, 3, blocks - 2, 9], dtype=I32)
    for col, i in enumerate(ids.tolist()):
        k[i], v[i] = c["k_cache"][c["block_table"][0, col]].cuda(), c["v_cache"][c["block_table"][0, col]].cuda()
    check_attention(c, k_cache=k, v_cache=v, block_table=ids[None].cuda())


def test_attention_in_a_graph_and_on_another_stream():
    c = attention_case([300, 129], tree(4, 2, 4), 8, 2, 128, torch.bfloat16, 16, seed=17)
    d = cuda(c)
    want = binding.tree_attention(**d).out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = binding.tree_attention(**d, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got.out, want)
    graphs, outs = [], []
    for _ in range(2):                                            # two graphs, replayed side by side
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(binding.tree_attention(**d).out)
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for o in outs:
            assert torch.equal(o, want)
    d["lengths"].copy_(torch.tensor([17, 250], dtype=I32))        # a replay reads the lengths as they are then
    fresh = binding.tree_attention(**d).out.clone()
    graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], fresh) and not torch.equal(fresh, want)


def test_attention_to_one_key_is_its_value():
    for length in (0, 700):
        c = attention_case([length, 0], tree(4, 2, 4), 4, 2, 128, torch.bfloat16, 16, seed=20, window=1)
        c["q"][:] = torch.randn_like(c["q"].float()).to(c["q"].dtype)
        got = binding.tree_attention(**cuda(c)).out.cpu()
        for b, n in enumerate((length, 0)):
            at = torch.arange(n, n + 19)
            v = c["v_cache"][c["block_table"][b, at // 16].long(), at % 16]
            assert torch.equal(got[b], v.repeat_interleave(2, 1))


def test_attention_is_the_same_every_time():
    for parent in (chain(1), tree(4, 2, 4), tree(8, 2, 6)):
        c = attention_case([3000, 129, 700, 1500, 2200], parent, 32, 8, 128, torch.bfloat16, 16, seed=18)
        d, want = cuda(c), ref.attention(**c)
        check_attention(c, want)
        first = binding.tree_attention(**d, want_lse=True)
        for _ in range(20):
            again = binding.tree_attention(**d, want_lse=True)
            assert torch.equal(first.out, again.out) and torch.equal(first.lse, again.lse)


# ---------------------------------------------------------------------------------------------
# verify_probs
# ---------------------------------------------------------------------------------------------
def chains_case(counts, V, dtype=torch.float32, seed=0, lookup=False, sigma=1.0, most=None):
    g = torch.Generator().manual_seed(seed)
    T, B = sum(counts), len(counts)
    cu = torch.tensor([0] + list(np.cumsum(counts)), dtype=I32)
    zq = 2 * torch.randn(T + B, V, generator=g)
    zp = zq + sigma * torch.randn(T + B, V, generator=g)
    row = torch.cat([torch.arange(int(cu[b]), int(cu[b + 1])) + b for b in range(B)] + [torch.zeros(0, dtype=torch.long)]).long()
    q = torch.softmax(zq[row], -1) if T else torch.zeros(0, V)
    token = torch.multinomial(q, 1, generator=g).flatten().int() if T else torch.zeros(0, dtype=I32)
    if lookup:
        zp[row, token.long()] += math.log(V) + 2.5
    return dict(target_probs=torch.softmax(zp, -1).to(dtype), draft_probs=None if lookup else q.to(dtype), token=token, cu_drafts=cu,
                u_accept=torch.rand(T, generator=g), u_bonus=torch.rand(T + B, generator=g), max_drafts=max(counts) if most is None else most)


def check_chains(c, **moved):
    want = ref.verify_probs(c["target_probs"], c["draft_probs"], c["token"], c["cu_drafts"], c["u_accept"], c["u_bonus"], c["max_drafts"])
    assert want["margin"] > 1e-13                                 # no decision hangs on the order of a sum in 64 bits
    got = binding.verify_probs(**dict(cuda(c), **moved))
    for name in ("status", "accept_len", "out_tokens", "bonus_token"):
        assert torch.equal(getattr(got, name).cpu(), want[name]), name
    return want


@pytest.mark.parametrize("V", [1, 2, 7, 129, 1000, 4097, 50257, 128256, 262145])
@pytest.mark.parametrize("counts", [[0], [1], [5, 0, 3, 8]])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lookup", [False, True])
def test_chains(V, counts, dtype, lookup):
    check_chains(chains_case(counts, V, dtype, seed=V + sum(counts), lookup=lookup))


def test_chains_of_many_requests_and_long_ones():
    g = torch.Generator().manual_seed(1)
    check_chains(chains_case(torch.randint(0, 6, (700,), generator=g).tolist(), 300, seed=1))
    c = chains_case([100, 33, 0, 64], 50, seed=2, sigma=0.05, most=130)
    want = check_chains(c)
    assert int(want["accept_len"].max()) > 32


def test_chains_that_end_at_borders():
    c = chains_case([4, 4, 4, 4], 300, seed=3)
    c["u_accept"][:4] = 0.0                                       # all accepted
    c["u_accept"][4:8] = 1.0 - 2**-24
    c["u_bonus"][:] = 0.0
    check_chains(c)
    c["u_bonus"][:] = 1.0 - 2**-24
    check_chains(c)
    c["target_probs"][5:7] = 0.0                                  # p = 0 at the draft; no mass in the row
    c["target_probs"][0, c["token"][0].long()] = 0.0
    c["draft_probs"][8, c["token"][8].long()] = 0.0               # q = 0 < p: accepted
    want = check_chains(c)
    assert ref.NONFINITE in want["status"].tolist()
    same = chains_case([2, 2], 64, seed=4)                        # p = q but for a draft that is refused all the same: nothing is left of p
    rows = torch.tensor([0, 1, 3, 4])
    same["target_probs"][rows] = 0.5 * same["draft_probs"]
    same["u_accept"][:] = 0.999
    check_chains(same)


def test_chains_with_bad_inputs():
    c = chains_case([3, 2, 4, 1, 2, 3], 100, seed=5, most=3)
    c["token"][0] = 100
    c["token"][4] = -1
    c["u_accept"][3] = 0.0                                        # reaches the bad token
    c["target_probs"][5 + 2 + 4 + 1, int(c["token"][9])] = float("nan")
    c["draft_probs"][12, int(c["token"][12])] = float("inf")
    want = check_chains(c)
    assert want["status"].tolist() == [2, 2, 1, 3, 0, 3]
    c = chains_case([3, 2], 100, seed=6)
    c["cu_drafts"] = torch.tensor([0, 4, 2], dtype=I32)
    c["max_drafts"] = 4
    assert check_chains(c)["status"].tolist()[1] == 1
    c["cu_drafts"] = torch.tensor([-1, 3, 900], dtype=I32)
    assert check_chains(c)["status"].tolist() == [1, 1]


def test_chains_strided_and_unaligned_rows():
    c = chains_case([3, 0, 5], 1001, seed=7)
    wide = torch.zeros(11, 1030, device="cuda")
    wide[:, 3:1004] = c["target_probs"].cuda()
    q = torch.zeros(8, 1001, device="cuda")
    q.copy_(c["draft_probs"])
    check_chains(c, target_probs=wide[:, 3:1004], draft_probs=q)


def test_chains_agree_with_the_tree_verifier():
    """A chain's probabilities and its logits give the same tokens."""
    w = synth.Workload("chain", 16, 4096, "f32", 1, 0, 5, 0.5)
    b = synth.make_batch(w, seed=3, device="cuda")
    tree_out = binding.verify_specinfer(b.target_logits, b.draft_logits, b.parent, b.token, b.u_accept, b.u_bonus)
    p = torch.softmax(b.target_logits.double(), -1).float().reshape(-1, w.V)
    q = torch.softmax(b.draft_logits[:, :-1].double(), -1).float().reshape(-1, w.V)
    got = binding.verify_probs(p, q, b.token[:, 1:].reshape(-1).contiguous(), torch.arange(0, 16 * 5 + 1, 5, dtype=I32, device="cuda"),
                               b.u_accept[:, 1:].reshape(-1).contiguous(), b.u_bonus.reshape(-1), 5)
    assert torch.equal(got.accept_len, tree_out.accept_len)
    assert torch.equal(got.out_tokens, tree_out.out_tokens)


# ---------------------------------------------------------------------------------------------
# cache_commit
# ---------------------------------------------------------------------------------------------
def commit_case(lengths, parent, accepted, caches, shape, dtype, block, seed=0, n_nodes=None):
    g = torch.Generator().manual_seed(seed)
    lengths = torch.tensor(lengths, dtype=I32)
    table, blocks = pages(lengths, parent.shape[-1], block, g)
    cache = torch.randn(caches, blocks, block, *shape, generator=g)
    cache = cache.to(dtype) if dtype.is_floating_point else (cache * 40).to(dtype)
    return dict(cache=cache, accepted_node=torch.tensor(accepted, dtype=I32), parent=parent, lengths=lengths, block_table=table,
                n_nodes=None if n_nodes is None else torch.tensor(n_nodes, dtype=I32))


def check_commit(c, **moved):
    want = ref.commit(c["cache"], c["accepted_node"], c["parent"], c["lengths"], c["block_table"], c["n_nodes"])
    d = dict(cuda(c), **moved)
    got = binding.cache_commit(**d)
    assert torch.equal(got.status.cpu(), want["status"])
    assert torch.equal(got.lengths.cpu(), want["lengths"])
    assert torch.equal(d["cache"].cpu(), want["cache"])
    return want


@pytest.mark.parametrize("caches,shape,dtype", [(1, (8,), torch.float32), (4, (2, 64), torch.bfloat16), (3, (1, 128), torch.uint8),
                                                (2, (5, 7), torch.float16), (2, (3,), torch.float32), (1, (5, 3), torch.uint8),
                                                (65, (8, 128), torch.bfloat16)])
@pytest.mark.parametrize("block", [1, 16, 24])
def test_commit(caches, shape, dtype, block):
    parent = tree(4, 2, 4)
    check_commit(commit_case([0, 5, 31, 100, 16, 17], parent, [0, 18, 6, 14, 2, 11], caches, shape, dtype, block))


def test_commit_of_random_trees_and_chains():
    g = torch.Generator().manual_seed(2)
    for n in (1, 2, 40, 300, 1024):
        parent = torch.stack([random_tree(n, g), chain(n), random_tree(n, g)])
        acc = [n - 1, n - 1, int(torch.randint(0, n, (1,), generator=g))]
        check_commit(commit_case([3, 40, 0], parent, acc, 2, (16,), torch.float32, 16, seed=n))
    deep = torch.tensor([-1, 0] + list(range(1, 200)), dtype=I32)   # a second child, then a chain: every entry moves down by one
    deep[2] = 0
    check_commit(commit_case([9], deep, [200], 2, (16,), torch.float32, 16))


def test_commit_refuses_what_it_cannot_place():
    parent = tree(4, 2, 4).repeat(8, 1)
    c = commit_case([5, -1, 20, 20, 20, 20, 20, 40], parent, [-1, 3, 19, -2, 18, 18, 18, 18], 2, (16,), torch.float32, 16,
                    n_nodes=[19, 19, 19, 19, 18, 20, 19, 19])
    c["parent"][6, 3] = 3
    c["block_table"][7, 3] = -1
    want = check_commit(c)
    assert want["status"].tolist() == [0, 0, 1, 1, 1, 1, 1, 5]


def test_commit_of_paths_in_place_without_blocks():
    # nothing of a chain moves, but what is not in the cache is not committed: a block missing, the table's end, lengths up to the largest
    c = commit_case([14, 14, 20, 20, 20, 20], chain(4).repeat(6, 1), [1, 2, 3, 3, 0, 2], 2, (16,), torch.float32, 16)
    c["block_table"][1, 1] = -1
    c["block_table"][2, 1] = c["cache"].shape[1]
    c["lengths"][3:] = torch.tensor([2**31 - 5, 2**31 - 2, 2**31 - 1], dtype=I32)
    want = check_commit(c)
    assert want["status"].tolist() == [0, 5, 5, 5, 5, 5]


def test_commit_strided_cache():
    c = commit_case([5, 31], tree(4, 2, 4), [18, 14], 4, (2, 64), torch.bfloat16, 16)
    P = c["cache"].shape[1]
    stacked = torch.zeros(P, 2, 16, 2, 3, 2, 64, dtype=torch.bfloat16, device="cuda")
    view = stacked[:, :, :, 1, 1:2].permute(1, 0, 2, 3, 4, 5)[:, :, :, 0]         # [2, P, 16, 2, 64], rows far apart
    small = dict(c, cache=c["cache"][:2].contiguous())
    view.copy_(small["cache"])
    check_commit(small, cache=view)


def test_arguments_out_of_range_are_refused():
    d = cuda(attention_case([10], tree(1, 0, 1), 2, 1, 64, torch.bfloat16, 16))
    for kw in (dict(window=2**32), dict(sinks=2**31), dict(window=-1), dict(scale=-1.0)):
        with pytest.raises(RuntimeError):
            binding.tree_attention(**d, **kw)
    with pytest.raises(TypeError):
        binding.tree_attention(**d, window=1.5)
    with pytest.raises(RuntimeError, match="backward"):
        binding.tree_attention(**dict(d, q=d["q"].requires_grad_()))
    r = cuda(rope_case(3, 2, 1, 64, 64, torch.bfloat16))
    m = cuda(commit_case([5], tree(1, 0, 1), [1], 2, (16,), torch.float32, 16))
    for call, args, name in ((binding.norm_rope_cache, r, "k_cache"), (binding.norm_rope_cache, r, "v_cache"), (binding.cache_commit, m, "cache")):
        with pytest.raises(RuntimeError, match="backward"):
            call(**dict(args, **{name: args[name].clone().requires_grad_()}))
    for name in ("k_cache", "v_cache", "q"):
        with pytest.raises(RuntimeError):
            binding.tree_attention(**dict(cuda(attention_case([10], tree(1, 0, 1), 2, 1, 64, torch.bfloat16, 16)), **{name: d[name].detach().half()}))


# ---------------------------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------------------------
def test_steps_of_a_decoding_loop():
    """Slots, keys and values into the cache, attention, a verifier, commit, over several steps: the cache's committed entries and the
    attention over them are those of a program that keeps every request's tokens in a list."""
    g = torch.Generator().manual_seed(0)
    B, Hq, Hkv, D, block, V, layers = 5, 4, 2, 64, 8, 500, 2
    parent = tree(3, 1, 3)
    N, P = len(parent), 80
    cache = torch.randn(2 * layers, P, block, Hkv, D, generator=g).to(torch.bfloat16).cuda()
    table = torch.full((B, 16), -1, dtype=I32, device="cuda")
    lengths, owned = torch.zeros(B, dtype=I32, device="cuda"), torch.zeros(B, dtype=I32, device="cuda")
    ring, free = torch.randperm(P, generator=g).int().cuda(), torch.tensor([0, P], dtype=I32, device="cuda")
    inv_freq = (10000.0 ** (-torch.arange(0, D, 2).double() / D)).float().cuda()
    kept = [[[] for _ in range(B)] for _ in range(layers)]        # (key, value) of every committed token
    parent_d = parent.cuda()
    for step in range(6):
        s = binding.cache_slots(lengths, parent_d, table, owned, ring, free, block)
        owned, free = s.owned, s.free_range
        w = synth.Workload("loop", B, V, "f32", 3, 1, 3, 0.4)
        batch = synth.make_batch(w, seed=step, device="cuda")
        rows = []
        for layer in range(layers):
            qkv = torch.randn(B * N, Hq + 2 * Hkv, D, generator=g).to(torch.bfloat16).cuda()
            q = binding.norm_rope_cache(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], inv_freq, s.positions, s.slots,
                                        cache[2 * layer], cache[2 * layer + 1])
            at = s.slots.long()
            k, v = (cache[2 * layer + i].flatten(0, 1)[at].cpu() for i in (0, 1))
            rows.append((k, v))
            got = binding.tree_attention(q.view(B, N, Hq, D), cache[2 * layer], cache[2 * layer + 1], table, lengths, parent_d)
            assert got.status.tolist() == [0] * B
            for b in range(B):
                old = kept[layer][b]
                own = attention_lists(old, k[b], v[b])
                c = dict(q=q.view(B, N, Hq, D)[b:b + 1].cpu(), k_cache=own[0], v_cache=own[1], parent=parent,
                         block_table=torch.zeros(1, 1, dtype=I32), lengths=torch.tensor([len(old)], dtype=I32))
                want = ref.attention(**c)
                bound = want["mass"] * (2.0**-8 + 2.0**-10) + want["out"].abs() * 2.0**-8
                assert bool(((got.out[b:b + 1].cpu().double() - want["out"]).abs() <= bound).all())
        verified = binding.verify_specinfer(batch.target_logits, batch.draft_logits, parent_d, batch.token, batch.u_accept, batch.u_bonus)
        done = binding.cache_commit(cache, verified.accepted_node, parent_d, lengths, table)
        tree_paths = ref.paths(parent.tolist())
        for b, node in enumerate(verified.accepted_node.tolist()):
            for layer in range(layers):
                for i in tree_paths[node]:
                    kept[layer][b].append((rows[layer][0][b, i], rows[layer][1][b, i]))
        lengths = done.lengths
        assert lengths.tolist() == [len(x) for x in kept[0]]
        for layer in range(layers):
            for b in range(B):
                for j, (k, v) in enumerate(kept[layer][b]):
                    i = int(table[b, j // block])
                    assert torch.equal(cache[2 * layer, i, j % block].cpu(), k) and torch.equal(cache[2 * layer + 1, i, j % block].cpu(), v)
    assert int(lengths.sum()) > 6 * B


def test_tree_cache():
    """The same steps through the class that keeps the state; a request ends and its blocks go to another."""
    g = torch.Generator().manual_seed(1)
    B, N, blocks, block = 3, 10, 12, 8
    cache = TreeCache(B, 1, blocks, block, 2, 64, width=8)
    parent = tree(3, 0, 3).cuda()
    lengths, held = [0] * B, {}
    for step in range(4):
        if step == 3:
            cache.release(1)
            assert int(cache.free_range[1]) + int(cache.owned.sum()) == blocks
        s = cache.begin(parent)
        assert s.status.tolist() == [0] * B
        used = [x for row in cache.block_table.tolist() for x in row if x >= 0]
        assert len(set(used)) == len(used)
        qkv = torch.randn(B * N, 8, 64, generator=g).to(torch.bfloat16).cuda()
        q = cache.write(0, qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], torch.ones(32, device="cuda") * 0.01)
        out = cache.attend(0, q.view(B, N, 4, 64), window=30, sinks=2)
        assert out.status.tolist() == [0] * B
        want = ref.attention(q.view(B, N, 4, 64).cpu(), cache.storage[0].cpu(), cache.storage[1].cpu(), cache.block_table.cpu(),
                             cache.lengths.cpu(), parent.cpu(), window=30, sinks=2)
        bound = want["mass"] * (2.0**-8 + 2.0**-10) + want["out"].abs() * 2.0**-8
        live = want["live"]
        assert bool(((out.out.cpu().double() - want["out"]).abs() <= bound)[live].all())
        accepted = torch.tensor([9, 4, 0], dtype=I32, device="cuda")
        done = cache.commit(accepted)
        lengths = [n + d if n >= 0 else n for n, d in zip(lengths, (4, 2, 1))]
        if step == 3:
            lengths[1] = -1
        assert done.lengths.tolist() == lengths


def attention_lists(old, k, v):
    """One block that holds a request's committed entries and its tree's."""
    return (torch.stack([x for x, _ in old] + list(k))[None], torch.stack([y for _, y in old] + list(v))[None])
