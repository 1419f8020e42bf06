"""Log probabilities and eviction against their restatements in 64 bits, at sizes, masks and layouts where they can go wrong."""
import math

import pytest
import torch

from . import serve_ref as ref
from paper_2602_16994_b200 import binding

pytestmark = pytest.mark.gpu

I32 = torch.int32
INF = math.inf


# ---------------------------------------------------------------------------------------------
# log probabilities
# ---------------------------------------------------------------------------------------------
def tolerance(V):
    """Of log S: an exponential is off by 2^-22, its argument by three roundings of up to log2 V on average, a thread adds up V / 512 of them,
    and four scalings by 2^-22 put the parts together."""
    return (V / 512 + 3 * math.log2(max(2, V)) + 24) * 2.0**-24


def check_rows(got, want, V, temperature, top, shape=None):
    eps = tolerance(V)
    assert torch.equal(got.status.cpu().view(-1), want["status"].view(-1))

    def near(x, y, slack):
        x, y = x.cpu().double().reshape(-1), y.reshape(-1)
        assert torch.equal(x.isnan(), y.isnan())
        fine = y.isfinite()
        assert torch.equal(x[~fine & ~y.isnan()], y[~fine & ~y.isnan()])
        bound = slack + y[fine].abs() * 2.0**-23
        assert bool(((x[fine] - y[fine]).abs() <= bound).all()), float(((x[fine] - y[fine]).abs() - bound).max())

    near(got.logprob, want["logprob"], eps)
    near(got.entropy, want["entropy"], eps * (1 + 2 * math.log(max(2, V))))
    if top:
        assert torch.equal(got.top_tokens.cpu().reshape(-1), want["top_tokens"].reshape(-1))
        near(got.top_logprobs, want["top_logprobs"], eps)
    else:
        assert got.top_tokens is None and got.top_logprobs is None


def check_logprobs(logits, tokens, temperature=1.0, top=0):
    want = ref.logprobs(logits.reshape(-1, logits.shape[-1]).cpu(), tokens.reshape(logits.shape[:-1].numel(), tokens.shape[-1]).cpu(), temperature, top)
    got = binding.token_logprobs(logits.cuda(), tokens.cuda(), temperature=temperature, top=top)
    assert got.logprob.shape == tokens.shape and got.entropy.shape == logits.shape[:-1]
    check_rows(got, want, logits.shape[-1], temperature, top)
    return got


def rows(R, V, K, dtype, seed, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(R, V, generator=g)).to(dtype), torch.randint(0, V, (R, K), generator=g).int()


@pytest.mark.parametrize("R,V,K,top", [(1, 1, 1, 1), (1, 7, 2, 7), (3, 33, 1, 5), (2, 1000, 4, 32), (1, 50257, 1, 20), (5, 4096, 0, 3),
                                       (1, 128256, 1, 5), (2, 262144, 3, 32), (40, 8200, 1, 20), (700, 1025, 1, 1), (150, 20001, 2, 0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_logprobs(R, V, K, top, dtype):
    check_logprobs(*rows(R, V, K, dtype, R + V), top=top)


@pytest.mark.parametrize("temperature", [1e-12, 1e-3, 0.3, 2.0, 1e4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logprobs_at_temperatures(temperature, dtype):
    z, t = rows(3, 30011, 2, dtype, 5)
    check_logprobs(z, t, temperature, 8)


@pytest.mark.parametrize("offset", [-60000.0, -300.0, 1000.0, 60000.0])
def test_logprobs_far_from_zero(offset):
    z, t = rows(2, 9000, 2, torch.float32, 6)
    check_logprobs(z + offset, t, 1.0, 4)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("R", [1, 300])
@pytest.mark.parametrize("value", ["-inf", "lowest"])
@pytest.mark.parametrize("left", [1, 3, 40, 700])
def test_logprobs_under_masks(dtype, R, value, left):
    """All but a few logits masked: the alternatives beyond them are the lowest masked indices, with a log probability of -inf (or of next to it)."""
    V = 20001
    z, t = rows(R, V, 2, dtype, left)
    g = torch.Generator().manual_seed(left)
    stay = torch.randperm(V, generator=g)[:left]
    mask = torch.ones(V, dtype=torch.bool)
    mask[stay] = False
    z[:, mask] = -INF if value == "-inf" else torch.finfo(dtype).min
    t[:, 0] = stay[0]
    check_logprobs(z, t, 1.0, 20)


@pytest.mark.parametrize("R", [1, 2, 400])
def test_logprobs_of_ties(R):
    V = 20001
    z = torch.zeros(R, V)
    z[:, 10000:10100] = 1.0
    z[-1] = 2.5                                                  # one value for all
    z[0, 5::256 * 8] = 2.0
    z[0, 1] = -0.0
    check_logprobs(z, torch.tensor([[7, 10050]], dtype=I32).repeat(R, 1), 1.0, 32)


@pytest.mark.parametrize("V", [20000, 151936])
@pytest.mark.parametrize("order", ["rising", "falling", "heaped"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logprobs_of_rows_made_for_the_search(V, order, dtype):
    """Sorted rows, and one whose largest entries by the hundred belong to a few threads."""
    z = torch.linspace(-20, 20, V)
    if order == "falling":
        z = z.flip(0)
    if order == "heaped":
        e = 4 if dtype == torch.float32 else 8
        z = torch.randn(V, generator=torch.Generator().manual_seed(1))
        owner = torch.arange(V) // e % 256
        z[owner < 3] += 30.0
    check_logprobs(torch.stack([z, z.roll(3)]).repeat(200, 1).to(dtype), torch.zeros(400, 1, dtype=I32), 1.0, 20)


@pytest.mark.parametrize("value,dtype", [(0.1, torch.float32), (-0.1, torch.float32), (-1.0, torch.bfloat16), (-2.5, torch.float16), (1.0009765625, torch.float16)])
@pytest.mark.parametrize("R,V", [(1, 128256), (300, 9001)])
def test_logprobs_of_rows_of_one_value(value, dtype, R, V):
    """More entries at the search's bound than there is room for, which the bound's bits do or do not name: the lowest indices, all of the same probability."""
    z, t = torch.full((R, V), value, dtype=dtype), torch.full((R, 1), V - 1, dtype=I32)
    z[-1, V // 2] += 0.5
    check_logprobs(z, t, 1.0, 20)


def entropy_case(near, D):
    """A logit alone in a thread's first batch, one `near` above it in a later batch of the same thread, all others far below."""
    batch = 4 * 256 * (128 // torch.finfo(D).bits)               # entries of a batch of all threads; its first chunk is the first thread's
    z = torch.full((2, 4 * batch), -1000.0)                      # (a row of four batches goes to one CTA)
    z[0, 0], z[0, 2 * batch] = 3.0, 3.0 + near
    z[1, 0], z[1, 2 * batch], z[1, 3 * batch] = 3.0 + near, 3.0, 3.0 + near
    return z.to(D)


@pytest.mark.parametrize("near", [0.125, 2.0, 4.0, 5.5, 6.0, 20.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logprobs_of_little_entropy(near, dtype):
    """The sums are taken about a logit below the largest, by up to 8 powers of two, and moved at the end: the entropy is off by what that costs, about 8 ln 2
    times a rounding for each of the two terms, and never below 0; no log probability lies above it."""
    z = entropy_case(near, dtype)
    got = binding.token_logprobs(z.cuda(), z.argmax(-1).int().cuda(), top=2)
    want = ref.logprobs(z, z.argmax(-1).int()[:, None], 1.0, 2)
    # S and U are off by 2^-22 (an exponential, and one that moves them) and 2^-24 a term (three, added up twice); U's terms are up to 8 ln 2 of S, log S and
    # U / S each bring that to the entropy
    off = (got.entropy.cpu().double() - want["entropy"]).abs()
    assert bool((off <= (1 + 8 * math.log(2)) * 2 * (2 * 2.0**-22 + 6 * 2.0**-24)).all()), off.tolist()
    assert bool((got.entropy >= 0).all()) and bool((got.logprob <= 0).all()) and bool((got.top_logprobs <= 0).all())
    check_rows(got, want, z.shape[1], 1.0, 2)


def test_logprobs_of_bad_rows_and_tokens():
    z, t = rows(9, 5000, 3, torch.float32, 8)
    z[0, 17], z[1, 4999], z[2, 0] = math.nan, INF, -INF
    z[3] = -INF
    z[4, 1:] = -INF
    t[4, 0], t[5, 1], t[6, 0], t[7, 2], t[0, 1] = 0, -1, 5000, -2, -1
    got = check_logprobs(z, t, 1.0, 3)
    assert got.status.tolist() == [3, 3, 0, 3, 0, 0, 2, 2, 0]
    assert float(got.logprob[4, 0]) == 0.0 and float(got.entropy[4]) == 0.0
    assert float(got.logprob[5, 1]) == 0.0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logprobs_of_rows_that_lie_anywhere(dtype):
    wide = torch.randn(6, 5, 3011, generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    t = torch.randint(0, 3000, (6, 5, 2), generator=torch.Generator().manual_seed(3)).int()
    for z in (wide[..., 3:3003], wide[::2, 1:4, 1:3001], wide.transpose(0, 1)[..., :2999], wide[:1, :1].expand(6, 5, -1)):
        check_logprobs(z, t[:z.shape[0], :z.shape[1]].contiguous() if z.shape[0] <= 6 and z.shape[1] <= 5 else t.transpose(0, 1).contiguous(), 1.0, 4)
    one = binding.token_logprobs(wide[:, 0], t[:, 0, 0].contiguous().cuda())
    assert one.logprob.shape == (6,)
    assert binding.token_logprobs(wide[:0, 0], t[:0, 0, 0].cuda(), top=2).top_tokens.shape == (0, 2)


def path_case(B, N, V, seed, per_request=False):
    g = torch.Generator().manual_seed(seed)
    z = (3 * torch.randn(B, N, V, generator=g)).bfloat16()
    trees = torch.stack([torch.tensor([-1] + [int(torch.randint(0, i, (1,), generator=g)) for i in range(1, N)], dtype=I32) for _ in range(B)])
    accepted = torch.randint(-1, N, (B,), generator=g).int()
    tokens = torch.randint(0, V, (B, N), generator=g).int()
    return z, accepted, tokens, trees if per_request else trees[0]


def check_path(z, accepted, tokens, parent, temperature=1.0, top=0):
    want = ref.path_logprobs(z, accepted, tokens, parent, temperature, top)
    got = binding.path_logprobs(z.cuda(), accepted.cuda(), tokens.cuda(), parent.cuda(), temperature=temperature, top=top)
    check_rows(got, want, z.shape[-1], temperature, top)
    return got


@pytest.mark.parametrize("B,N,V,per_request", [(1, 1, 100, False), (8, 19, 12000, False), (20, 9, 3001, True), (3, 200, 1000, True)])
@pytest.mark.parametrize("top", [0, 5])
def test_path_logprobs(B, N, V, per_request, top):
    check_path(*path_case(B, N, V, B + N, per_request), 0.7, top)


def test_path_logprobs_of_bad_trees():
    z, accepted, tokens, parent = path_case(7, 6, 500, 4, True)
    accepted[:] = torch.tensor([5, 6, -2, -1, 5, 0, 3])
    parent[0] = torch.tensor([-1, 0, 1, 2, 4, 4])                # its own parent
    parent[4] = torch.tensor([0, 0, 1, 2, 3, 4])                 # a root with a parent
    parent[6] = torch.tensor([-1, 0, 1, 2, 9, 9])                # bad beside the path
    got = check_path(z, accepted, tokens, parent, 1.0, 3)
    assert got.status[:, 0].tolist() == [1, 1, 1, 0, 1, 0, 0]


def test_path_logprobs_after_a_verification():
    from paper_2602_16994_b200 import synth
    batch = synth.make_batch(synth.Workload("logprobs", 4, 5000, "bf16", 3, 1, 2, 0.5), seed=2, device="cuda")
    v = binding.verify_specinfer(batch.target_logits, batch.draft_logits, batch.parent, batch.token, batch.u_accept, batch.u_bonus, 0.8)
    got = binding.path_logprobs(batch.target_logits, v.accepted_node, v.out_tokens, batch.parent, temperature=0.8, top=2)
    want = ref.path_logprobs(batch.target_logits.cpu(), v.accepted_node.cpu(), v.out_tokens.cpu(), batch.parent.cpu(), 0.8, 2)
    check_rows(got, want, 5000, 0.8, 2)
    assert bool((got.status == 0).all()) and bool((got.logprob[v.out_tokens >= 0] < 0).all())


# ---------------------------------------------------------------------------------------------
# eviction
# ---------------------------------------------------------------------------------------------
def evict_case(B, L, block, caches, row, dtype=torch.bfloat16, seed=0, spare=3, ties=False, protected=None):
    g = torch.Generator().manual_seed(seed)
    lengths = torch.randint(0, L + 1, (B,), generator=g).int()
    lengths[0] = L
    owned = (lengths + block - 1) // block + torch.randint(0, 3, (B,), generator=g).int()
    width = int(owned.max()) + 1
    total = int(owned.sum()) + spare
    ids = torch.randperm(total, generator=g).int()
    table, at = torch.full((B, width), -1, dtype=I32), 0
    for b in range(B):
        table[b, :owned[b]] = ids[at:at + int(owned[b])]
        at += int(owned[b])
    ring = torch.full((total,), -7, dtype=I32)
    begin = int(torch.randint(0, total, (1,), generator=g))
    ring[(begin + torch.arange(spare)) % total] = ids[at:]
    cache = torch.randn(caches, total, block, *row, generator=g).to(dtype)
    weights = torch.rand(total, block, generator=g)
    if ties:
        weights = (weights * 4).floor()
    return dict(cache=cache, weights=weights, lengths=lengths, block_table=table, owned=owned.int(), free_blocks=ring,
                free_range=torch.tensor([begin, spare], dtype=I32), protected=protected)


def check_evict(c, budget, recent=0):
    want, _ = ref.evict(c["cache"], c["weights"], c["lengths"], c["block_table"], c["owned"], c["free_blocks"], c["free_range"], budget,
                        recent, c["protected"])
    d = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    got = binding.cache_evict(d["cache"], d["weights"], d["lengths"], d["block_table"], d["owned"], d["free_blocks"], d["free_range"], budget,
                              recent=recent, protected=d["protected"])
    for name in ("status", "lengths", "owned", "free_range"):
        assert torch.equal(getattr(got, name).cpu(), want[name]), name
    assert torch.equal(d["free_blocks"].cpu(), want["free_blocks"])
    assert torch.equal(d["weights"].cpu().view(I32), want["weights"].view(I32))
    assert torch.equal(d["cache"].cpu(), want["cache"])
    for name in ("lengths", "owned", "free_range", "block_table"):
        assert torch.equal(d[name].cpu(), c[name]), name
    return want


@pytest.mark.parametrize("B,L,block,caches,row,budget,recent", [
    (1, 2, 1, 1, (1,), 1, 0), (1, 100, 16, 2, (2, 64), 33, 7), (5, 300, 16, 4, (2, 64), 128, 32), (3, 3000, 7, 2, (40,), 1024, 100),
    (9, 257, 64, 3, (8, 128), 100, 200), (2, 5000, 32, 2, (1, 64), 4999, 0), (2, 20000, 16, 1, (4,), 9000, 500), (300, 60, 8, 1, (8,), 20, 5),
    (4, 400, 16, 2, (3, 33), 150, 0)])
@pytest.mark.parametrize("ties", [False, True])
def test_evict(B, L, block, caches, row, budget, recent, ties):
    check_evict(evict_case(B, L, block, caches, row, seed=B + L, ties=ties), budget, recent)


@pytest.mark.parametrize("block,L,budget,recent,protected", [(8, 60000, 30000, 100, None), (1, 5000, 4990, 0, [4500, 10]), (4, 52000, 51990, 3, [0, 4000]),
                                                             (16, 66000, 500, 0, [20, 0])])
@pytest.mark.parametrize("ties", [False, True])
def test_evict_beyond_what_is_on_chip(block, L, budget, recent, protected, ties):
    """Rows of the table of more than 4096 columns, requests of more than 47104 entries behind the protected ones: what lies beyond is read from memory, the
    weights while those of earlier entries are written."""
    c = evict_case(2, L, block, 2, (4,), seed=L, ties=ties, protected=None if protected is None else torch.tensor(protected, dtype=I32))
    c["lengths"][1] = L - 1                                      # (the second as long: its blocks behind those of the first)
    c["owned"][1] = (L - 1 + block - 1) // block
    total = int(c["owned"].sum()) + 3
    ids = torch.randperm(total, generator=torch.Generator().manual_seed(L)).int()
    c["block_table"] = torch.full((2, int(c["owned"].max()) + 1), -1, dtype=I32)
    c["block_table"][0, :c["owned"][0]] = ids[:int(c["owned"][0])]
    c["block_table"][1, :c["owned"][1]] = ids[int(c["owned"][0]):-3]
    g = torch.Generator().manual_seed(L + 1)
    c["cache"] = torch.randn(2, total, block, 4, generator=g).bfloat16()
    c["weights"] = torch.rand(total, block, generator=g)
    if ties:
        c["weights"] = (c["weights"] * 4).floor()
    c["free_blocks"], c["free_range"] = torch.full((total,), -7, dtype=I32), torch.tensor([total - 2, 3], dtype=I32)
    want = check_evict(c, budget, recent)
    assert want["status"].tolist() == [0, 0]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.uint8])
def test_evict_of_types_and_protected(dtype):
    protected = torch.tensor([0, 4, 64, 100], dtype=I32)
    c = evict_case(4, 500, 16, 3, (2, 40), torch.float32, 3, protected=protected)
    c["cache"] = (100 * c["cache"]).abs().to(dtype)
    check_evict(c, 100, 50)


def test_evict_of_odd_weights():
    """NaN below everything, infinities, zeros of both signs, negative numbers."""
    c = evict_case(3, 600, 16, 1, (8,), seed=4)
    w = c["weights"].view(-1)
    pick = torch.randint(0, 7, w.shape, generator=torch.Generator().manual_seed(5))
    for i, x in enumerate((math.nan, INF, -INF, 0.0, -0.0, -1.0)):
        w[pick == i] = x
    for budget in (50, 200, 400, 590):
        check_evict(c, budget, 3)


def test_evict_refuses_requests_and_leaves_them():
    protected = torch.tensor([0, 101, -1, 0, 0, 0, 0, 100], dtype=I32)
    c = evict_case(8, 400, 16, 2, (8,), seed=6, protected=protected)
    c["lengths"][:] = torch.tensor([400, 300, 300, 300, 300, 300, -5, 300])
    need = (c["lengths"].clamp(min=0) + 15) // 16
    total = int(need.sum()) + 9
    ids, at = torch.randperm(total).int(), 0
    c["block_table"] = torch.full((8, 30), -1, dtype=I32)
    for b in range(8):
        c["block_table"][b, :need[b]] = ids[at:at + int(need[b])]
        at += int(need[b])
    c["owned"] = need.int()
    c["cache"], c["weights"] = torch.randn(2, total, 16, 8).bfloat16(), torch.rand(total, 16)
    c["free_blocks"], c["free_range"] = torch.full((200,), -3, dtype=I32), torch.tensor([195, 3], dtype=I32)
    c["owned"][3] = 18                                           # one block too few
    c["owned"][4] = 31                                           # beyond the row
    c["block_table"][5, 2] = total
    want = check_evict(c, 100, 10)
    assert want["status"].tolist() == [0, 1, 1, 5, 5, 5, 0, 0]


@pytest.mark.parametrize("size,count", [(0, 0), (10, 10), (20, 3), (45, 0), (10, 11)])
def test_evict_into_a_ring_without_room(size, count):
    c = evict_case(6, 400, 16, 1, (8,), seed=7)
    c["free_blocks"], c["free_range"] = torch.full((size,), -3, dtype=I32), torch.tensor([size // 2, count], dtype=I32)
    want = check_evict(c, 100, 10)
    assert (want["status"] == ref.BLOCKS).any()


def test_evict_again_and_in_views():
    """A second eviction follows the first; caches and tables that are views."""
    c = evict_case(4, 500, 16, 3, (2, 64), seed=8)
    wide = torch.zeros(6, c["cache"].shape[1], 16, 2, 64, dtype=torch.bfloat16)
    wide[1:4] = c["cache"]
    host = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    dev = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    stack, table = wide.cuda(), torch.full((8, c["block_table"].shape[1] + 5), -9, dtype=I32, device="cuda")
    table[::2, :c["block_table"].shape[1]] = dev["block_table"]
    view = table[::2, :c["block_table"].shape[1]]
    for budget in (300, 120, 1):
        want, _ = ref.evict(host["cache"], host["weights"], host["lengths"], host["block_table"], host["owned"], host["free_blocks"],
                            host["free_range"], budget, 20)
        got = binding.cache_evict(stack[1:4], dev["weights"], dev["lengths"], view, dev["owned"], dev["free_blocks"], dev["free_range"],
                                  budget, recent=20)
        assert torch.equal(stack[1:4].cpu(), want["cache"]) and torch.equal(dev["weights"].cpu(), want["weights"])
        assert torch.equal(got.free_range.cpu(), want["free_range"]) and torch.equal(dev["free_blocks"].cpu(), want["free_blocks"])
        host.update(want)
        dev.update(lengths=got.lengths, owned=got.owned, free_range=got.free_range)
    assert bool((stack[0] == 0).all()) and bool((stack[4:] == 0).all())


# ---------------------------------------------------------------------------------------------
# streams, graphs, refusals
# ---------------------------------------------------------------------------------------------
def test_calls_on_another_stream_and_in_a_graph():
    z, t = rows(4, 30000, 1, torch.bfloat16, 9)
    z, t = z.cuda(), t.cuda()
    c = evict_case(4, 500, 16, 3, (2, 64), seed=9)
    d = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    base, base_w, base_r = d["cache"].clone(), d["weights"].clone(), d["free_blocks"].clone()

    def evict(stream=None):
        return binding.cache_evict(d["cache"], d["weights"], d["lengths"], d["block_table"], d["owned"], d["free_blocks"], d["free_range"], 100,
                                   recent=10, stream=stream)

    def again():
        d["cache"].copy_(base)
        d["weights"].copy_(base_w)
        d["free_blocks"].copy_(base_r)

    want = binding.token_logprobs(z, t, top=5)
    e = evict()
    moved = d["cache"].clone()
    side = torch.cuda.Stream()
    again()
    side.wait_stream(torch.cuda.current_stream())
    got, e2 = binding.token_logprobs(z, t, top=5, stream=side), evict(side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got.logprob, want.logprob) and torch.equal(got.top_tokens, want.top_tokens)
    assert torch.equal(d["cache"], moved) and torch.equal(e2.owned, e.owned)
    again()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, e2 = binding.token_logprobs(z, t, top=5), evict()
    for _ in range(3):
        again()
        z.add_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got.top_logprobs, want.top_logprobs) and torch.equal(d["cache"], moved) and torch.equal(e2.lengths, e.lengths)


def test_refusals():
    z, t = rows(4, 300, 1, torch.float32, 9)
    z, t = z.cuda(), t.cuda()
    with pytest.raises(RuntimeError, match="gradient"):
        binding.token_logprobs(z.clone().requires_grad_(), t)
    for bad in (dict(temperature=0.0), dict(temperature=math.nan), dict(top=33), dict(top=-1), dict(temperature=1e31)):
        with pytest.raises(RuntimeError, match="PARAM"):
            binding.token_logprobs(z, t, **bad)
    with pytest.raises(RuntimeError, match="PARAM"):
        binding.token_logprobs(z[:, :3], t, top=4)
    for x, y in ((z.double(), t), (z, t.long()), (z, t[:3]), (z.t(), t), (z[0], t[0])):
        with pytest.raises(RuntimeError):
            binding.token_logprobs(x, y)
    c = evict_case(2, 50, 16, 1, (8,), seed=9)
    d = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}

    def call(budget=10, recent=0, **kw):
        e = dict(d, **kw)
        return binding.cache_evict(e["cache"], e["weights"], e["lengths"], e["block_table"], e["owned"], e["free_blocks"], e["free_range"], budget,
                                   recent=recent)

    for bad in (dict(budget=0), dict(recent=-1)):
        with pytest.raises(RuntimeError, match="PARAM"):
            call(**bad)
    for bad in (dict(cache=d["cache"].expand(3, -1, -1, -1)), dict(weights=d["weights"].double()), dict(weights=d["weights"][:-1]),
                dict(weights=d["weights"].clone().requires_grad_()), dict(owned=d["owned"][:1]), dict(free_range=d["free_range"][:1]),
                dict(cache=d["cache"][..., ::2])):
        with pytest.raises(RuntimeError):
            call(**bad)
