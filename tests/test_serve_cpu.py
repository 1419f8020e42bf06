"""Host-side checks of log probabilities and of the calls on a bounded cache: what they refuse, before a device is touched."""
import ctypes as C

import pytest
import torch

from paper_2602_16994_b200 import binding
from .test_step_cpu import Attention, F, I, L, P, S3, filled, good_attention, lib, struct  # noqa: F401

Logprobs = struct("SpecLogprobs", (I, "B N V K top dtype"), (P, "logits"), (L, "seq_stride node_stride"), (P, "parent"), (L, "topo_seq_stride"),
                  (P, "accepted_node token"), (F, "temperature"), (P, "logprob entropy top_tokens top_logprobs status"))
Evict = struct("SpecEvict", (I, "B caches budget recent num_blocks block_size table_width"), (P, "cache"), (S3, "stride"), (L, "row_bytes"),
               (P, "weights block_table"), (L, "table_stride"), (P, "lengths owned protected_len free_blocks"), (I, "free_size"),
               (P, "free_range lengths_out owned_out free_range_out status"))

Weights = struct("SpecWeights", (I, "B N Hq Hkv D dtype num_blocks block_size table_width fresh"), (F, "scale"), (P, "q"), (S3, "q_stride"),
                 (P, "k_cache"), (S3, "k_cache_stride"), (P, "lse block_table"), (L, "table_stride"), (P, "lengths n_nodes parent"),
                 (L, "topo_seq_stride"), (P, "protected_len weights status"))

class Prefix(C.Structure):
    _fields_ = [("attention", Attention)] + [(f, I) for f in ("n_groups", "n_members", "prefix_width")] + [
        (f, P) for f in ("group", "members", "first", "place", "shared_blocks", "prefix_table")] + [("prefix_stride", L)]


def prefix(**kw):
    own = {k: kw.pop(k) for k in list(kw) if k in dict(Prefix._fields_)}
    s = Prefix()
    s.attention = good_attention(**dict(dict(window=0, sinks=0), **kw))
    for n, (f, t) in enumerate(Prefix._fields_[1:]):
        setattr(s, f, own.get(f, 0x900000 + 0x1000 * n if t is P else 1))
    return s


def test_prefix_refusals(lib):  # noqa: F811
    n = L()
    size = lambda **kw: lib.spec_prefix_attention_workspace_bytes(C.byref(prefix(**kw)), C.byref(n))  # noqa: E731
    assert size() == 0 and n.value >= 256
    assert lib.spec_prefix_attention_workspace_bytes(None, C.byref(n)) == -1
    assert lib.spec_prefix_attention_workspace_bytes(C.byref(prefix()), None) == -1
    for f in ("q", "k_cache", "v_cache", "block_table", "lengths", "parent", "out", "status", "group", "members", "first", "place", "shared_blocks",
              "prefix_table"):
        assert size(**{f: None}) == -1, f
    assert size(n_groups=0, members=None, first=None, place=None, shared_blocks=None, prefix_table=None, n_members=0) == 0
    for kw in (dict(B=0), dict(N=0), dict(N=1025), dict(Hkv=0), dict(Hq=7), dict(num_blocks=0), dict(block_size=0), dict(table_width=0),
               dict(topo_seq_stride=18), dict(n_groups=-1), dict(n_groups=65536), dict(n_members=-1), dict(n_members=3), dict(n_members=0),
               dict(prefix_width=0), dict(prefix_width=2)):
        assert size(**kw) == -2, kw
    for dtype in (-1, 0, 3):
        assert size(dtype=dtype) == -3
    for kw in (dict(scale=float("nan")), dict(scale=-0.5), dict(window=1), dict(sinks=1)):
        assert size(**kw) == -4, kw
    for kw in (dict(D=96), dict(q=0x10008), dict(out=0x10004), dict(k_cache_stride=(8, 8, 12)),
               dict(B=4096, N=1024, Hq=512, n_members=4096), dict(prefix_width=1 << 30, prefix_stride=1 << 30, n_groups=60000, n_members=2, block_size=2)):
        assert size(**kw) == -6, kw
    call = lambda ws, b: lib.spec_prefix_attention(C.byref(prefix()), P(ws), L(b), None)  # noqa: E731
    size()
    assert call(None, 1 << 30) == -5 and call(0x10010, 1 << 30) == -5 and call(0x10000, n.value - 1) == -5


def test_prefix_rows_take_two_blocks_beyond_one(lib):  # noqa: F811
    """The form of the kernel goes by the rows that a prefix has on average: scratch for the CTAs' parts tells which it is."""
    def bytes_of(members, groups, N=1, D=128):
        n, s = L(), prefix(B=512, N=N, Hq=8, Hkv=2, D=D, n_members=members, n_groups=groups, topo_seq_stride=0)
        assert lib.spec_prefix_attention_workspace_bytes(C.byref(s), C.byref(n)) == 0
        each = 512 + members                                     # (rows that are not cut, and records of units, for every request and member)
        return n.value - each * 8 * N * (D * 4 + 8)
    block = 148 * 2 * 128 * (128 * 4 + 8)
    for members, groups, N, blocks in ((32, 1, 1, 1), (33, 1, 1, 2), (64, 1, 1, 2), (128, 4, 1, 1), (129, 4, 1, 2), (1, 1, 19, 1), (2, 1, 19, 2), (16, 8, 19, 2),
                                       (2, 2, 19, 1), (1, 1, 33, 2)):
        assert abs(bytes_of(members, groups, N) - blocks * block) < block // 2, (members, groups, N)


def test_prefix_plan():
    """Members in the order of groups, places among them, requests of no group in none."""
    group = torch.tensor([2, 0, -1, 2, 0, 5, 2], dtype=torch.int32)
    p = binding.prefix_plan(group, torch.tensor([3, 1, 2], dtype=torch.int32), torch.zeros(3, 4, dtype=torch.int32))
    assert p.members.tolist() == [2, 1, 4, 0, 3, 6, 5] and p.first.tolist() == [1, 3, 3, 6]
    for b, g in enumerate(group.tolist()):
        if 0 <= g < 3:
            assert p.members[p.first[g] + p.place[b]] == b
    none = binding.prefix_plan(group, torch.zeros(0, dtype=torch.int32), torch.zeros(0, 1, dtype=torch.int32))
    assert none.first.numel() == 1 and none.place.numel() == 7


def test_prefix_plan_of_those_that_share():
    """Told how many requests have a group, the plan lists no others."""
    table = torch.zeros(3, 4, dtype=torch.int32)
    for groups in ([2, 0, -1, 2, 0, -7, 2], [-1, -1, 1], [0, 0], [-1, 0, 5], [-1, -1]):
        group, sharing = torch.tensor(groups, dtype=torch.int32), sum(g >= 0 for g in groups)
        p = binding.prefix_plan(group, torch.tensor([3, 1, 2], dtype=torch.int32), table, sharing)
        assert p.members.numel() == max(1, sharing) and p.first.dtype == torch.int32
        first = p.first.tolist()
        assert 0 <= first[0] and first == sorted(first) and first[-1] <= p.members.numel()
        for b, g in enumerate(groups):
            if 0 <= g < 3:
                assert p.members[first[g] + p.place[b]] == b and first[g] + int(p.place[b]) < first[g + 1]
    for wrong in (-1, 4):
        with pytest.raises(RuntimeError, match="sharing"):
            binding.prefix_plan(torch.tensor([0, -1, 0], dtype=torch.int32), torch.tensor([3, 1, 2], dtype=torch.int32), table, wrong)


def test_weights_refusals(lib):  # noqa: F811
    good = dict(B=2, N=19, Hq=8, Hkv=2, D=128, scale=0.1, table_stride=1)
    n = L()
    call = lambda **kw: lib.spec_cache_weights_workspace_bytes(C.byref(filled(Weights, **dict(good, **kw))), C.byref(n))  # noqa: E731
    assert call() == 0 and n.value >= 256
    assert lib.spec_cache_weights_workspace_bytes(None, C.byref(n)) == -1
    assert lib.spec_cache_weights_workspace_bytes(C.byref(filled(Weights, **good)), None) == -1
    for f in ("q", "k_cache", "lse", "block_table", "lengths", "parent", "weights", "status"):
        assert call(**{f: None}) == -1, f
    for kw in (dict(B=0), dict(N=0), dict(N=1025), dict(Hkv=0), dict(Hq=7), dict(Hq=1), dict(num_blocks=0), dict(block_size=0),
               dict(table_width=0), dict(table_width=5, table_stride=4), dict(topo_seq_stride=18), dict(num_blocks=1 << 20, block_size=1 << 12)):
        assert call(**kw) == -2, kw
    for dtype in (-1, 0, 3):
        assert call(dtype=dtype) == -3
    for kw in (dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=-0.5)):
        assert call(**kw) == -4, kw
    for kw in (dict(D=96), dict(D=512), dict(q=0x10008), dict(k_cache=0x10002), dict(q_stride=(1, 8, 8)), dict(k_cache_stride=(8, 8, 12)),
               dict(B=65535, N=1024, Hq=64, Hkv=64, table_width=1 << 20, table_stride=1 << 20, block_size=1 << 10)):
        assert call(**kw) == -6, kw
    use = lambda ws, b: lib.spec_cache_weights(C.byref(filled(Weights, **good)), P(ws), L(b), None)  # noqa: E731
    call()
    assert use(None, 1 << 30) == -5 and use(0x10010, 1 << 30) == -5 and use(0x10000, n.value - 1) == -5


def test_logprobs_refusals(lib):  # noqa: F811
    good = dict(V=100, temperature=1.0, parent=None)
    call = lambda **kw: lib.spec_token_logprobs(C.byref(filled(Logprobs, **dict(good, **kw))), None)  # noqa: E731
    assert lib.spec_token_logprobs(None, None) == -1
    for f in ("logits", "token", "logprob", "entropy", "top_tokens", "top_logprobs", "status"):
        assert call(**{f: None}) == -1, f
    assert call(parent=0x9000, accepted_node=None) == -1
    for kw in (dict(B=0), dict(N=0), dict(V=0), dict(K=-1), dict(seq_stride=-1), dict(node_stride=-5), dict(B=1 << 14, N=1 << 14),
               dict(parent=0x9000, K=2), dict(parent=0x9000, N=1025), dict(parent=0x9000, N=5, topo_seq_stride=4)):
        assert call(**kw) == -2, kw
    for dtype in (-1, 3):
        assert call(dtype=dtype) == -3
    for kw in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=1e31), dict(top=33), dict(top=-1),
               dict(V=4, top=5)):
        assert call(**kw) == -4, kw
    assert call(logits=0x10001) == -6 and call(logits=0x10002, dtype=0) == -6


def test_evict_refusals(lib):  # noqa: F811
    good = dict(table_stride=1, row_bytes=16)
    n = L()
    size = lambda **kw: lib.spec_cache_evict_workspace_bytes(C.byref(filled(Evict, **dict(good, **kw))), C.byref(n))  # noqa: E731
    assert size() == 0 and n.value >= 8
    assert lib.spec_cache_evict_workspace_bytes(None, C.byref(n)) == -1
    assert lib.spec_cache_evict_workspace_bytes(C.byref(filled(Evict, **good)), None) == -1
    for f in ("cache", "weights", "block_table", "lengths", "owned", "free_blocks", "free_range", "lengths_out", "owned_out", "free_range_out",
              "status"):
        assert size(**{f: None}) == -1, f
    assert size(free_size=0, free_blocks=None) == 0 and size(protected_len=None) == 0
    for kw in (dict(B=0), dict(B=65536), dict(caches=0), dict(num_blocks=0), dict(block_size=0), dict(table_width=0), dict(row_bytes=0),
               dict(row_bytes=2**31), dict(table_width=2), dict(free_size=-1), dict(num_blocks=1 << 20, block_size=1 << 12)):
        assert size(**kw) == -2, kw
    for kw in (dict(budget=0), dict(budget=-3), dict(recent=-1), dict(lengths=0x50000, lengths_out=0x50000), dict(owned=0x50000, owned_out=0x50000),
               dict(owned=0x50000, lengths_out=0x50000), dict(lengths=0x50000, owned_out=0x50000), dict(free_range=0x50000, free_range_out=0x50000)):
        assert size(**kw) == -4, kw
    # a budget beyond the table costs no more than the table
    size(budget=2**31 - 1, table_width=4, table_stride=4, block_size=16)
    assert n.value <= 256 + 64 * 8
    call = lambda ws, b: lib.spec_cache_evict(C.byref(filled(Evict, **good)), P(ws), L(b), None)  # noqa: E731
    size()
    assert call(None, 1 << 30) == -5 and call(0x10010, 1 << 30) == -5 and call(0x10000, n.value - 1) == -5


@pytest.mark.parametrize("name,args", [
    ("prefix_attention", lambda t, i: (t, t, t, i[None], i, i, binding.PrefixPlan(i, i, i, i, i, i[None]))),
    ("token_logprobs", lambda t, i: (t[0, 0], i)),
    ("path_logprobs", lambda t, i: (t[0], i, i[None], i)),
    ("cache_weights", lambda t, i: (t[0, 0], t, t, t, i[None], i, i)),
    ("cache_evict", lambda t, i: (t, t[0, 0], i, i[None], i, i, i, 1))])
def test_the_calls_refuse_to_run_without_a_gpu(lib, name, args):  # noqa: F811
    with pytest.raises(RuntimeError, match="CUDA device"):
        getattr(binding, name)(*args(torch.zeros(1, 1, 1, 8), torch.zeros(1, dtype=torch.int32)))
    with pytest.raises(TypeError):
        getattr(binding, name)(*([None] * len(args(torch.zeros(1, 1, 1, 8), torch.zeros(1, dtype=torch.int32)))))


def test_paths_without_a_tree_are_refused():
    t, i = torch.zeros(1, 2, 8), torch.zeros(1, 2, dtype=torch.int32)
    for accepted, parent in ((i[0, :1], None), (None, i[0]), (None, None)):
        with pytest.raises(TypeError, match="must be tensors"):
            binding.path_logprobs(t, accepted, i, parent)
