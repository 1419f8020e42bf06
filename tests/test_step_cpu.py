"""Host-side checks of the operators around a verification: what they refuse, before a device is touched."""
import ctypes as C

import pytest
import torch

from paper_2602_16994_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


P, S3, S2 = C.c_void_p, C.c_int64 * 3, C.c_int64 * 2
I, L, F = C.c_int32, C.c_int64, C.c_float


def struct(name, *fields):
    return type(name, (C.Structure,), {"_fields_": [(f, t) for t, names in fields for f in names.split()]})


Slots = struct("SpecSlots", (I, "B N block_size table_width"), (P, "lengths n_nodes parent"), (L, "topo_seq_stride"), (P, "block_table"),
               (L, "table_stride"), (P, "owned free_blocks"), (I, "free_size"),
               (P, "free_range slots positions owned_out free_range_out status"))
Rope = struct("SpecNormRope", (I, "T Hq Hkv D rot pairs dtype num_blocks block_size"), (P, "q k v"), (S2, "q_stride k_stride v_stride"),
              (P, "q_weight k_weight"), (F, "eps"), (P, "inv_freq positions slots q_out"), (S2, "q_out_stride"), (P, "k_cache v_cache"),
              (S3, "k_cache_stride v_cache_stride"))
Attention = struct("SpecAttention", (I, "B N Hq Hkv D dtype num_blocks block_size table_width window sinks"), (F, "scale"), (P, "q"),
                   (S3, "q_stride"), (P, "k_cache v_cache"), (S3, "k_cache_stride v_cache_stride"), (P, "block_table"), (L, "table_stride"),
                   (P, "lengths n_nodes parent"), (L, "topo_seq_stride"), (P, "out"), (S3, "out_stride"), (P, "lse status"))
Commit = struct("SpecCommit", (I, "B N caches num_blocks block_size table_width"), (P, "cache"), (S3, "stride"), (L, "row_bytes"),
                (P, "block_table"), (L, "table_stride"), (P, "lengths n_nodes parent"), (L, "topo_seq_stride"),
                (P, "accepted_node lengths_out status"))
Chains = struct("SpecChains", (I, "B V max_drafts dtype"), (L, "n_drafts"), (P, "target_probs draft_probs"), (L, "target_stride draft_stride"),
                (P, "token cu_drafts u_accept u_bonus accept_len out_tokens bonus_token status"))


def filled(cls, **kw):
    """Sizes of 1, strides of 0, a distinct address for every pointer; then what is given."""
    s = cls()
    for n, (f, t) in enumerate(cls._fields_):
        if t is P:
            setattr(s, f, 0x10000 * (n + 1))
        elif t is I:
            setattr(s, f, 1)
    for f, v in kw.items():
        setattr(s, f, S3(*v) if isinstance(v, tuple) and len(v) == 3 else S2(*v) if isinstance(v, tuple) else v)
    return s


def good_attention(**kw):
    return filled(Attention, **dict(dict(B=2, N=19, Hq=8, Hkv=2, D=128, scale=0.1, table_stride=1), **kw))


def test_attention_refusals(lib):
    n = L()
    size = lambda **kw: lib.spec_tree_attention_workspace_bytes(C.byref(good_attention(**kw)), C.byref(n))  # noqa: E731
    assert size() == 0 and n.value >= 256
    assert lib.spec_tree_attention_workspace_bytes(None, C.byref(n)) == -1
    assert lib.spec_tree_attention_workspace_bytes(C.byref(good_attention()), None) == -1
    for f in ("q", "k_cache", "v_cache", "block_table", "lengths", "parent", "out", "status"):
        assert size(**{f: None}) == -1, f
    for kw in (dict(B=0), dict(N=0), dict(N=1025), dict(Hkv=0), dict(Hq=7), dict(Hq=1), dict(num_blocks=0), dict(block_size=0),
               dict(table_width=0), dict(table_width=5, table_stride=4), dict(topo_seq_stride=18), dict(num_blocks=1 << 20, block_size=1 << 12)):
        assert size(**kw) == -2, kw
    for dtype in (-1, 0, 3):
        assert size(dtype=dtype) == -3
    for kw in (dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=-0.5), dict(window=-1), dict(sinks=-1)):
        assert size(**kw) == -4, kw
    for kw in (dict(D=96), dict(D=512), dict(q=0x10008), dict(k_cache=0x10002), dict(out=0x10004), dict(q_stride=(1, 8, 8)),
               dict(k_cache_stride=(8, 8, 12)), dict(out_stride=(8, 4, 8))):
        assert size(**kw) == -6, kw
    assert size(n_nodes=None, lse=None) == 0
    call = lambda ws, b: lib.spec_tree_attention(C.byref(good_attention()), P(ws), L(b), None)  # noqa: E731
    size()
    assert call(None, 1 << 30) == -5 and call(0x10010, 1 << 30) == -5 and call(0x10000, n.value - 1) == -5


def test_slots_refusals(lib):
    call = lambda **kw: lib.spec_cache_slots(C.byref(filled(Slots, **dict(dict(table_stride=1, n_nodes=None), **kw))), None)  # noqa: E731
    assert lib.spec_cache_slots(None, None) == -1
    for f in ("lengths", "parent", "block_table", "owned", "free_blocks", "free_range", "slots", "positions", "owned_out", "free_range_out",
              "status"):
        assert call(**{f: None}) == -1, f
    for kw in (dict(B=0), dict(N=0), dict(N=1025), dict(block_size=0), dict(table_width=0), dict(table_width=2), dict(free_size=-1),
               dict(N=4, topo_seq_stride=3)):
        assert call(**kw) == -2, kw
    assert call(owned=0x50000, owned_out=0x50000) == -4
    assert call(free_range=0x50000, free_range_out=0x50000) == -4


def test_norm_rope_refusals(lib):
    call = lambda **kw: lib.spec_norm_rope_cache(C.byref(filled(Rope, **dict(dict(D=64, rot=64), **kw))), None)  # noqa: E731
    assert lib.spec_norm_rope_cache(None, None) == -1
    for f in ("q", "k", "v", "inv_freq", "positions", "slots", "q_out", "k_cache", "v_cache"):
        assert call(**{f: None}) == -1, f
    for kw in (dict(T=0), dict(Hq=0), dict(Hkv=0), dict(num_blocks=0), dict(block_size=0), dict(num_blocks=1 << 30, block_size=4)):
        assert call(**kw) == -2, kw
    assert call(dtype=3) == -3
    for kw in (dict(pairs=2), dict(pairs=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(rot=-2)):
        assert call(**kw) == -4, kw
    for kw in (dict(D=4), dict(D=12), dict(D=264), dict(rot=80), dict(rot=24)):
        assert call(**kw) == -6, kw


def test_commit_refusals(lib):
    good = dict(table_stride=1, row_bytes=16)
    call = lambda **kw: lib.spec_cache_commit(C.byref(filled(Commit, **dict(good, **kw))), None)  # noqa: E731
    assert lib.spec_cache_commit(None, None) == -1
    for f in ("cache", "block_table", "lengths", "parent", "accepted_node", "lengths_out", "status"):
        assert call(**{f: None}) == -1, f
    for kw in (dict(B=0), dict(B=65536), dict(N=1025), dict(caches=0), dict(num_blocks=0), dict(row_bytes=0), dict(row_bytes=2**31), dict(table_stride=0)):
        assert call(**kw) == -2, kw
    assert call(lengths=0x50000, lengths_out=0x50000) == -4


def test_chains_refusals(lib):
    good = dict(n_drafts=3, target_stride=1, draft_stride=1)
    call = lambda **kw: lib.spec_verify_probs(C.byref(filled(Chains, **dict(good, **kw))), None)  # noqa: E731
    assert lib.spec_verify_probs(None, None) == -1
    for f in ("target_probs", "token", "cu_drafts", "u_accept", "u_bonus", "accept_len", "out_tokens", "bonus_token", "status"):
        assert call(**{f: None}) == -1, f
    for kw in (dict(B=0), dict(V=0), dict(max_drafts=-1), dict(n_drafts=-1), dict(V=2), dict(V=2, target_stride=2)):
        assert call(**kw) == -2, kw
    assert call(dtype=2) == -3
    assert call(V=1 << 30, target_stride=1 << 30, draft_stride=1 << 30) == -6


@pytest.mark.parametrize("name,args", [
    ("cache_slots", lambda t, i: (i, i, i[None], i, i, i, 16)),
    ("norm_rope_cache", lambda t, i: (t[None], t[None], t[None], t[0, 0], i, i, t, t)),
    ("tree_attention", lambda t, i: (t, t, t, i[None], i, i)),
    ("cache_commit", lambda t, i: (t, i, i, i, i[None])),
    ("verify_probs", lambda t, i: (t[0], None, i, i, t, t, 1))])
def test_the_calls_refuse_to_run_without_a_gpu(lib, name, args):
    with pytest.raises(RuntimeError, match="CUDA device"):
        getattr(binding, name)(*args(torch.zeros(1, 1, 1, 8), torch.zeros(1, dtype=torch.int32)))
    with pytest.raises(TypeError):
        getattr(binding, name)(*([None] * len(args(torch.zeros(1, 1, 1, 8), torch.zeros(1, dtype=torch.int32)))))
