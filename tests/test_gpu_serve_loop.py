"""The operators together, as a decoding loop uses them: a shared prompt, steps of draft trees in two layers, weights of entries, log probabilities of
what was put out, commits and evictions; each against its restatement on what the caches hold then."""
import pytest
import torch

from . import serve_ref, step_ref as ref
from .test_gpu_serve import check_rows
from .test_gpu_step import chain, tree
from paper_2602_16994_b200 import binding
from paper_2602_16994_b200.tree_cache import TreeCache

pytestmark = pytest.mark.gpu

I32 = torch.int32


def attend_and_check(cache, layer, q):
    """One layer's attention and its weights; the bounds are those of the tests of each call."""
    before, fresh = cache.weights.cpu(), cache.fresh
    k, v = cache.storage[2 * layer].cpu(), cache.storage[2 * layer + 1].cpu()
    got = cache.attend(layer, q, want_lse=True)
    torch.cuda.synchronize()
    lengths, parent, table, D = cache.lengths.cpu(), cache.parent.cpu(), cache.block_table.cpu(), q.shape[-1]
    want = ref.attention(q.cpu(), k, v, table, lengths, parent)
    assert got.status.cpu().tolist() == want["status"].tolist() == [0] * len(lengths)
    score = want["reach"][..., None] * (D + 4) * 2.0**-24
    bound = want["mass"] * (2 * score + 2.0**-8 + 2.0**-19) + want["out"].abs() * 2.0**-8
    live = want["live"]
    assert bool(((got.out.cpu().double() - want["out"]).abs() <= bound)[live].all())
    w = serve_ref.weights(before, q.cpu(), k, got.lse.cpu(), table, lengths, parent, protected=cache.protected.cpu(), fresh=fresh)
    assert cache.weigh_status.cpu().tolist() == w["status"].tolist()
    terms = q.shape[1] * q.shape[2]
    bound = w["size"] * 3 * 2.0**-24 + w["reach"] * (D // 16 + 1) * 2.0**-22 + w["got"] * (2.0**-22 + terms * 2.0**-24) + w["weights"].abs() * 2.0**-23
    assert bool(((cache.weights.cpu().double() - w["weights"]).abs() <= bound).all())


def test_a_loop_of_shared_prompts_steps_and_evictions():
    g = torch.Generator().manual_seed(0)
    B, layers, Hq, Hkv, D, V = 4, 2, 8, 2, 64, 3000
    cache = TreeCache(B, layers, 60, 16, Hkv, D, width=14, weigh=True)
    cache.lengths = torch.tensor([0, -1, -1, 0], dtype=I32, device="cuda")
    turn = (10000.0 ** (-torch.arange(0, D, 2).double() / D)).float().cuda()
    draft = tree(2, 1, 2)
    evicted = 0
    for step in range(9):
        parent = chain(70) if step == 0 else draft
        N = parent.shape[0]
        s = cache.begin(parent.cuda())
        assert s.status.tolist() == [0] * B
        for layer in range(layers):
            qkv = torch.randn(B * N, Hq + 2 * Hkv, D, generator=g).bfloat16().cuda()
            q = cache.write(layer, qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], turn)
            attend_and_check(cache, layer, q.view(B, N, Hq, D))
        if step == 0:
            node = torch.tensor([69, -1, -1, 65], dtype=I32)
        else:
            node = torch.randint(0, N, (B,), generator=g).int()
            logits = torch.randn(B, N, V, generator=g).bfloat16()
            tokens = torch.randint(0, V, (B, N), generator=g).int()
            got = binding.path_logprobs(logits.cuda(), node.cuda(), tokens.cuda(), parent.cuda(), top=3)
            check_rows(got, serve_ref.path_logprobs(logits, node, tokens, parent, 1.0, 3), V, 1.0, 3)
        done = cache.commit(node.cuda())
        assert done.status.tolist() == [0] * B
        if step == 0:
            assert cache.share(0, [1, 2]) == 64
            continue
        args = [x.cpu() for x in (cache.storage, cache.weights, cache.lengths, cache.block_table, cache.owned, cache.free_blocks, cache.free_range)]
        want, _ = serve_ref.evict(*args, 72, 4, cache.protected.cpu())
        cut = cache.evict(72, recent=4)
        evicted += int((args[2] - cut.lengths.cpu()).sum())
        for name in ("lengths", "owned", "free_range", "status"):
            assert torch.equal(getattr(cut, name).cpu(), want[name]), name
        assert torch.equal(cache.storage.cpu(), want["cache"]) and torch.equal(cache.free_blocks.cpu(), want["free_blocks"])
        assert torch.equal(cache.weights.cpu(), want["weights"])
    assert evicted > 20 and int(cache.dropped.sum()) == evicted and cache.plan is not None


def test_the_cache_s_calls_on_another_stream():
    """The whole step on a stream that is named, against the same step on the current one."""
    out = []
    for named in (False, True):
        g = torch.Generator().manual_seed(1)
        side = torch.cuda.Stream() if named else None
        kw = dict(stream=side) if named else {}
        cache = TreeCache(2, 1, 40, 16, 2, 64, width=8, weigh=True)
        for step in range(4):
            parent = (chain(40) if step == 0 else tree(2, 1, 2)).cuda()
            N = parent.shape[0]
            qkv = torch.randn(2 * N, 12, 64, generator=g).bfloat16().cuda()
            node = torch.full((2,), N - 1, dtype=I32, device="cuda")
            if named:
                side.wait_stream(torch.cuda.current_stream())
            cache.begin(parent, **kw)
            q = cache.write(0, qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], torch.full((32,), 0.1, device="cuda"), **kw)
            y = cache.attend(0, q.view(2, N, 8, 64), **kw)
            cache.commit(node, **kw)
            if step:
                cache.evict(41, recent=2, **kw)
            if named:
                torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        out.append((y.out.clone(), cache.weights.clone(), cache.lengths.clone(), cache.dropped.clone(), cache.step.positions.clone()))
    for a, b in zip(*out):
        assert torch.equal(a, b)
