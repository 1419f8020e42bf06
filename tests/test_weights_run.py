"""How a CTA of the weights' kernel finds its run, on the CPU: its warps over the words that they share, laid out as the source declares them, under random
interleavings between the two barriers.  Every warp has to read what all of them wrote."""
import os
import random
import re

import pytest

SOURCE = os.path.join(os.path.dirname(__file__), "..", "paper_2602_16994_b200", "csrc", "weigh.cuh")


def layout():
    """Warps of a CTA, and the places of `found`, `sums` and `request` (in words) as they follow one another in `Bars`."""
    text = re.sub(r"//.*", "", open(SOURCE).read())
    known = {}
    for names in re.findall(r"constexpr int (SUM_WARPS = .*?);", text, re.S):
        for name, value in re.findall(r"(\w+) = ([^,]+)", names):
            known[name] = eval(value.replace("/", "//"), {}, dict(known))
    body = re.search(r"struct Bars \{(.*?)\n\};", text, re.S).group(1)
    at, place = 0, {}
    for kind, rest in re.findall(r"(int|Request) (.*?);", body, re.S):
        for name, many in re.findall(r"(\w+)(?:\[(.*?)\])?(?:,|$)", rest.strip()):
            place[name] = at
            at += (eval(many.replace("/", "//"), {}, dict(known)) if many else 1) * (4 if kind == "Request" else 1)
    return known["NT"] // 32, place, at


def runs(lengths, ctas, c, warps, place, words, rng):
    """What each warp of CTA c takes for the length of all units, and the request that the CTA begins in; `lengths` of the requests in order."""
    memory = [rng.randrange(1, 10**6) for _ in range(words)]      # (whatever was there before)
    threads = warps * 32
    per = -(-len(lengths) // threads)
    mine = [sum(lengths[t * per:(t + 1) * per]) for t in range(threads)]
    for w in rng.sample(range(warps), warps):
        memory[place["sums"] + w] = sum(mine[w * 32:w * 32 + 32])
    memory[place["found"]:place["found"] + 2] = [len(lengths), 0]
    # ---- the first barrier
    got = {}
    for w in rng.sample(range(warps), warps):
        sums = [memory[place["sums"] + x] for x in range(warps)]
        total = sum(sums)
        got[w] = total
        start = total // ctas * c + min(c, total % ctas)
        ahead = sum(sums[:w])
        for t in range(w * 32, w * 32 + 32):
            if ahead <= start < ahead + mine[t]:
                for b in range(t * per, min(len(lengths), (t + 1) * per)):
                    if start < ahead + lengths[b]:
                        memory[place["found"]:place["found"] + 2] = [b, start - ahead]
                        memory[place["request"]:place["request"] + 4] = [777, 19, 0, 796]         # (of a request: its tokens, nodes and entries)
                        break
                    ahead += lengths[b]
                break
            ahead += mine[t]
    # ---- the second barrier
    return got, memory[place["found"]:place["found"] + 2], memory[place["request"]:place["request"] + 4]


@pytest.mark.parametrize("requests", [1, 8, 333, 640, 641, 700, 768, 769, 2000])
def test_every_warp_reads_what_all_of_them_wrote(requests):
    warps, place, words = layout()
    rng = random.Random(requests)
    for _ in range(60):
        lengths = [rng.choice([0, 2, 7, 100]) for _ in range(requests - 1)] + [5]
        ctas, total = 148, sum(lengths)
        c = rng.randrange(min(ctas, total))
        got, found, request = runs(lengths, ctas, c, warps, place, words, rng)
        assert set(got.values()) == {total}
        start = total // ctas * c + min(c, total % ctas)
        b = next(b for b in range(requests) if sum(lengths[:b + 1]) > start)
        assert found == [b, start - sum(lengths[:b])] and request == [777, 19, 0, 796]


def test_the_model_sees_a_warp_without_an_entry():
    warps, place, words = layout()
    short = dict(place, request=place["sums"] + warps - 4)        # (four warps' entries lie in the request)
    rng, wrong = random.Random(1), 0
    for _ in range(40):
        got, _, request = runs([10] * 8, 148, rng.randrange(80), warps, short, words, rng)
        wrong += set(got.values()) != {80}
    assert wrong > 10
