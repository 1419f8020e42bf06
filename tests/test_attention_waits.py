"""The waits of the tree attention's kernel, on the CPU: a model of its roles (copying warps, product warps, row warps, the tensor cores' queue and
copies that end whenever they like) over barriers whose phases tell only even from odd, under random interleavings.

A run fails where it comes to a stand, or where a wait passes before the phase that it means is complete.  The protocol as it is must not fail; each of
three earlier forms of it must, so that the model is known to see such faults."""
import random

import pytest

# row blocks of 128, row warpgroups (one in turns: two of one block), slots in flight, slots of a tile's keys or values, parts of a tile
FORMS = {"turns, D 128": (1, 2, 5, 1, 1), "turns, D 64": (1, 2, 10, 1, 1), "two blocks, D 128": (2, 2, 4, 1, 2), "two blocks, D 64": (2, 2, 10, 1, 2),
         "one warpgroup, D 256": (1, 1, 4, 2, 1)}
FILLED, COPIERS = 132, 4                                         # arrivals that fill a slot; copying warps


class Fault(Exception):
    pass


class Barrier:
    def __init__(self, name, count):
        self.name, self.count, self.pending, self.bytes, self.done = name, count, count, 0, 0

    def arrive(self, n=1):
        if self.pending < n:
            raise Fault(f"{self.name}: more arrivals than its count")
        self.pending -= n
        self.turn()

    def land(self, n):
        self.bytes -= n
        self.turn()

    def turn(self):
        if self.pending == 0 and self.bytes == 0:
            self.done, self.pending = self.done + 1, self.count

    def passes(self, parity):
        return self.done & 1 != parity


def wait(bar, phase):
    """Waits for a phase by its number, which the barrier knows as even or odd."""
    while not bar.passes(phase & 1):
        yield bar.name
    if bar.done < phase + 1:
        raise Fault(f"{bar.name}: passed after {bar.done} phases, phase {phase} was meant")


class Run:
    def __init__(self, rng, form, boxes, earlier=None, units=None):
        self.rng, self.boxes, self.earlier = rng, boxes, earlier
        self.blocks, self.groups, self.slots, self.step, self.parts = FORMS[form]
        self.turns = self.blocks == 1 and self.groups == 2
        # tiles of each unit of the run, and whether its second block has rows
        self.units = units or [(rng.choice([1, 1, 1, 2, 2, 3, 4, 7]), rng.random() < 0.5) for _ in range(rng.randint(1, 9))]
        many = lambda name, n, count: [Barrier(f"{name}{i}", count) for i in range(n)]  # noqa: E731
        self.full, self.empty = many("full", self.slots, FILLED), many("empty", self.slots, self.blocks)
        self.q_full, self.q_empty = Barrier("q_full", 128), Barrier("q_empty", self.groups)
        self.s_full, self.p_full = many("s_full", 4, 1), many("p_full", 4, 4)
        self.pv_done = [many(f"pv_done{o}", 2, 1) for o in range(2)]
        self.o_empty = many("o_empty", 2, 8 if self.turns else 4)
        # how each copying warp copies its part of each tile: by map, by threads, or by threads with values held back
        self.kinds = {}
        tile = 0
        for steps, _ in self.units:
            for i in range(steps):
                for w in range(COPIERS):
                    self.kinds[tile, w] = rng.choice(["map", "map", "threads"] if i else ["map", "hold", "threads"])
                tile += 1
        self.tensor, self.flying, self.meeting = [], [], [0, 0]  # products and arrivals behind them; copies; the barrier of both warpgroups

    # ---- rows -----------------------------------------------------------------------------------------------------------------
    def products(self, o, n):
        return wait(self.pv_done[o][0], n) if self.earlier == "one barrier" else wait(self.pv_done[o][n & 1], n >> 1)

    def meet(self):
        mine = self.meeting[1]
        self.meeting[0] += 1
        if self.meeting[0] == 8:
            self.meeting[0], self.meeting[1] = 0, mine + 1
        while self.meeting[1] == mine:
            yield "both warpgroups"

    def rows(self, warp):
        w = warp >> 2
        t = w if self.blocks == 2 else 0
        part = tile = 0
        for steps, second in self.units:
            if t == 1 and not second:
                tile += steps
                continue
            begun = False
            for _ in range(steps):
                if self.turns and tile & 1 != w:
                    tile += 1
                    continue
                for h in range(self.parts):
                    buf = t * self.parts + h if self.blocks == 2 else tile & 1
                    yield from wait(self.s_full[buf], part // self.parts if self.blocks == 2 else tile >> 1)
                    yield None
                    if begun and self.rng.random() < 0.2:        # a new reference
                        yield from self.products(w, part - 1)
                    yield None
                    self.p_full[buf].arrive()
                    begun, part = True, part + 1
                    yield None
                tile += 1
            if begun:
                if self.earlier == "one barrier" and not self.turns and part > 1:
                    yield from self.products(w, part - 2)
                yield from self.products(w, part - 1)
            if self.turns:
                yield from self.meet()
            for _ in range(self.rng.choice([0, 0, 3])):
                yield None
            self.o_empty[t].arrive()
            yield None

    # ---- products -------------------------------------------------------------------------------------------------------------
    def copied(self, k):
        for k in range(k, k + self.step):
            if self.turns and k >= self.slots and self.earlier != "not seen let go":
                yield from wait(self.empty[k % self.slots], k // self.slots - 1)
            yield from wait(self.full[k % self.slots], k // self.slots)

    def release(self, k):
        self.tensor += [self.empty[x % self.slots] for x in range(k, k + self.step)]

    def product(self, k, bar, release):
        self.tensor.append(None)
        if release:
            self.release(k)
        self.tensor.append(bar)

    def sums(self, o, part, k, release):
        self.product(k, self.pv_done[o][0 if self.earlier == "one barrier" else part & 1], release)

    def issue(self, m):
        n = tile = own = units = own_units = 0
        for steps, second in self.units:
            keys = [n + 2 * self.step * i for i in range(steps)]
            values = [k + self.step for k in keys]
            yield from wait(self.q_full, units)
            if self.blocks == 2 and m == 1 and not second:
                for k in (x for pair in zip(keys, values) for x in pair):
                    yield from self.copied(k)
                    self.release(k)
                self.tensor.append(self.q_empty)
            elif self.blocks == 2:
                yield from self.copied(keys[0])
                for h in range(self.parts):
                    self.product(keys[0], self.s_full[m * self.parts + h], h == self.parts - 1)
                if steps == 1:
                    self.tensor.append(self.q_empty)
                for i in range(steps):
                    yield from self.copied(values[i])
                    for h in range(self.parts):
                        buf, last = m * self.parts + h, h == self.parts - 1
                        yield from wait(self.p_full[buf], own)
                        if i == 0 and h == 0 and own_units:
                            yield from wait(self.o_empty[m], own_units - 1)
                        self.sums(m, own * self.parts + h, values[i], last)
                        if i + 1 == steps:
                            continue
                        if h == 0:
                            yield from self.copied(keys[i + 1])
                        self.product(keys[i + 1], self.s_full[buf], last)
                        yield None
                    if i + 2 == steps:
                        self.tensor.append(self.q_empty)
                    own += 1
                own_units += 1
            elif self.turns:
                first = (m - tile) & 1
                if first >= steps:
                    self.tensor.append(self.q_empty)
                for i in range(first, steps, 2):
                    yield from self.copied(keys[i])
                    self.product(keys[i], self.s_full[m], True)
                    if i + 2 >= steps:
                        self.tensor.append(self.q_empty)
                    yield None
                    yield from self.copied(values[i])
                    yield from wait(self.p_full[m], own)
                    if i == first and units:
                        yield from wait(self.o_empty[0], units - 1)
                    self.sums(m, own, values[i], True)
                    own += 1
                    yield None
            else:
                yield from self.copied(keys[0])
                self.product(keys[0], self.s_full[tile & 1], True)
                if steps == 1:
                    self.tensor.append(self.q_empty)
                for i in range(steps):
                    at = tile + i
                    if i + 1 < steps:
                        yield from self.copied(keys[i + 1])
                        self.product(keys[i + 1], self.s_full[at + 1 & 1], True)
                        if i + 2 == steps:
                            self.tensor.append(self.q_empty)
                    yield from self.copied(values[i])
                    yield from wait(self.p_full[at & 1], at >> 1)
                    if i == 0 and units:
                        yield from wait(self.o_empty[0], units - 1)
                    self.sums(0, at, values[i], True)
                    yield None
            tile, n, units = tile + steps, n + 2 * self.step * steps, units + 1

    # ---- copies ---------------------------------------------------------------------------------------------------------------
    def copy(self, w):
        n, held, queries, tile = 0, None, 0, 0

        def clean():
            nonlocal held
            for k in range(held, held + self.step):
                self.full[k % self.slots].arrive(FILLED // COPIERS)
            held = None

        def room(bar, phase):
            if held is not None and not bar.passes(phase & 1):
                clean()
            yield from wait(bar, phase)

        def copy_rows(kind, values):
            nonlocal n, held
            for k in range(n, n + self.step):
                if k >= self.slots:
                    yield from room(self.empty[k % self.slots], k // self.slots - 1)
            hold = values and kind == "hold"
            for k in range(n, n + self.step):
                bar = self.full[k % self.slots]
                if kind == "map":
                    bar.bytes += 8
                    bar.arrive(FILLED // COPIERS)
                    self.flying += [lambda bar=bar: bar.land(4)] * 2
                elif not hold:
                    bar.arrive()
                    self.flying.append(lambda bar=bar: bar.arrive(FILLED // COPIERS - 1))
            yield None
            if held is not None:
                clean()
            if hold:
                held = n
            n += self.step

        def copy_q():
            nonlocal queries
            if self.boxes and w and self.earlier != "all ask":
                return
            if queries:
                yield from room(self.q_empty, queries - 1)
            queries += 1
            if not self.boxes:
                self.flying.append(lambda: self.q_full.arrive(32))
            elif w == 0:
                self.q_full.bytes += 4
                self.q_full.arrive(128)
                self.flying.append(lambda: self.q_full.land(4))

        for steps, _ in self.units:
            for i in range(steps):
                kind, tile = self.kinds[tile, w], tile + 1
                yield from copy_rows(kind, False)
                if i == 0:
                    yield from copy_q()
                yield None
                yield from copy_rows(kind, True)
        if held is not None:
            clean()

    # ---- interleaving ---------------------------------------------------------------------------------------------------------
    def go(self):
        roles = {f"rows {i}": self.rows(i) for i in range(4 * self.groups)}
        roles.update({f"products {m}": self.issue(m) for m in range(self.groups)})
        roles.update({f"copies {w}": self.copy(w) for w in range(COPIERS)})
        speed, at, idle, turn = {}, {}, 0, 0
        while roles:
            if turn % 40 == 0:                                   # who is slow changes
                speed = {name: self.rng.choice([0.02, 0.3, 1, 1, 1]) for name in [*roles, "tensor", "flying"]}
            turn += 1
            names = list(roles) + ["tensor"] * bool(self.tensor) + ["flying"] * bool(self.flying)
            name = self.rng.choices(names, [speed[x] for x in names])[0]
            if name == "tensor":                                 # in order
                bar = self.tensor.pop(0)
                if bar:
                    bar.arrive()
            elif name == "flying":                               # in any order
                self.flying.pop(self.rng.randrange(len(self.flying)))()
            else:
                try:
                    at[name] = next(roles[name])
                    idle = idle + 1 if at[name] else 0
                    if idle > 4000 and not self.tensor and not self.flying:
                        raise Fault(f"at a stand: { {k: at.get(k) for k in roles} }")
                    continue
                except StopIteration:
                    del roles[name]
            idle = 0


def faults(seeds, form, boxes, **kw):
    found = []
    for seed in seeds:
        try:
            Run(random.Random(seed), form, boxes, **kw).go()
        except Fault as e:
            found.append(f"seed {seed}: {e}")
    return found


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("boxes", [True, False])
def test_no_interleaving_comes_to_a_stand_or_passes_too_early(form, boxes):
    assert not faults(range(60), form, boxes)
    assert not faults(range(30), form, boxes, units=[(1, True)] * 10)


@pytest.mark.parametrize("earlier,form,units", [
    # the last but one product and the last waited for on one barrier
    ("one barrier", "two blocks, D 128", None), ("one barrier", "one warpgroup, D 256", None),
    # all copying warps wait for room for queries that one of them brings
    ("all ask", "turns, D 128", [(1, True)] * 10), ("all ask", "one warpgroup, D 256", [(1, True)] * 10),
    # a filling of a slot waited for whose last filling was the other warp's
    ("not seen let go", "turns, D 128", None)])
def test_the_model_sees_what_was_wrong_with_earlier_forms(earlier, form, units):
    assert faults(range(150), form, True, earlier=earlier, units=units)
