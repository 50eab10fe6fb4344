"""The waits of the kernels for a bias by buckets (csrc/rib_bias_fwd_sm100.cu, csrc/rib_bias_bwd_sm100.cu) in the model of tests/test_frame_barriers.py.
What they have beside those of the rank-r kernels: items decoded once by the producer, eight at a time into a ring of two eights that nothing
guards; in the backward pass two to four items' K and V in flight, a ring of three query tiles, and warps that sum the gradient of the bias from
the dS tiles in shared memory.  No GPU needed."""
import heapq

import pytest

from test_frame_barriers import Model, WrongPhase

EIGHT = 8


class Items(Model):
    """The ring of items: `n` counts them."""
    eights = 2

    def write_items(self, n, readers):
        if n % EIGHT == 0:
            for old in range(n - self.eights * EIGHT, n - (self.eights - 1) * EIGHT):
                assert old < 0 or all(("item", old, r) in self.finished for r in readers), "an item is overwritten before all have read it"
            self.issued.update(("item", n + k) for k in range(EIGHT))
            self.arrive("items")

    def read_item(self, n, reader):
        if n % EIGHT == 0:
            yield "wait", "items", n // EIGHT
        assert ("item", n) in self.issued and ("item", n + self.eights * EIGHT) not in self.issued
        yield "delay", self.delay("soft") / 4
        assert ("item", n + self.eights * EIGHT) not in self.issued
        self.finished.add(("item", n, reader))

    def copy(self, what, bar):
        self.issued.add(what)

        def complete():
            self.finished.add(what)
            self.arrive(bar)
        self.later(self.delay("load"), complete)

    def go(self, processes):
        self.pipe = {}
        for process in processes:
            self.later(self.delay("soft"), lambda process=process: self.step(process))
        while self.queue:
            self.now, _, what = heapq.heappop(self.queue)
            what()


class Forward(Items):
    """An item's output is read inside the next item's first block, with the item read once more."""
    STAGES = 4

    def __init__(self, items, seed):
        super().__init__(items, seed, True)
        self.scale["load"] = self.rng.choice((0.1, 1.0, 5.0))
        self.readers = ["s", ("pv", 0), ("pv", 1)] + [("out", t, h) for t in range(2) for h in range(2)]

    def producer(self):
        block = 0
        for n, blocks in enumerate(self.items):
            self.write_items(n, self.readers)
            if n >= 2:
                yield "wait", ("qempty", n & 1), (n >> 1) - 1
            self.copy(("q", n), ("qfull", n & 1))
            for block in range(block, block + blocks):
                for x in "kv":
                    if block >= self.STAGES:
                        yield "wait", (x + "empty", block % self.STAGES), block // self.STAGES - 1
                    self.copy((x, block), (x + "full", block % self.STAGES))
            block += 1

    def arrive(self, bar, count=1):
        super().arrive(bar, 2 if bar[0] == "vempty" else count)

    def scores(self):
        block = 0
        for n, blocks in enumerate(self.items):
            yield from self.read_item(n, "s")
            yield "wait", ("qfull", n & 1), n >> 1
            for j in range(blocks):
                yield "wait", ("kfull", block % self.STAGES), block // self.STAGES
                for tile in range(2):
                    yield ("wait", *self.pv_phase(1 - tile, (2 * block + tile - 3) >> 1))
                    assert 2 * block + tile < 3 or ("pv", 2 * block + tile - 3) in self.finished
                    bars = [self.score_phase(tile, block)[0]]
                    if tile:
                        bars += [("kempty", block % self.STAGES)] + ([("qempty", n & 1)] if j == blocks - 1 else [])
                    self.contract("s", ("s", 2 * block + tile), bars)
                block += 1

    def pv(self, tile):
        block = 0
        for n, blocks in enumerate(self.items):
            yield from self.read_item(n, ("pv", tile))
            for j in range(blocks):
                yield "wait", ("vfull", block % self.STAGES), block // self.STAGES
                yield "wait", ("pready", tile, block & 1), block >> 1
                self.contract(f"pv{tile}", ("pv", 2 * block + tile), [self.pv_phase(tile, block)[0], ("vempty", block % self.STAGES)])
                block += 1

    def epilogue(self, n, tile, half, block):
        yield ("wait", *self.pv_phase(tile, block))
        assert ("pv", 2 * block + tile) in self.finished and ("pv", 2 * block + 2 + tile) not in self.issued
        assert ("item", n + self.eights * EIGHT) not in self.issued
        self.finished.add(("item", n, ("out", tile, half)))
        yield "delay", self.delay("soft") / 4

    def softmax(self, tile, half):
        block = 0
        for n, blocks in enumerate(self.items):
            yield from self.read_item(n, ("softmax", tile, half))
            for j in range(blocks):
                yield ("wait", *self.score_phase(tile, block))
                assert ("s", 2 * block + tile) in self.finished
                yield "delay", self.delay("soft")
                if j == 0 and n:
                    yield from self.epilogue(n - 1, tile, half, block - 1)
                self.arrive(("pready", tile, block & 1), 2)
                block += 1
        yield from self.epilogue(n, tile, half, block - 1)

    def run(self):
        self.go([self.producer(), self.scores(), self.pv(0), self.pv(1)] + [self.softmax(t, h) for t in range(2) for h in range(2)])
        assert sum(f[0] == "item" and f[2][0] == "out" for f in self.finished if len(f) == 3) == 4 * len(self.items), "the warps wait for one another"


class Backward(Items):
    """Items of `tiles[n]` query tiles; unit u = 2 * tile + half, its scores in buffer u mod 3.  A role of several warps is two processes, the
    four that sum the gradient of the bias are four.  `fault`: a rule left out."""
    STAGES, WARPS = 3, (0, 1)

    def __init__(self, tiles, seed, slots, fault=None):
        super().__init__(tiles, seed, True)
        self.slots, self.fault = slots, fault
        for name in ("load", "dq", "v", "drain", "sum"):
            self.scale[name] = self.rng.choice((0.1, 1.0, 5.0))
        if fault == "ring":
            self.eights = 1
        self.counts = {"pready": 2, "dqfree": 2, "accfree": 2, "dsfree": 1 if fault == "sums" else 5, "kvempty": 1 if fault == "slot" else 3}
        self.sums = [("sum", h, sub) for h in range(2) for sub in range(2)]
        self.readers = ["s", "v", "dq"] + [("p", h, w) for h in range(2) for w in self.WARPS] + [("drain", w) for w in self.WARPS] + self.sums
        self.first = [sum(tiles[:n]) for n in range(len(tiles) + 1)]

    def arrive(self, bar, count=1):
        super().arrive(bar, self.counts.get(bar if isinstance(bar, str) else bar[0], 1))

    def tiles_of(self, n):
        return range(self.first[n], self.first[n + 1])

    def all_done(self, *what):
        return all((*what, w) in self.finished for w in self.WARPS)

    def producer(self):
        for n in range(len(self.items)):
            self.write_items(n, self.readers)
            slot, before = n % self.slots, n - self.slots
            yield "wait", ("kvempty", slot), n // self.slots - 1
            if before >= 0:
                assert all(("s", 2 * g + h) in self.finished and ("dq", g) in self.finished for g in self.tiles_of(before) for h in range(2)), "K or V in use"
                assert self.all_done("out", before), "V under the rows of dV"
            self.copy(("kv", n), ("kvfull", slot))
            for g in self.tiles_of(n):
                if g >= self.STAGES:
                    yield "wait", ("qempty", g % self.STAGES), g // self.STAGES - 1
                    for u in (2 * (g - self.STAGES), 2 * (g - self.STAGES) + 1):
                        assert ("s", u) in self.finished and ("v", u) in self.finished, "query rows in use"
                self.copy(("q", g), ("qfull", g % self.STAGES))

    def scores(self):
        for n in range(len(self.items)):
            yield from self.read_item(n, "s")
            yield "wait", ("kvfull", n % self.slots), n // self.slots
            for g in self.tiles_of(n):
                yield "wait", ("qfull", g % self.STAGES), g // self.STAGES
                for u in (2 * g, 2 * g + 1):
                    yield "wait", ("pfree", (u - 3) & 3), (u - 3) >> 2
                    assert ("kv", n) in self.finished and ("q", g) in self.finished and (u < 3 or ("v", u - 3) in self.finished)
                    self.contract("s", ("s", u), [("sfull", u & 3)])

    def gradients(self):
        for n in range(len(self.items)):
            yield from self.read_item(n, "v")
            for g in self.tiles_of(n):
                for u in (2 * g, 2 * g + 1):
                    yield "wait", ("pready", u & 3), u >> 2
                    assert self.all_done("p", u)
                    if u == 2 * self.first[n] and n:
                        yield "wait", "accfree", n - 1
                        assert self.all_done("acc", n - 1)
                    yield "delay", self.delay("v")
                    last = u == 2 * self.first[n + 1] - 1
                    self.contract("v", ("v", u), [("pfree", u & 3)] + ([("qempty", g % self.STAGES)] if u & 1 else []) + (["accfull"] if last else []))

    def query_gradients(self):
        for n in range(len(self.items)):
            yield from self.read_item(n, "dq")
            for g in self.tiles_of(n):
                for u in (2 * g, 2 * g + 1):
                    yield "wait", ("pready", u & 3), u >> 2
                    assert self.all_done("p", u)
                if g:
                    yield "wait", "dqfree", g - 1
                    assert self.all_done("drained", g - 1)
                yield "delay", self.delay("dq")
                last = g == self.first[n + 1] - 1
                self.contract("dq", ("dq", g), [("dsfree", g & 1), "dqfull"] + ([("kvempty", n % self.slots)] if last else []))

    def arithmetic(self, h, warp):
        for n in range(len(self.items)):
            yield from self.read_item(n, ("p", h, warp))
            for g in self.tiles_of(n):
                u = 2 * g + h
                yield "wait", ("sfull", u & 3), u >> 2
                assert ("s", u) in self.finished
                yield "wait", ("dsfree", g & 1), (g >> 1) - 1
                assert g < 2 or ("dq", g - 2) in self.finished and all((*s, g - 2) in self.finished for s in self.sums), "dS in use"
                yield "delay", self.delay("soft")
                self.finished.add(("p", u, warp))
                self.arrive(("pready", u & 3))

    def bias_sums(self, h, sub):
        for n in range(len(self.items)):
            yield from self.read_item(n, ("sum", h, sub))
            for g in self.tiles_of(n):
                u = 2 * g + h
                yield "wait", ("pready", u & 3), u >> 2
                assert self.all_done("p", u)
                yield "delay", self.delay("sum")
                assert not any(("p", u + 4, w) in self.finished for w in self.WARPS), "dS overwritten"
                self.finished.add(("sum", h, sub, g))
                if self.fault != "sums":
                    self.arrive(("dsfree", g & 1))

    def drain(self, warp):
        for n in range(len(self.items)):
            yield from self.read_item(n, ("drain", warp))
            for g in self.tiles_of(n):
                if g == self.first[n + 1] - 1:
                    yield "wait", "accfull", n
                    assert ("v", 2 * g + 1) in self.finished and ("v", 2 * g + 2) not in self.issued
                    assert ("kv", n + self.slots) not in self.issued and (n == 0 or ("out", n - 1, warp) in self.finished)
                    yield "delay", self.delay("drain")
                    self.finished.add(("acc", n, warp))
                    self.arrive("accfree")
                    self.copy(("out", n, warp), ("group", warp))
                yield "wait", "dqfull", g
                assert ("dq", g) in self.finished and ("dq", g + 1) not in self.issued
                yield "delay", self.delay("drain")
                self.finished.add(("drained", g, warp))
                self.arrive("dqfree")
            yield "wait", ("group", warp), n
            assert ("kv", n + self.slots) not in self.issued, "the slot went before its rows had been read"
            if self.fault != "slot":
                self.arrive(("kvempty", n % self.slots))

    def run(self):
        self.go([self.producer(), self.scores(), self.gradients(), self.query_gradients()] + [self.arithmetic(h, w) for h in range(2) for w in self.WARPS] +
                [self.drain(w) for w in self.WARPS] + [self.bias_sums(h, sub) for h in range(2) for sub in range(2)])
        assert sum(f[0] == "drained" for f in self.finished) == 2 * self.first[-1], "the warps wait for one another"
        assert sum(f[0] == "sum" and len(f) == 4 for f in self.finished) == 4 * self.first[-1]


SHAPES = [[1], [1] * 40, [2, 1] * 20, [8, 8, 8], [3, 5, 2, 7, 1, 4] * 5, [1] * 19 + [6] + [1] * 18]


@pytest.mark.parametrize("items", SHAPES, ids=lambda s: f"{len(s)}x{s[0]}")
def test_forward(items):
    for seed in range(60):
        Forward(items, seed).run()


@pytest.mark.parametrize("slots", [2, 3, 4])
@pytest.mark.parametrize("items", SHAPES, ids=lambda s: f"{len(s)}x{s[0]}")
def test_backward(items, slots):
    for seed in range(60):
        Backward(items, seed, slots).run()


@pytest.mark.parametrize("fault", ["slot", "sums", "ring"])
def test_the_model_finds_a_rule_that_is_left_out(fault):
    """slot: V's slot is given back by the last dQ alone.  sums: a dS tile goes when dQ has read it.  ring: one eight of items instead of two."""
    found = 0
    for items in SHAPES:
        for seed in range(40):
            try:
                Backward(items, seed, 4, fault).run()
            except (AssertionError, WrongPhase):
                found += 1
    assert found


def test_the_model_finds_a_ring_of_one_eight_in_the_forward_pass():
    found = 0
    for items in SHAPES:
        for seed in range(40):
            model = Forward(items, seed)
            model.eights = 1
            try:
                model.run()
            except (AssertionError, WrongPhase):
                found += 1
    assert found
