"""The waits of the kernels for attention to states (csrc/rib_cross_fwd_sm100.cu, csrc/rib_cross_bwd_sm100.cu) in the model of tests/test_frame_barriers.py: random
delays, waits by parity, and a check that each sees its own phase and that nothing is read or written out of turn.  `items` are the key blocks (or row tiles) of a CTA's items; items without
any are no steps and are left out.  No GPU needed."""
import heapq

import pytest

from test_frame_barriers import Model


class Steps(Model):
    BUFFERS = 3

    def __init__(self, items, seed, stages, tiles):
        super().__init__(items, seed, True)
        self.stages, self.tiles = stages, tiles
        self.scale.update({name: self.rng.choice((0.1, 1.0, 5.0)) for name in ("load", "issue", "store")})
        self.first = [sum(items[:n]) for n in range(len(items))]
        self.steps = sum(items)

    def copy(self, what, bar):
        self.issued.add(what)

        def complete():
            self.finished.add(what)
            self.arrive(bar)
        self.later(self.delay("load"), complete)

    def run(self):
        self.pipe = {}
        for process in self.processes():
            self.later(self.delay("soft"), lambda process=process: self.step(process))
        while self.queue:
            self.now, _, what = heapq.heappop(self.queue)
            what()
        assert len([f for f in self.finished if f[0] == "last"]) == self.steps, "the warps wait for one another"
        assert len([f for f in self.finished if f[0] == "out"]) == 4 * len(self.items), "outputs are missing"


class Forward(Steps):
    """One warp loads and issues all products; four warps have the exponentials, and an item's output behind those of the next item's first block."""

    def control(self):
        n_of = [n for n, blocks in enumerate(self.items) for _ in range(blocks)]
        loads, scores = 0, 0

        def load_ahead(value, scored):
            nonlocal loads
            while loads < self.steps:
                n = n_of[loads]
                if loads == value + self.stages or (loads == self.first[n] and n == scored + self.tiles):
                    return
                if loads == self.first[n]:
                    assert n < self.tiles or all(("s", u) in self.finished for u in range(self.first[n - self.tiles], self.first[n - self.tiles] + self.items[n - self.tiles]))
                    self.copy(("q", n), ("qfull", n % self.tiles))
                assert loads < self.stages or ("last", loads - self.stages) in self.finished
                self.copy(("k", loads), ("kfull", loads % self.stages))
                loads += 1

        def issue():
            nonlocal scores
            n = n_of[scores]
            if scores == self.first[n]:
                yield "wait", ("qfull", n % self.tiles), n // self.tiles
            yield "wait", ("kfull", scores % self.stages), scores // self.stages
            assert scores < self.BUFFERS or ("last", scores - self.BUFFERS) in self.finished
            self.contract("tensor", ("s", scores), [("sfull", scores % self.BUFFERS)])
            scores += 1

        load_ahead(0, 0)
        for _ in range(self.BUFFERS):
            if scores < self.steps:
                yield from issue()
        for u in range(self.steps):
            yield "wait", ("ready", u % self.BUFFERS), u // self.BUFFERS
            yield "delay", self.delay("issue")
            assert all(("p", u, w) in self.finished for w in range(4))
            self.contract("tensor", ("last", u), [("pvdone", u % self.BUFFERS)])
            if u:
                yield "wait", ("pvdone", (u - 1) % self.BUFFERS), (u - 1) // self.BUFFERS
            n = n_of[u]
            load_ahead(u, n + (1 if u + 1 == self.first[n] + self.items[n] else 0))
            if u and scores < self.steps:
                yield from issue()

    def softmax(self, w):
        u = 0

        def output(n):
            last = self.first[n] + self.items[n] - 1
            yield "wait", ("pvdone", last % self.BUFFERS), last // self.BUFFERS
            assert ("last", last) in self.finished and ("last", last + 1) not in self.issued
            yield "delay", self.delay("store")
            assert ("last", last + 1) not in self.issued, "the output is overwritten before it is read"
            self.finished.add(("out", n, w))

        for n, blocks in enumerate(self.items):
            for j in range(blocks):
                yield "wait", ("sfull", u % self.BUFFERS), u // self.BUFFERS
                assert ("s", u) in self.finished
                yield "delay", self.delay("soft")
                if j and self.rng.random() < 0.3:       # the maximum grew
                    yield "wait", ("pvdone", (u - 1) % self.BUFFERS), (u - 1) // self.BUFFERS
                    assert ("last", u - 1) in self.finished and ("last", u) not in self.issued
                if j == 0 and n:
                    yield from output(n - 1)
                self.finished.add(("p", u, w))
                self.arrive(("ready", u % self.BUFFERS), 4)
                u += 1
        yield from output(len(self.items) - 1)

    def processes(self):
        return [self.control()] + [self.softmax(w) for w in range(4)]


class Dq(Steps):
    """Loads, scores and dQ in a warp each; three sets of four warps take the steps in turn; four warps store dQ, of which there are two accumulators."""
    BUFFERS = 3

    def producer(self):
        u = 0
        for n, blocks in enumerate(self.items):
            if n >= self.tiles:
                yield "wait", ("qempty", n % self.tiles), n // self.tiles - 1
                assert all(("arith", v) in self.finished for v in range(self.first[n - self.tiles], self.first[n - self.tiles] + self.items[n - self.tiles]))
            self.copy(("q", n), ("qfull", n % self.tiles))
            for _ in range(blocks):
                if u >= self.stages:
                    yield "wait", ("kempty", u % self.stages), u // self.stages - 1
                    assert ("last", u - self.stages) in self.finished
                self.copy(("k", u), ("kfull", u % self.stages))
                u += 1

    def scores(self):
        u = 0
        for n, blocks in enumerate(self.items):
            yield "wait", ("qfull", n % self.tiles), n // self.tiles
            for _ in range(blocks):
                yield "wait", ("kfull", u % self.stages), u // self.stages
                if u >= self.BUFFERS:
                    yield "wait", ("free", u % self.BUFFERS), u // self.BUFFERS - 1
                    assert ("last", u - self.BUFFERS) in self.finished
                yield "delay", self.delay("issue")
                self.contract("scores", ("s", u), [("sfull", u % self.BUFFERS)])
                u += 1

    def products(self):
        u = 0
        for n, blocks in enumerate(self.items):
            for j in range(blocks):
                yield "wait", ("ready", u % self.BUFFERS), u // self.BUFFERS
                if j == 0 and n >= 2:
                    yield "wait", ("accfree", n & 1), n // 2 - 1
                    assert all(("out", n - 2, w) in self.finished for w in range(4))
                yield "delay", self.delay("issue")
                bars = [("free", u % self.BUFFERS), ("kempty", u % self.stages)]
                if j == blocks - 1:
                    bars += [("accfull", n & 1), ("qempty", n % self.tiles)]
                self.contract("products", ("last", u), bars)
                u += 1

    def arithmetic(self, which, w):
        n_of = [n for n, blocks in enumerate(self.items) for _ in range(blocks)]
        for u in range(which, self.steps, self.BUFFERS):
            yield "wait", ("sfull", which), u // self.BUFFERS
            yield "wait", ("kfull", u % self.stages), u // self.stages
            yield "wait", ("qfull", n_of[u] % self.tiles), n_of[u] // self.tiles
            assert ("s", u) in self.finished
            yield "delay", self.delay("soft")
            self.finished.add(("w", u, w))
            if all(("w", u, x) in self.finished for x in range(4)):
                self.finished.add(("arith", u))
            self.arrive(("ready", which), 4)

    def store(self, w):
        for n in range(len(self.items)):
            yield "wait", ("accfull", n & 1), n // 2
            assert ("last", self.first[n] + self.items[n] - 1) in self.finished and (n + 2 >= len(self.items) or ("last", self.first[n + 2]) not in self.issued)
            yield "delay", self.delay("store")
            self.finished.add(("out", n, w))
            self.arrive(("accfree", n & 1), 4)

    def processes(self):
        return [self.producer(), self.scores(), self.products()] + [self.arithmetic(s, w) for s in range(3) for w in range(4)] + [self.store(w) for w in range(4)]


class Dkv(Dq):
    """One item: its row tiles are the steps, and what waits for the accumulators reads them at the end."""

    def producer(self):
        self.copy(("q", 0), ("qfull", 0))
        for u in range(self.steps):
            if u >= self.stages:
                yield "wait", ("kempty", u % self.stages), u // self.stages - 1
                assert ("last", u - self.stages) in self.finished
            self.copy(("k", u), ("kfull", u % self.stages))

    def arithmetic(self, which, w):
        for u in range(which, self.steps, self.BUFFERS):
            yield "wait", ("sfull", which), u // self.BUFFERS
            yield "wait", ("kfull", u % self.stages), u // self.stages
            assert ("s", u) in self.finished
            yield "delay", self.delay("soft")
            self.finished.add(("w", u, w))
            self.arrive(("ready", which), 4)


SHAPES = [[1], [1, 1, 1, 1, 1, 1, 1, 1, 1], [2] * 9, [2, 1, 3, 1, 1, 4], [12, 12], [1, 7, 1, 1, 1, 9, 2, 2]]


@pytest.mark.parametrize("items", SHAPES, ids=str)
@pytest.mark.parametrize("kind,stages,tiles", [(Forward, 8, 4), (Forward, 4, 3), (Dq, 8, 4), (Dq, 6, 3)])
def test_every_wait_sees_its_own_phase(kind, stages, tiles, items):
    for seed in range(200):
        kind(items, seed, stages, tiles).run()


@pytest.mark.parametrize("tiles", [1, 2, 3, 4, 6, 7, 40])
def test_every_wait_sees_its_own_phase_along_the_rows(tiles):
    for seed in range(200):
        Dkv([tiles], seed, 6, 1).run()


def test_the_model_finds_too_few_tiles_of_rows():
    """Scores of three items of one block each are taken before the first product: with two tiles of rows the warps wait for one another."""
    with pytest.raises(AssertionError):
        Forward([1] * 9, 0, 8, 2).run()
