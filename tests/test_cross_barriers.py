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
        self.complete()

    def complete(self):
        assert len([f for f in self.finished if f[0] == "last"]) == self.steps, "the warps wait for one another"
        assert len([f for f in self.finished if f[0] == "out"]) == 4 * len(self.items), "outputs are missing"


class Forward(Steps):
    """Two tiles of rows; unit 2 block + tile has its scores, and P over them, in buffer unit mod 3.  Two warps, one for each half of the keys, own a row: they meet once a
    block, and store an item's output behind the exponentials of the next item's first block.  (One quarter of the rows: the others are alike.)"""

    def producer(self):
        u = 0
        for n, blocks in enumerate(self.items):
            if n >= 2:
                yield "wait", ("qempty", n & 1), n // 2 - 1
                assert all(("s", 2 * v + 1) in self.finished for v in range(self.first[n - 2], self.first[n - 2] + self.items[n - 2]))
            self.copy(("q", n), ("qfull", n & 1))
            for _ in range(blocks):
                for x in "kv":
                    if u >= self.stages:
                        yield "wait", (x + "empty", u % self.stages), u // self.stages - 1
                        old = 2 * (u - self.stages)
                        assert all(({"k": "s", "v": "pv"}[x], old + t) in self.finished for t in range(2))
                    self.copy((x, u), (x + "full", u % self.stages))
                u += 1

    def arrive(self, bar, count=1):
        super().arrive(bar, {"vempty": 2, "ready": 2, "pair": 2}.get(bar[0], count))

    def scores(self):
        u = 0
        for n, blocks in enumerate(self.items):
            yield "wait", ("qfull", n & 1), n // 2
            for j in range(blocks):
                yield "wait", ("kfull", u % self.stages), u // self.stages
                for t in range(2):
                    if t and u == 0 and blocks >= 4:
                        yield "wait", ("ready", 0, 0), 0
                    yield ("wait", *self.pv_phase(1 - t, (2 * u + t - 3) >> 1))
                    assert 2 * u + t < self.BUFFERS or ("pv", 2 * u + t - self.BUFFERS) in self.finished
                    bars = [self.score_phase(t, u)[0]]
                    if t:
                        bars += [("kempty", u % self.stages)] + ([("qempty", n & 1)] if j == blocks - 1 else [])
                    yield "delay", self.delay("issue")
                    self.contract("s", ("s", 2 * u + t), bars)
                u += 1

    def pv(self, t):
        for u in range(self.steps):
            yield "wait", ("vfull", u % self.stages), u // self.stages
            yield "wait", ("ready", t, u & 1), u // 2
            assert all(("p", 2 * u + t, half) in self.finished for half in range(2))
            yield "delay", self.delay("issue")
            self.contract(f"pv{t}", ("pv", 2 * u + t), [self.pv_phase(t, u)[0], ("vempty", u % self.stages)])

    def softmax(self, t, half):
        u, met = 0, 0

        def meet(what):
            nonlocal met
            self.finished.add(("told", t, half, what))
            self.arrive(("pair", t))
            yield "wait", ("pair", t), met
            met += 1
            assert ("told", t, 1 - half, what) in self.finished

        def output(n):
            last = self.first[n] + self.items[n] - 1
            yield ("wait", *self.pv_phase(t, last))
            assert ("pv", 2 * last + t) in self.finished and ("pv", 2 * last + 2 + t) not in self.issued
            assert ("sum", t, 1 - half, n) in self.finished and ("sum", t, 1 - half, n + 2) not in self.finished
            yield "delay", self.delay("store")
            assert ("pv", 2 * last + 2 + t) not in self.issued, "the output is overwritten before it is read"
            assert ("sum", t, 1 - half, n + 2) not in self.finished, "a sum is overwritten before it is read"
            self.finished.add(("out", n, t, half))

        for n, blocks in enumerate(self.items):
            for j in range(blocks):
                yield ("wait", *self.score_phase(t, u))
                assert ("s", 2 * u + t) in self.finished
                yield "delay", self.delay("soft")
                assert ("told", t, half, u - 2) not in self.finished or ("heard", t, 1 - half, u - 2) in self.finished, "a maximum is overwritten before it is read"
                yield from meet(u)
                yield "delay", self.delay("soft")
                self.finished.add(("heard", t, half, u))
                if j and (n + j) % 3 == 0:               # the maximum grew
                    yield ("wait", *self.pv_phase(t, u - 1))
                    assert ("pv", 2 * u - 2 + t) in self.finished and ("pv", 2 * u + t) not in self.issued
                if j == 0 and n:
                    yield from output(n - 1)
                self.finished.add(("p", 2 * u + t, half))
                self.arrive(("ready", t, u & 1))
                u += 1
            self.finished.add(("sum", t, half, n))
        yield from meet("end")
        yield from output(len(self.items) - 1)

    def processes(self):
        return [self.producer(), self.scores(), self.pv(0), self.pv(1)] + [self.softmax(t, half) for t in range(2) for half in range(2)]

    def complete(self):
        assert len([f for f in self.finished if f[0] == "pv"]) == 2 * self.steps, "the warps wait for one another"
        assert len([f for f in self.finished if f[0] == "out"]) == 4 * len(self.items), "outputs are missing"


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
@pytest.mark.parametrize("kind,stages,tiles", [(Forward, 4, 2), (Forward, 3, 2), (Dq, 8, 4), (Dq, 6, 3)])
def test_every_wait_sees_its_own_phase(kind, stages, tiles, items):
    for seed in range(200):
        kind(items, seed, stages, tiles).run()


@pytest.mark.parametrize("tiles", [1, 2, 3, 4, 6, 7, 40])
def test_every_wait_sees_its_own_phase_along_the_rows(tiles):
    for seed in range(200):
        Dkv([tiles], seed, 6, 1).run()


class Impatient(Forward):
    """P handed over before the output of the item before is read."""

    def softmax(self, t, half):
        for what in super().softmax(t, half):
            if what[0] == "wait" and what[1][0] == "pv" and self.rng.random() < 0.5:
                continue
            yield what


def test_the_model_finds_a_missing_wait():
    found = 0
    for seed in range(50):
        try:
            Impatient([1, 2, 1, 1, 3], seed, 4, 2).run()
        except AssertionError:
            found += 1
    assert found
