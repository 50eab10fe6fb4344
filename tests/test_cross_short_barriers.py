"""The waits of the kernels for attention to short sequences of states (csrc/rib_cross_short_sm100.cu, csrc/rib_cross_short_bwd_sm100.cu) in the model of tests/test_frame_barriers.py: random delays, waits by parity, and a check that
each sees its own phase and that nothing is read or written out of turn.  `groups` are the tiles of a CTA's groups; those of negative groups have no keys.  No GPU needed."""
import pytest

from test_cross_barriers import Steps

SLOTS, WARPS = 4, 2


class Short(Steps):
    def __init__(self, groups, seed, ring):
        super().__init__([abs(g) for g in groups], seed, ring, 0)
        # of each tile: its group among those with keys (or None), and whether that group begins or ends with it
        self.tile, kvs = [], 0
        for g in groups:
            self.tile += [(kvs if g > 0 else None, i == 0 and g > 0, i == abs(g) - 1 and g > 0) for i in range(abs(g))]
            kvs += g > 0

    def products_of(self, kv, kind):
        return {(kind, t) for t, (k, _, _) in enumerate(self.tile) if k == kv}

    def producer(self):
        for t, (kv, first, _) in enumerate(self.tile):
            if first:
                if kv >= 2:
                    yield "wait", ("kvempty", kv & 1), (kv >> 1) - 1
                    assert self.products_of(kv - 2, "s") <= self.finished and self.products_of(kv - 2, "pv") <= self.finished
                self.copy(("kv", kv), ("kvfull", kv & 1))
            if t >= self.stages:
                yield "wait", ("qempty", t % self.stages), t // self.stages - 1
                assert ("s", t - self.stages) in self.finished
            self.copy(("q", t), ("qfull", t % self.stages))

    def scores(self):
        for t, (kv, first, _) in enumerate(self.tile):
            if first:
                yield "wait", ("kvfull", kv & 1), kv >> 1
            yield "wait", ("qfull", t % self.stages), t // self.stages
            if t >= SLOTS:
                yield "wait", ("free", t % SLOTS), t // SLOTS - 1
                assert all(("out", t - SLOTS, w) in self.finished for w in range(WARPS)) and ("pv", t - SLOTS) in self.finished
            assert kv is None or ("kv", kv) in self.finished and ("kv", kv + 2) not in self.issued
            yield "delay", self.delay("issue")
            self.contract("scores", ("s", t), [("sfull", t % SLOTS), ("qempty", t % self.stages)])

    def pv(self):
        for t, (kv, first, last) in enumerate(self.tile):
            if first:
                yield "wait", ("kvfull", kv & 1), kv >> 1
                yield "delay", self.delay("issue")       # values behind the last key
            yield "wait", ("ready", t % SLOTS), t // SLOTS
            assert all(("p", t, w) in self.finished for w in range(WARPS))
            assert kv is None or ("kv", kv) in self.finished and ("kv", kv + 2) not in self.issued
            yield "delay", self.delay("issue")
            self.contract("pv", ("pv", t), [("pvdone", t % SLOTS)] + ([("kvempty", kv & 1)] if last else []))

    def softmax(self, slot, w):
        for t in range(slot, len(self.tile), SLOTS):
            yield "wait", ("sfull", slot), t // SLOTS
            assert ("s", t) in self.finished and ("s", t + SLOTS) not in self.issued
            yield "delay", self.delay("soft")
            self.finished.add(("p", t, w))
            self.arrive(("ready", slot), WARPS)
            yield "wait", ("pvdone", slot), t // SLOTS
            assert ("pv", t) in self.finished
            yield "delay", self.delay("store")
            assert ("s", t + SLOTS) not in self.issued, "the output is overwritten before it is read"
            self.finished.add(("out", t, w))
            self.arrive(("free", slot), WARPS)

    def processes(self):
        return [self.producer(), self.scores(), self.pv()] + [self.softmax(s, w) for s in range(SLOTS) for w in range(WARPS)]

    def complete(self):
        assert len([f for f in self.finished if f[0] == "out"]) == WARPS * len(self.tile), "the warps wait for one another"


@pytest.mark.parametrize("groups", [[1], [-1], [20], [1] * 9, [2, 1, 3, -2, 1, 4], [-3, 5, -1, -1, 1, 1, 1, 12], [3] * 7], ids=str)
@pytest.mark.parametrize("ring", [4, 6])
def test_every_wait_sees_its_own_phase(ring, groups):
    for seed in range(200):
        Short(groups, seed, ring).run()


class Impatient(Short):
    """Scores that do not wait until the output before them is read."""

    def scores(self):
        for what in super().scores():
            if what[0] == "wait" and what[1][0] == "free" and self.rng.random() < 0.5:
                continue
            yield what


def test_the_model_finds_a_missing_wait():
    found = 0
    for seed in range(50):
        try:
            Impatient([9, 3], seed, 6).run()
        except AssertionError:
            found += 1
    assert found


class ShortBackward(Steps):
    """Unit u: row tile 2 (u / 2 / blocks) + (u mod 2), block (u / 2) mod blocks of keys.  Two arithmetic sets (WARPS warps each here) take the even and the odd tiles; two buffers of dS for pairs of tiles."""

    STAGES = 6

    def __init__(self, pairs, blocks, accs, seed):
        super().__init__([1], seed, 0, 0)
        self.third = blocks == 1 and accs == 2
        self.pairs, self.blocks, self.accs, self.units = pairs, blocks, accs, 2 * pairs * blocks

    def where(self, u):
        g, b = divmod(u >> 1, self.blocks)
        return 2 * g + (u & 1), b

    def units_of(self, tile):
        return [2 * (tile // 2 * self.blocks + b) + (tile & 1) for b in range(self.blocks)]

    def producer(self):
        self.copy("kv", "kvfull")
        for t in range(2 * self.pairs):
            if t >= self.STAGES:
                yield "wait", ("empty", t % self.STAGES), t // self.STAGES - 1
                assert all(("dk", u) in self.finished and ("s", u) in self.finished for u in self.units_of(t - self.STAGES))
            self.copy(("rows", t), ("full", t % self.STAGES))
        yield "wait", "kvfull", 0

    def statistics(self, h):
        for t in range(h, 2 * self.pairs, 2):
            yield "wait", ("full", t % self.STAGES), t // self.STAGES
            assert ("rows", t) in self.finished
            yield "delay", self.delay("store")
            assert t < self.STAGES or all(("read", u, w) in self.finished for u in self.units_of(t - self.STAGES) for w in range(WARPS))
            self.finished.add(("stats", t))
            self.arrive(("stats", t % self.STAGES))

    def scores(self):
        """S^T, then dP^T, of which there are three buffers as well, or two."""
        yield "wait", "kvfull", 0
        for u in range(self.units):
            t, b = self.where(u)
            if b == 0:
                yield "wait", ("full", t % self.STAGES), t // self.STAGES
            if u >= 3:
                yield "wait", ("pfree", u % 3), u // 3 - 1
                assert ("dv", u - 3) in self.finished
            assert ("rows", t) in self.finished and ("rows", t + self.STAGES) not in self.issued
            yield "delay", self.delay("issue")
            self.contract("scores", ("s", u), [])
            if not self.third and u >= 2:
                yield "wait", ("dpfree", u & 1), u // 2 - 1
            before = u - (3 if self.third else 2)
            assert before < 0 or all(("read", before, w) in self.finished for w in range(WARPS))
            self.contract("scores", ("dp", u), [("sfull", u % 6)])

    def keys(self):
        for u in range(self.units):
            t, b = self.where(u)
            yield "wait", ("ready", u % 6), u // 6
            assert all(("p", u, w) in self.finished for w in range(WARPS)) and ("s", u + 3) not in self.issued
            yield "delay", self.delay("issue")
            self.contract("keys", ("dv", u), [("pfree", u % 3)])
            self.contract("keys", ("dk", u), ([("dsfree", u >> 1 & 1)] if u & 1 else []) + ([("empty", t % self.STAGES)] if b == self.blocks - 1 else []) + (["accfull"] if u == self.units - 1 else []))

    def rows(self):
        for w in range(self.units // 2):
            g, b = divmod(w, self.blocks)
            for u in (2 * w, 2 * w + 1):
                yield "wait", ("ready", u % 6), u // 6
                assert all(("p", u, x) in self.finished for x in range(WARPS))
            if b == 0 and g >= self.accs:
                yield "wait", ("dqfree", g % self.accs), g // self.accs - 1
                assert all(("out", g - self.accs, x) in self.finished for x in range(4))
            yield "delay", self.delay("issue")
            self.contract("rows", ("dq", w), [("dsfree", w & 1)] + ([("dqfull", g % self.accs)] if b == self.blocks - 1 else []))

    def arithmetic(self, h, warp):
        for u in range(h, self.units, 2):
            t, b = self.where(u)
            w = u >> 1
            yield "wait", ("sfull", u % 6), u // 6
            assert ("s", u) in self.finished and ("dp", u) in self.finished
            if b == 0:
                yield "wait", ("stats", t % self.STAGES), t // self.STAGES
            assert ("stats", t) in self.finished and ("stats", t + self.STAGES) not in self.finished
            yield "delay", self.delay("soft")
            if w >= 2:
                yield "wait", ("dsfree", w & 1), w // 2 - 1
                assert ("dk", 2 * w - 3) in self.finished and ("dk", 2 * w - 4) in self.finished and ("dq", w - 2) in self.finished
            assert ("dp", u + (3 if self.third else 2)) not in self.issued
            self.finished.add(("read", u, warp))
            self.arrive(("dpfree", h))
            yield "delay", self.delay("soft")
            assert ("dq", w) not in self.issued and ("dk", u) not in self.issued
            self.finished.add(("p", u, warp))
            self.arrive(("ready", u % 6))
        yield "wait", "accfull", 0
        assert all(("dk", u) in self.finished for u in range(self.units))
        self.finished.add(("end", h, warp))

    def arrive(self, bar, count=1):
        super().arrive(bar, {"dpfree": WARPS, "ready": WARPS, "dsfree": 2, "dqfree": 4}.get(bar[0], count))

    def store(self, w):
        for g in range(self.pairs):
            yield "wait", ("dqfull", g % self.accs), g // self.accs
            assert ("dq", (g + 1) * self.blocks - 1) in self.finished and ("dq", (g + self.accs) * self.blocks) not in self.issued
            yield "delay", self.delay("store")
            assert ("dq", (g + self.accs) * self.blocks) not in self.issued, "a gradient is overwritten before it is read"
            self.finished.add(("out", g, w))
            self.arrive(("dqfree", g % self.accs))

    def processes(self):
        return [self.producer(), self.scores(), self.keys(), self.rows(), self.statistics(0), self.statistics(1)] + [self.arithmetic(h, w) for h in range(2) for w in range(WARPS)] + [self.store(w) for w in range(4)]

    def complete(self):
        assert len([f for f in self.finished if f[0] == "out"]) == 4 * self.pairs and len([f for f in self.finished if f[0] == "end"]) == 2 * WARPS, "the warps wait for one another"


@pytest.mark.parametrize("pairs", [1, 2, 3, 4, 5, 6, 7, 13])
@pytest.mark.parametrize("blocks,accs", [(1, 2), (2, 2), (1, 1)])
def test_every_wait_of_the_backward_pass_sees_its_own_phase(pairs, blocks, accs):
    for seed in range(100):
        ShortBackward(pairs, blocks, accs, seed).run()


class ImpatientBackward(ShortBackward):
    """dS written without a look at who reads what was there."""

    def arithmetic(self, h, warp):
        for what in super().arithmetic(h, warp):
            if what[0] == "wait" and what[1][0] == "dsfree" and self.rng.random() < 0.5:
                continue
            yield what


def test_the_model_of_the_backward_pass_finds_a_missing_wait():
    found = 0
    for seed in range(50):
        try:
            ImpatientBackward(9, 1, 2, seed).run()
        except AssertionError:
            found += 1
    assert found
