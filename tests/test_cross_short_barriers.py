"""The waits of the kernel for attention to short sequences of states (csrc/rib_cross_short_sm100.cu) in the model of tests/test_frame_barriers.py: random delays, waits by parity, and a check that
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
