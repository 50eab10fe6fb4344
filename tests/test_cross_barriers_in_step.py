"""The waits of the forward pass of the attention to states when both tiles begin at once, whatever the number of blocks: the scores of the second tile wait for nothing of the first."""
import pytest

from test_cross_barriers import SHAPES, Forward


class InStep(Forward):
    def scores(self):
        for what in super().scores():
            if what != ("wait", ("ready", 0, 0), 0):
                yield what


@pytest.mark.parametrize("items", [*SHAPES, [4], [16], [5, 4, 8, 16]], ids=str)
@pytest.mark.parametrize("stages", [3, 4])
def test_every_wait_sees_its_own_phase(items, stages):
    for seed in range(200):
        InStep(items, seed, stages, 2).run()
