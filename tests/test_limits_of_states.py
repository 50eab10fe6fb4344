"""The longest sequence of states that attention to them takes: positions are 32-bit numbers in the kernels, and each way in which they count on beyond the last state stays in range.
Sizes alone: the addresses are never read."""
import ctypes

import pytest

from paper_2603_06738_b200 import binding, build

MOST = 2 ** 31 - 4096
SMS = 148


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.library()


def call(lib, L, backward=False):
    at = [ctypes.c_void_p(1024 * (i + 1)) for i in range(9)]
    # q, k, v misaligned: a size that is taken is refused for that (-4), one that is not for itself (-3)
    q = ctypes.c_void_p(1024 + 8)
    shape = (1, 1, 1, 1, 1, 8, L, 1)
    if backward:
        return lib.rib_cross_attn_bwd(q, at[1], at[2], None, at[3], at[4], at[5], *shape, at[6], at[7], at[8], None, 0, None)
    return lib.rib_cross_attn_fwd(q, at[1], at[2], None, *shape, at[3], at[4], None, 0, None)


@pytest.mark.parametrize("backward", [False, True])
def test_the_longest_sequence(lib, backward):
    assert call(lib, MOST, backward) == -4
    for L in (MOST + 1, 2 ** 31 - 8 * SMS, 2 ** 31 - 256, 2 ** 31 - 1):
        assert call(lib, L, backward) == -3


@pytest.mark.parametrize("length", [MOST, MOST - 1, MOST - 8 * SMS, 2 ** 30, 1])
def test_runs_of_few_rows_stay_in_32_bits(length):
    """The arithmetic of a run of keys as the kernel for few rows has it, with the most runs that there are (eight to an SM)."""
    splits = 8 * SMS
    whole = lambda x: x if -2 ** 31 <= x < 2 ** 31 else pytest.fail(f"{x} passes 32 bits")  # noqa: E731
    run = whole(length + splits - 1) // splits
    covered = 0
    for split in range(splits):
        first = min(length, whole(split * run))
        last = min(length, whole(first + run))
        covered += last - first
        whole(last + 4 * 32 * 8)                 # the step beyond the last keys of a run, and keys that are not there
    assert covered == length
