"""Angles of the rotation's table at places as far as the calls take, against whole-number arithmetic: an entry is rounded to 32 bits, at most 2^-25 of 1, from a sine or cosine
whose own error and that of its angle are below 2^-40."""
from fractions import Fraction
import math
import struct

import pytest
import torch

from paper_2603_06738_b200 import binding as rib

pytestmark = pytest.mark.gpu


def arctan_of_inverse(n, digits):
    """arctan(1 / n), n whole, by its series."""
    total, power, k = 0, 10 ** digits // n, 0
    while power:
        total += (-1) ** k * (power // (2 * k + 1))
        power //= n * n
        k += 1
    return Fraction(total, 10 ** digits)


TURN = 8 * (4 * arctan_of_inverse(5, 80) - arctan_of_inverse(239, 80))        # 2 pi: Machin's formula, 78 digits


def cosine_and_sine(position, frequency):
    """Of a whole number times an fp32 number."""
    angle = position * Fraction(frequency)                                     # exact
    angle -= TURN * round(angle / TURN)
    return math.cos(float(angle)), math.sin(float(angle))


@pytest.mark.parametrize("far", [0, 2 ** 28 + 3, 2 ** 29 + 1, 2 ** 33 + 7, -(2 ** 36) - 5, 2 ** 40 - 11, 2 ** 40, -(2 ** 40)])
def test_angles_of_far_places(far):
    frequencies = torch.stack([rib.rib_rope_frequencies(32, sequence=True)[0], 0.1 + torch.rand(16, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) * 900]).contiguous()
    H, W = 9, 5
    table = rib.rib_rope_table(frequencies, H, W, y0=far, x0=far).cpu().double()
    worst = 0.0
    for row in range(H + W):
        for i in range(16):
            f = frequencies[0 if row < H else 1, i].item()
            want = cosine_and_sine(far + (row if row < H else row - H), struct.unpack("f", struct.pack("f", f))[0])
            worst = max(worst, abs(table[row, i, 0].item() - want[0]), abs(table[row, i, 1].item() - want[1]))
    assert worst <= 2.0 ** -25 + 2.0 ** -40
