"""Rotary angles at far positions, against angles reduced exactly."""
import math
from fractions import Fraction

import pytest
import torch

import paper_2510_22641_gb300 as lib
from tests.test_gpu_rows import normal

pytestmark = pytest.mark.gpu

# to 59 digits
PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494")


def root8(v: int, digits: int = 60) -> Fraction:
    """v^(1/8) to 10^-digits, by three integer square roots."""
    scale = 10 ** (8 * digits)
    return Fraction(math.isqrt(math.isqrt(math.isqrt(v * scale))), 10 ** digits)


@pytest.mark.parametrize("pos", [0, 1, -1, 4097, 131071, 1 << 24, 2 ** 31 - 1, -2 ** 31])
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_keep_their_angles(pos, interleaved):
    """theta 1e4 over 32 pairs: frequencies 10^(-i / 8).  A step is a double, computed in doubles, so an angle is within
    |pos| 2^-52 of a radian, plus 2^-29 for its 32 bits; sines of it to 2^-23 and three roundings make 2^-21 of the pair."""
    dim = 64
    x = normal((1, 2, dim), 1)
    y, _ = lib.Rotary(dim, theta=1e4, interleaved=interleaved).rotate(x, None, torch.tensor([pos], dtype=torch.int32, device="cuda"))
    for i in range(dim // 2):
        turn = Fraction(pos) / root8(10 ** i)
        rest = float(turn - 2 * PI * round(turn / (2 * PI)))
        c, s = math.cos(rest), math.sin(rest)
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + dim // 2)
        a, b = x[0, :, p].double(), x[0, :, q].double()
        bound = (2.0 ** -21 + abs(pos) * 2.0 ** -52) * (a.abs() + b.abs())
        assert ((y[0, :, p].double() - (a * c - b * s)).abs() <= bound).all(), i
        assert ((y[0, :, q].double() - (b * c + a * s)).abs() <= bound).all(), i
