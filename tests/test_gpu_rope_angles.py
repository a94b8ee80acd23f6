"""Sine and cosine that a rotation uses, against exact fractions of a turn."""

import math
import random
from fractions import Fraction

import pytest
import torch

from paper_2608_09231_gb300 import bag

pytestmark = pytest.mark.gpu
DEV = "cuda"
TURN = Fraction("0.1591549430918953357688837633725143620344596457404564487476673440588967")  # 1 / (2 pi)
UNIT = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx(lib):
    c = bag.create("tiny", T=2, B=1)
    yield c
    c.close()


def turned(ctx, pos, freqs, **more):
    """(cos, sin) [rows, pairs] as (1, 0) becomes them, in float64 on the host."""
    n = len(freqs)
    x = torch.zeros(len(pos), 2 * n, device=DEV)
    x[:, :n] = 1.0
    y = torch.empty_like(x)
    ctx.rope(x, y, freqs, 2 * n, pos=torch.tensor(pos, device=DEV, dtype=torch.int32), **more)
    y = y.double().cpu()
    return y[:, :n], y[:, n:]


@pytest.mark.parametrize("inverse", [False, True])
def test_slow_pairs_at_near_positions(inverse, ctx):
    """Small angles keep their bits: the sine is off by 2^-65 turns a position (the frequency's rounding) and, of itself, by
    one rounding of the angle to 24 bits and sincospif's two units of at most 2^-23."""
    freqs = [1e-6, 1.5e-7, 3e-5, 1e-4, 7e-4, 1e-3, 2.0 ** -20, 1e-9]
    pos = [0, 1, 2, 3, 7, 19, 100, 501]
    _, sin = turned(ctx, pos, freqs, inverse=inverse)
    sign = -1.0 if inverse else 1.0
    for i, p in enumerate(pos):
        for j, f in enumerate(freqs):
            want = sign * math.sin(p * f)
            assert abs(float(sin[i, j]) - want) <= 5 * UNIT * abs(want) + p * 2 * math.pi * 2.0 ** -65, (p, f)


@pytest.mark.parametrize("inverse", [False, True])
def test_every_part_of_a_turn(inverse, ctx):
    """Angles all around, near and far: off by the frequency's rounding, an angle of at most an eighth of a turn rounded to
    24 bits, and two units of sincospif, which are at most 2^-24 each below 1."""
    rng = random.Random(5)
    freqs = [rng.uniform(0.1, 3.2) for _ in range(60)] + [math.pi / 2, math.pi, math.pi / 4, -1.0]
    pos = [rng.randrange(1 << rng.randrange(3, 31)) for _ in range(40)] + [0, 1, 2, 3, 4, 5, -1, -6, (1 << 31) - 1, -(1 << 31)]
    cos, sin = turned(ctx, pos, freqs, inverse=inverse)
    sign = -1.0 if inverse else 1.0
    for i, p in enumerate(pos):
        for j, f in enumerate(freqs):
            turn = 2 * math.pi * float(Fraction(f) * p * TURN % 1)
            tol = (math.pi / 4 + 2) * UNIT + abs(p) * 2 * math.pi * 2.0 ** -65 + 2.0 ** -50
            assert abs(float(cos[i, j]) - math.cos(turn)) <= tol, (p, f)
            assert abs(float(sin[i, j]) - sign * math.sin(turn)) <= tol, (p, f)
