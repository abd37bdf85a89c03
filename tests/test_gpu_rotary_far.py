"""Rotary positions at the largest frequencies and positions (fsx_rotary_rows), against angles from exact rationals.

Tolerance as in test_gpu_rotary.py: with u = 2^-24, 6 u (|x_a| + |x_b|) and half a step of the output's type.  The angle's place in
its turn may be off by 2^-32 turns and the rounding of the frequency's fraction of a turn (2^-65, times a position of 2^31 at most:
2^-34 turns), 0.03 u together, which those 6 u hold.  The reference's place is exact to 2^-52."""

from __future__ import annotations

from decimal import Decimal, getcontext
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2607_15621_amd import fsx

pytestmark = pytest.mark.gpu


def two_pi():
    """2 pi to 90 digits: Machin, pi / 4 = 4 atan(1/5) - atan(1/239)."""
    getcontext().prec = 100

    def atan(n):
        total, term, i = Decimal(0), Decimal(1) / n, 0
        while abs(term) > Decimal(10) ** -98:
            total += term / (2 * i + 1) * (-1) ** i
            term /= n * n
            i += 1
        return total
    return Fraction(8 * (4 * atan(5) - atan(239)))


TURN = two_pi()
FREQS = [2.0 ** 20, 2.0 ** 20 - 0.37, 987654.321, -777777.7, 12345.678, 1000.0 / 3, 10.0, 1.0, 0.1, -2.0 ** -30 * 1.7]
POSITIONS = [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 12345, -1999999999, 1 << 30, 123456789, 16001, 1, 0]


@pytest.mark.parametrize("layout", [fsx.ROTARY_HALVES, fsx.ROTARY_ADJACENT], ids=["halves", "adjacent"])
def test_far_positions_at_high_frequencies(layout):
    n, R = len(FREQS), len(POSITIONS)
    g = torch.Generator().manual_seed(5)
    x = torch.randn(R, 3, 2 * n, generator=g)
    out = torch.empty_like(x, device="cuda")
    plan = fsx.RotaryPlan([0] * n, FREQS, layout)
    fsx.rotary_rows(x.cuda(), out, torch.tensor([POSITIONS], dtype=torch.int32, device="cuda"), plan)
    angle = np.array([[float((Fraction(p) * Fraction(f) / TURN) % 1) * 2 * np.pi for f in FREQS] for p in POSITIONS])
    c, s = (torch.from_numpy(f(angle))[:, None] for f in (np.cos, np.sin))
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if layout == fsx.ROTARY_ADJACENT else (slice(0, n), slice(n, 2 * n))
    y, xd, got = torch.empty_like(x, dtype=torch.float64), x.double(), out.cpu().double()
    y[..., a], y[..., b] = xd[..., a] * c - xd[..., b] * s, xd[..., b] * c + xd[..., a] * s
    tol = torch.empty_like(y)
    tol[..., a] = tol[..., b] = 6 * 2.0 ** -24 * (xd[..., a].abs() + xd[..., b].abs())
    tol += 2.0 ** -24 * (y.abs() + tol)
    worst = ((got - y).abs() / tol).amax((0, 1))
    assert bool(((got - y).abs() <= tol).all()), worst
