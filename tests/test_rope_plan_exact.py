"""The rotary plan's steps to the last bits (no GPU): a frequency's error is multiplied by the position."""

import math
from decimal import Decimal, getcontext

import pytest

from paper_2605_01910_amd import santa as S

getcontext().prec = 60
PI2 = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494")


@pytest.mark.parametrize("theta", [10000.0, 500000.0, 1.1])
@pytest.mark.parametrize("R", [16, 32, 96, 128])
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "bands", "ramp"])
def test_steps(scaling, R, theta):
    """Within 16 units of 2^-64 of a turn: the power's exponent is off by 2^-64 of itself, at most 14
    (ln theta) times that of f, and f is at most 1 / (2 pi) of a turn; a handful of other roundings."""
    factor, N, lo, hi = 8.0, 8192.0, 1.0, 4.0
    plan = S.rope_plan(R, False, theta, scaling, factor, N, lo, hi)
    th, fa = Decimal(theta), Decimal(factor)
    if scaling == "base":
        th *= fa ** (Decimal(R) / (R - 2))
    for i in range(R // 2):
        f = th ** (Decimal(-2 * i) / R)
        if scaling == "linear":
            f /= fa
        elif scaling == "bands":
            keep = min(Decimal(1), max(Decimal(0), (Decimal(N) * f / PI2 - Decimal(lo)) / Decimal(hi - lo)))
            f = f * keep + f / fa * (1 - keep)
        elif scaling == "ramp":
            at = [Decimal(R) * (Decimal(N) / (PI2 * Decimal(t))).ln() / (2 * th.ln()) for t in (hi, lo)]
            a, b = max(0, math.floor(at[0])), min(R - 1, math.ceil(at[1]))
            mix = min(Decimal(1), max(Decimal(0), Decimal(i - a) / max(Decimal(b - a), Decimal("0.001"))))
            f = f / fa * mix + f * (1 - mix)
        assert abs(plan.step[i] - (f / PI2 % 1) * 2 ** 64) <= 16, i
