"""The rotary plan against frequencies of 60 decimal digits: host only, no GPU."""
from decimal import Decimal, getcontext

import pytest

getcontext().prec = 60
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.fixture(scope="module")
def a2sf():
    from paper_2407_20485_b200 import build

    build.build()
    from paper_2407_20485_b200 import binding

    return binding


def frequencies(r, theta, scaling, factor, L, low, high, between):
    """f_k by the header's definition; RAMP takes its two pair indexes, which are whole numbers, from ``between``."""
    theta, factor, L, low, high = (Decimal(x) for x in (theta, factor, L, low, high))
    if scaling == "ntk":
        theta *= (factor.ln() * r / (r - 2)).exp()
    for k in range(r // 2):
        f = (-theta.ln() * 2 * k / r).exp()
        keep = Decimal(1)
        if scaling == "linear":
            keep = Decimal(0)
        elif scaling == "bands":
            keep = (L * f / (2 * PI) - low) / (high - low)
        elif scaling == "ramp":
            keep = 1 - (k - Decimal(between[0])) / Decimal(between[1] - between[0])
        keep = min(max(keep, Decimal(0)), Decimal(1))
        yield keep * f + (1 - keep) * f / factor


@pytest.mark.parametrize("scaling,factor,high,between", [
    ("none", 1, 4, None), ("linear", 4, 4, None), ("linear", 3, 4, None), ("ntk", 3, 4, None), ("bands", 8, 4, None), ("ramp", 16, 32, (0, 0))])
@pytest.mark.parametrize("r,theta", [(126, 10000), (128, 500000), (128, 1000000), (64, 10000), (24, 500000)])
def test_angles_of_the_farthest_positions(a2sf, r, theta, scaling, factor, high, between):
    """A turn per position is a 64-bit fraction: off by 2^-62 at most, cutting included, so that 2^31 positions make 2^-31 of a
    turn, 3e-9 of an angle."""
    if scaling == "ramp":
        at = [r * (Decimal(8192) / (beta * 2 * PI)).ln() / (2 * Decimal(theta).ln()) for beta in (high, 1)]
        between = (int(at[0]), int(at[1]) + 1)                   # both are positive and no whole numbers
    plan = a2sf.a2sf_rotary_plan_init(r, theta=float(theta), scaling=scaling, factor=float(factor), original_length=8192, low=1.0,
                                      high=float(high))
    worst = max(abs(Decimal(plan.turn[k]) - f / (2 * PI) * 2 ** 64)
                for k, f in enumerate(frequencies(r, theta, scaling, factor, 8192, 1, high, between)))
    assert worst <= 4, f"{float(worst):.3g} of 2^-64"
