"""Angles of the rotation at positions of all sizes, against frequencies of 60 decimal digits."""
import math
import random
from decimal import Decimal

import pytest
import torch

from test_rotary_plan import PI, frequencies

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def a2sf():
    from paper_2407_20485_b200 import binding

    return binding


@pytest.mark.parametrize("r,theta,transpose", [(128, 1000000, False), (126, 10000, True), (64, 500000, False)])
def test_cosines_and_sines_at_all_positions(a2sf, r, theta, transpose):
    """Rows that are 1 in a pair's first element turn into its cosine and sine: off by the angle's 3e-8 and the functions' last
    place (2^-24 below 1)."""
    rng = random.Random(r)
    pos = [0, 1, 2 ** 31 - 1, 2 ** 30, 2 ** 31 - 2 ** 20, -1, -2 ** 31] + [int(2 ** rng.uniform(1, 31)) for _ in range(400)]
    d, n = 128, len(pos)
    x = torch.zeros((1, 1, n, d), device="cuda")
    x[..., : r // 2] = 1.0
    plan = a2sf.a2sf_rotary_plan_init(r, theta=float(theta))
    y = a2sf.a2sf_rotary(plan, x, positions=torch.tensor([pos], dtype=torch.int32).cuda(), transpose=transpose).cpu()[0, 0].double()
    turns = [f / (2 * PI) for f in frequencies(r, theta, "none", 1, 1, 1, 4, None)]
    angle = torch.tensor([[float((t * p) % 1 * 2 * PI) for t in turns] for p in map(Decimal, pos)], dtype=torch.float64)
    sign = -1.0 if transpose else 1.0
    worst = max(float((y[:, : r // 2] - torch.cos(angle)).abs().max()), float((y[:, r // 2: r] - sign * torch.sin(angle)).abs().max()))
    assert worst <= 3e-8 + 2.0 ** -24, f"{worst:.3g}"
    # a turn keeps lengths, whatever the quarter
    assert float((y[:, : r // 2] ** 2 + y[:, r // 2: r] ** 2 - 1).abs().max()) <= 4 * math.sqrt(2) * 2.0 ** -24
