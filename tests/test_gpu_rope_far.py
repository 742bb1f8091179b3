"""Angles of far positions against 60 digits: the whole range of positions, frequencies between the two that a long context
keeps and slows, in a ramp that is steep."""
import math
from decimal import Decimal, getcontext

import pytest
import torch

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


@pytest.fixture(scope="module")
def rs3():
    from paper_2608_22526_gb300 import rs3
    return rs3


def turns(n, base, factor, context, fast, slow):
    """Turns per position of n pairs, of the numbers in the description as they are."""
    getcontext().prec = 60
    out = []
    for i in range(n):
        f = (Decimal(base).ln() * -i / n).exp()
        g = Decimal(0)
        if context > 0:
            g = min(Decimal(1), max(Decimal(0), (Decimal(context) * f / (2 * PI) - Decimal(slow)) / (Decimal(fast) - Decimal(slow))))
        out.append(f * (g + (1 - g) / Decimal(factor)) / (2 * PI))
    return out


SPECS = [dict(rot=64, base=10000.0, factor=3.0), dict(rot=64, base=10000.0, factor=8.0, context=64.0), dict(rot=256, base=1e12),
         dict(rot=64, base=10000.0, factor=8.0, context=1e7, beta_slow=1.185e6, beta_fast=1.195e6),
         dict(rot=32, base=500000.0, factor=1e6, context=1e5, beta_slow=7000.0, beta_fast=7010.0), dict(rot=2, base=1.0), dict(rot=16, base=1.0, factor=7.0),
         dict(rot=16, base=100.0, factor=2.0, context=64.0, beta_slow=0.0, beta_fast=1e-310)]


@pytest.mark.parametrize("spec", SPECS)
@pytest.mark.parametrize("inverse", [False, True])
def test_an_angle_is_within_a_billionth_of_a_turn_anywhere(rs3, spec, inverse):
    pos = [0, 1, -1, 1000, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, -(2 ** 30) - 999, 123456789, -987654321]
    n, rot = spec["rot"] // 2, spec["rot"]
    f = turns(n, spec["base"], spec.get("factor", 1.0), spec.get("context", 0.0), spec.get("beta_fast", 32.0), spec.get("beta_slow", 1.0))
    want = torch.tensor([[[math.cos(a), -math.sin(a) if inverse else math.sin(a)] for a in (float((p * x) % 1 * 2 * PI) for x in f)] for p in pos],
                        dtype=torch.float64, device="cuda")
    s = rs3.rope_spec(inverse=inverse, **spec)
    at = torch.tensor(pos, device="cuda").to(torch.int32)
    table = torch.zeros((len(pos), n, 2), device="cuda")
    rs3.rs3_rope_table(at, s, table)
    # the angle, in radians; t = rest * step takes three roundings of |t| <= pi / 4 (2.4 half-steps), its sine or cosine 1.5
    # more of values up to 1, the magnitude one
    tol = 2 * math.pi * 2.0 ** -30 + 5 * STEP
    err = (table.double() - want).abs()
    assert (err <= tol).all(), float(err.max())
    # rows turned by the same angles: ones in the pairs' first elements
    x = torch.zeros((len(pos), rot), device="cuda")
    x[:, 0::2] = 1.0
    if rot % 4 == 0:
        y = torch.zeros_like(x)
        rs3.rs3_rope_rows(x, y, at, None, None, None, "f32", 1, 0, rot, s)
        err = (y.view(len(pos), n, 2).double() - want).abs()
        assert (err <= tol + 3 * STEP).all(), float(err.max())
