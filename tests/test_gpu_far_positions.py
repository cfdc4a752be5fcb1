"""Angles of far positions: nothing is lost however many turns away a token lies, whatever the frequency.

Element pairs (1, 0) come out as (cos, sin).  What is left of the angle after whole turns is cut to 2^-32 turns and rounded to
single precision (2^-25 half turns: 1.6 u, u = 2^-24), the functions are off by 2 units in the last place (2 u) at most, products
with 1 and 0 by nothing: 4 u in all.  The product of position and frequency may add 2^31 * 2^-63 turns, far below u."""
import math
from decimal import Decimal, getcontext

import pytest
import torch

import paper_1911_00472_b200 as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
PI = "3.14159265358979323846264338327950288419716939937510582097494459230781640628620899"
FREQ = [1.0, 0.9999, 6.0, -6.1, 0.7071067811865476, 100.3, -1.0 / 3, 12345.678, 2.0 ** 40 + 1.0 / 3, 1e-3, -1e-9, 0.0, 77.77, 1e-20, -1e-20, 31.0]
POSITIONS = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, -1234567891, 1999999999, -2 ** 31 + 1, 1000003]


def exact():
    getcontext().prec = 110
    two_pi = 2 * Decimal(PI)
    got = []
    for p in POSITIONS:
        for f in FREQ:
            turns = Decimal(p) * Decimal(f) / two_pi
            left = float((turns - turns.to_integral_value()) * two_pi)
            got.append((math.cos(left), math.sin(left)))
    return torch.tensor(got, dtype=torch.float64, device="cuda").view(len(POSITIONS), len(FREQ), 2)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shift", [0, 1], ids=["whole vectors", "value by value"])
def test_angles_of_far_positions(shift, interleaved):
    n, half = len(POSITIONS), len(FREQ)
    pair = torch.tensor([1.0, 0.0], device="cuda")
    head = pair.repeat(half) if interleaved else pair.repeat_interleave(half)
    q = torch.zeros(2 * half * n + shift, device="cuda")[shift:].view(n, 1, 2 * half)
    q.copy_(head)
    positions = torch.tensor(POSITIONS, dtype=torch.int32, device="cuda")[None]
    inv_freq, axes = torch.tensor(FREQ, dtype=torch.float64, device="cuda"), torch.zeros(half, dtype=torch.int32, device="cuda")
    for inverse in (False, True):
        y = P.rotate(q, None, positions, inv_freq, axes, interleaved=interleaved, inverse=inverse)[0][:, 0].double()
        got = y.view(n, half, 2) if interleaved else y.view(n, 2, half).transpose(1, 2)
        want = exact()
        if inverse:
            want[..., 1].neg_()
        off = (got - want).abs() / U
        assert float(off.max()) <= 4, (float(off.max()), off.amax((0, 2)).tolist())
