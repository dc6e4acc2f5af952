"""Angles of the rotation of queries and keys at the farthest positions, against products of whole numbers.

A result of unit pairs is cos t -+ sin t in binary32: sincospif is within two units in the last place, which is 2^-24 at most below 1; turning on by what its
binary32 argument has left is one rounding, half of that; the angle itself is off by 2^-50.  So cos and sin are within 3 * 2^-24, at every position."""
import math
from decimal import Decimal, getcontext
from fractions import Fraction

import pytest
import torch

from paper_2501_09767_amd import lemo

PI = Fraction(Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798"))
BOUND = 3 * 2.0 ** -24


def turns(position, freq):
    """What is left of position * freq after whole turns, as an angle, exactly but for the last rounding."""
    getcontext().prec = 60
    angle = Fraction(position) * Fraction(freq)
    return float(angle - 2 * PI * round(angle / (2 * PI)))


def places(far):
    g = torch.Generator().manual_seed(far % 1000)
    pos = torch.randint(-far, far, (60,), generator=g).tolist()
    return [far - 1, -far + 1, far - 2, 0, 1, -1, *pos]


def frequencies(n):
    g = torch.Generator().manual_seed(n)
    return torch.cat([torch.tensor([1.0, 0.1, 3.0, 500000.0 ** -0.5]), torch.rand(n - 4, generator=g)]).float()


def test_the_reference():
    assert turns(0, 1.0) == 0 and abs(turns(22, 1.0) - (22 - 8 * math.pi)) < 1e-14
    for p in (1, 355, 10 ** 6, -(2 ** 31) + 1):  # whole angles, which the host's cos reduces exactly
        assert abs(math.cos(turns(p, 1.0)) - math.cos(p)) < 1e-14 and abs(math.sin(turns(p, 1.0)) - math.sin(p)) < 1e-14


@pytest.mark.gpu
@pytest.mark.parametrize("far, start", [(2 ** 17, 0), (2 ** 31, 0), (2 ** 31, 2 ** 31 - 1), (2 ** 31, 1 - 2 ** 31)])
@pytest.mark.parametrize("pairs", [False, True])
def test_far_positions_are_as_exact_as_near_ones(far, start, pairs):
    pos, f = places(far), frequencies(32)
    M, d = len(pos), 64
    a = torch.arange(32)
    first, second = (2 * a, 2 * a + 1) if pairs else (a, a + 32)
    angle = torch.tensor([[turns(p + start, x) for x in f.tolist()] for p in pos], dtype=torch.float64)
    ones = torch.zeros(M, 1, d)
    ones[:, 0, first] = 1.0
    how = dict(pos_start=start, norm=lemo.NORM_NONE, flags=lemo.ROTATE_PAIRS if pairs else 0)
    at = torch.tensor(pos, dtype=torch.int32).cuda()
    y = lemo.lemo_qk_rotate(ones.cuda(), None, f.cuda(), at, **how)[0].double().cpu()[:, 0]
    back = lemo.lemo_qk_rotate_grad(ones.cuda(), None, None, None, f.cuda(), at, **how).dQ.double().cpu()[:, 0]
    worst = [(x - want).abs().max().item() * 2 ** 24 for x, want in ((y[:, first], angle.cos()), (y[:, second], angle.sin()), (back[:, first], angle.cos()), (back[:, second], -angle.sin()))]
    print(f"positions to {far} + {start}: {worst} of 2^-24", flush=True)
    assert max(worst) <= BOUND * 2 ** 24


@pytest.mark.gpu
def test_numbers_of_turns_that_pass_binary64():
    """Frequencies that no model has: exact up to 2^62 turns, beyond that still a rotation."""
    pos = places(2 ** 31)
    f = torch.tensor([1e7, 3e7, 1e9, 123456789.0, 8.5e8, 2.0 ** 30, 2.0 ** 30 + 64, 7e8], dtype=torch.float32)
    angle = torch.tensor([[turns(p, x) for x in f.tolist()] for p in pos], dtype=torch.float64)
    ones = torch.zeros(len(pos), 1, 64)
    ones[:, 0, :8] = 1.0
    at = torch.tensor(pos, dtype=torch.int32).cuda()
    y = lemo.lemo_qk_rotate(ones.cuda(), None, f.cuda(), at, norm=lemo.NORM_NONE)[0].double().cpu()[:, 0]
    worst = max((y[:, :8] - angle.cos()).abs().max().item(), (y[:, 8:16] - angle.sin()).abs().max().item())
    print(f"{worst * 2 ** 24} of 2^-24", flush=True)
    assert worst <= BOUND
    far_off = torch.tensor([1e12, 1e20, 1e30, 3e38] * 2, dtype=torch.float32)
    y = lemo.lemo_qk_rotate(ones.cuda(), None, far_off.cuda(), at, norm=lemo.NORM_NONE)[0].double().cpu()[:, 0]
    assert ((y[:, :8] ** 2 + y[:, 8:16] ** 2 - 1).abs() <= 4 * BOUND).all()
