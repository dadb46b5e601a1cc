"""Rotary positions at far times against angles of 70 digits."""
import math
from decimal import Decimal, localcontext

import pytest
import torch

from paper_2309_16849_amd import snls as B
from tests.test_layer_angles_cpu import PI

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()
    return torch.device("cuda:0")


# (theta, pairs): exponents that 53 bits do not hold
FAR = [(1e4, 100), (1e6, 50), (1e30, 100), (3e38, 127)]


@pytest.mark.parametrize("theta,n", FAR)
@pytest.mark.parametrize("time", [2 ** 52 - 1, -(2 ** 53) + 5, 3 ** 25])
def test_angles_of_far_times(dev, theta, n, time):
    """(1, 0) turned is the cosine and the sine: |angle| 2^-51 off by the angle, 2^-24 by its last rounding, and two
    roundings of the function and two of the products."""
    rp = dict(B=1, T=1, C=2 * n, H=1, W=1, HD=1, pairs=(n, 0, 0), theta=(theta, 1.0, 1.0), interleaved=True)
    q = torch.zeros(1, 1, 2 * n, 1, 1)
    q[0, 0, ::2] = 1
    out, _ = B.snls_rotate(q.to(dev), None, rp, times=torch.tensor([[time]]).to(dev))
    points = torch.zeros(1, 3, dtype=torch.int32, device=dev)
    token = B.snls_rotate_points(q.view(1, -1).to(dev), points, rp, times=torch.tensor([time]).to(dev))
    assert torch.equal(out.view(-1), token.view(-1))
    got = out.view(n, 2).cpu().double()
    base = Decimal(float(torch.tensor(theta, dtype=torch.float32)))
    with localcontext() as c:
        c.prec = 70
        for i in range(n):
            angle = Decimal(time) * base ** (-(Decimal(i) / Decimal(n)))
            rest = float(angle.remainder_near(2 * PI))
            bound = abs(float(angle)) * 2.0 ** -51 + 5 * U
            assert abs(float(got[i, 0]) - math.cos(rest)) <= bound, (i, "cos")
            assert abs(float(got[i, 1]) - math.sin(rest)) <= bound, (i, "sin")
