"""The factor that clips gradients whose norm is near either end of fp32's numbers: mul * min(1, max_norm / norm) as in 64 bits.

u = 2^-24: the norm is off by 10 u (sixteen squares in fp32, half of that in the root, one rounding), the factor by that, a quotient and a product.  Norms below 2^-126 have
a last place of 2^-149, half of which is the norm's rounding.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    assert torch.cuda.is_available()
    return m


@pytest.fixture(scope="module")
def ctx(mqg):
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    return mqg.Context(g, 1, [1])


@pytest.mark.parametrize("size", [-149, -146, -140, -130, -127, -126, -120, 100, 120, 124, 125, 126, 127])
@pytest.mark.parametrize("n", [1, 4, 100_000])
def test_limits_below_and_above_the_norm(mqg, ctx, n, size):
    g = torch.full((n,), 2.0 ** size / math.sqrt(n) if size > 0 else 2.0 ** size, device="cuda")
    total = math.sqrt(float((g.double() ** 2).sum()))
    for share in (2.0 ** -20, 0.25, 0.7, 1.5):
        limit = float(torch.tensor(share * total, dtype=torch.float32).clamp(min=2.0 ** -149, max=3.4e38))
        for mul in (1.0, 0.5):
            norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
            mqg.mqg_grad_norm(ctx, mqg.Params(grads=[g]), max_norm=limit, mul=mul, norm=norm, scale=scale)
            torch.cuda.synchronize()
            off = 10 * U * mul * total + 2.0 ** -150
            assert abs(float(norm) - mul * total) <= off * 1.0001
            least, most = (mul * min(1.0, limit / t) if t > 0 else mul for t in (mul * total + off, mul * total - off))
            assert least * (1 - 3 * U) <= float(scale) <= most * (1 + 3 * U), (share, mul)
