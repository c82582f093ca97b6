"""Layer norm of rows that spread far less than their mean's rounding, against the formula in 64 bits.

u = 2^-24; the tolerance is that of test_gpu_layer_norm.py: a unit value is off by 55 u of itself and 46 u, and the result by half a unit of its type.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F16, BF16 = torch.float16, torch.bfloat16
UNIT = {F16: 2.0 ** -11, BF16: 2.0 ** -8}
LEAST = {F16: 2.0 ** -25, BF16: 2.0 ** -130}


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    assert torch.cuda.is_available()
    return m


@pytest.fixture(scope="module")
def ctx(mqg):
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    return mqg.Context(g, 1, [1])


@pytest.mark.parametrize("eps", [0.0, 2.0 ** -110, 2.0 ** -60])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dim", [40, 250, 1000, 4100, 8192, 16_384])
def test_sums_of_16_bit_rows_that_differ_in_one_column(mqg, ctx, dim, dtype, eps):
    """Equal inputs, equal residuals but for one column, where they differ by a last place: sums that are exact in fp32 and spread 2^-10 of what a mean of 12 bits is off by."""
    rows = 64
    gen = torch.Generator().manual_seed(dim)
    x = (1 + torch.rand((rows, 1), generator=gen)).to(dtype).expand(rows, dim).contiguous()
    r = (2.0 ** -10 * (1 + 0.9 * torch.rand((rows, 1), generator=gen))).to(dtype).expand(rows, dim).contiguous()
    at = torch.randint(0, dim, (rows,), generator=gen)
    at[0], at[1] = 0, dim - 1
    step = 2.0 ** -10 * 2 * UNIT[dtype]
    r[torch.arange(rows), at] = (r[torch.arange(rows), at].float() + step).to(dtype)
    s = x.double() + r.double()
    assert torch.equal(s, (x.float() + r.float()).double())                # (no bit of the sums is lost)
    w, b = (1 + 0.3 * torch.randn(dim, generator=gen)), torch.randn(dim, generator=gen)
    y = torch.zeros((rows, dim), dtype=dtype, device="cuda")
    mqg.mqg_layer_norm(ctx, x.cuda(), w.cuda(), b.cuda(), residual=r.cuda(), y=y, eps=eps)
    torch.cuda.synchronize()
    d = s - s.mean(1, keepdim=True)
    unit = d / torch.sqrt((d * d).mean(1, keepdim=True) + eps)
    want = unit * w.double() + b.double()
    off = w.double().abs() * (55 * U * unit.abs() + 46 * U) + U * b.double().abs()
    assert bool(((y.double().cpu() - want).abs() <= UNIT[dtype] * 1.0001 * want.abs() + off * 1.01 + LEAST[dtype]).all())
