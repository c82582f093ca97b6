"""Layer norm of rows of equal values of any size: the bias, exactly, and gradients that go through the mean alone, by 1/sqrt(eps).

u = 2^-24; the tolerances are those of test_gpu_layer_norm.py: grad_x is off by 192 u of its terms' sizes and half a unit of its type, sums of `rows` terms by that many u and 60.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
UNIT = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
LEAST = {F32: 2.0 ** -140, F16: 2.0 ** -25, BF16: 2.0 ** -130}
TYPES = [F32, F16, BF16]
DIMS = [1, 5, 40, 41, 100, 249, 700, 3000, 9000, 16_384]


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    assert torch.cuda.is_available()
    return m


@pytest.fixture(scope="module")
def ctx(mqg):
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    return mqg.Context(g, 1, [1])


def rows_of(dim, dtype):
    """Rows of zeros, of ordinary values and of values at both ends of fp32's numbers, with and without their sums."""
    values = torch.tensor([0.0, 0.1, -30000.0, 1.3 * 2.0 ** -12] + [1.7 * 2.0 ** e for e in (-120, -100, -80, -60, -40, 60, 100, 112, 116, 120, 126, 127)] + [-3.3e38])
    # and of whole 24 bits, whose mean's error has a square below fp32's numbers
    values = torch.cat([values, (1 + torch.rand(40, generator=torch.Generator().manual_seed(dim))) * 2.0 ** torch.linspace(-120, -50, 40)])
    if dtype == F16:
        values = values[values.abs() <= 65504]
    x = values.to(dtype).unsqueeze(1).expand(len(values), dim).contiguous().cuda()
    assert bool(x.isfinite().all())
    return x


def epsilons(dtype):
    return (1e-5, 1.0, 2.0 ** -20, 2.0 ** 20) if dtype == F16 else (1e-5, 1.0, 2.0 ** -60, 2.0 ** -99, 2.0 ** -110, 2.0 ** -130, 2.0 ** 40)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_the_gradient_goes_through_the_mean(mqg, ctx, dim, dtype):
    gen = torch.Generator().manual_seed(dim)
    x = rows_of(dim, dtype)
    rows = x.shape[0]
    gy, gs = (torch.randn((rows, dim), generator=gen).to(dtype).cuda() for _ in range(2))
    w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
    for eps in epsilons(dtype):
        gx, gb = torch.full_like(x, 3.0), torch.full((dim,), 3.0, device="cuda")
        mqg.mqg_layer_norm_backward(ctx, gy, x, w, gx, grad_bias=gb, grad_sum=gs, eps=eps)
        torch.cuda.synchronize()
        factor = float(torch.tensor(eps, dtype=F32).double()) ** -0.5
        h = gy.double().cpu() * w.double().cpu()
        want = factor * (h - h.mean(1, keepdim=True)) + gs.double().cpu()
        terms = factor * (h.abs() + h.abs().mean(1, keepdim=True)) + gs.double().cpu().abs()
        assert bool(((gx.double().cpu() - want).abs() <= 192 * U * terms + UNIT[dtype] * 1.0001 * want.abs() + LEAST[dtype]).all()), eps
        assert bool(((gb.double().cpu() - gy.double().cpu().sum(0)).abs() <= (rows + 60) * U * gy.double().cpu().abs().sum(0)).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_the_bias_and_nothing_else(mqg, ctx, dim, dtype):
    gen = torch.Generator().manual_seed(dim)
    x = rows_of(dim, dtype)
    rows = x.shape[0]
    gy = torch.randn((rows, dim), generator=gen).to(dtype).cuda()
    w, b = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda(), torch.randn(dim, generator=gen).cuda()
    for eps in epsilons(dtype) + (0.0,):
        y, z, gx = (torch.full_like(x, 3.0) for _ in range(3))
        gw = torch.full((dim,), 3.0, device="cuda")
        q, scale = torch.ones((rows, dim), dtype=torch.int8, device="cuda"), torch.zeros((rows, 1), device="cuda")
        mqg.mqg_layer_norm(ctx, x, w, b, y=y, eps=eps)
        mqg.mqg_layer_norm(ctx, x, w, None, y=z, q=q, q_scale=scale, eps=eps)
        mqg.mqg_layer_norm_backward(ctx, gy, x, w, gx, grad_weight=gw, eps=eps)
        torch.cuda.synchronize()
        assert torch.equal(y, b.to(dtype).expand_as(y)), eps
        assert bool((z == 0).all()) and bool((q == 0).all()) and bool((scale == 2.0 ** -126).all()), eps
        assert bool((gw == 0).all()), eps
