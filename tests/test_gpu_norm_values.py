"""Values at the ends of their ranges in the root-mean-square norm and its backward, against the formulas in 64 bits.

Tolerances as in test_gpu_norm.py: 2e-6 of a value for what is computed in fp32, half a unit of the last place of its type for the rounding.
"""
import pytest
import torch

from test_gpu_norm import FP32, LEAST, TYPES, UNIT, check_backward, check_q

pytestmark = pytest.mark.gpu

MARK = 7.0


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    assert torch.cuda.is_available()
    return m


@pytest.fixture(scope="module")
def ctx(mqg):
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    return mqg.Context(g, 1, [1])


def formulas(s, w, gy, gs, eps):
    """y, grad_x, the sizes of its terms, grad_weight and those of its terms in 64 bits; a row of zeros with eps = 0 has the factor 0."""
    s, gy = s.double().cpu(), gy.double().cpu()
    w = torch.ones(s.shape[1], dtype=torch.float64) if w is None else w.double().cpu()
    mean = (s * s).mean(1, keepdim=True) + eps
    r = torch.where(mean == 0, torch.zeros_like(mean), 1 / torch.sqrt(mean))
    gw = gy * w
    back = s * r * (r * (gw * s).mean(1, keepdim=True)) * r
    gx = r * gw - back
    terms = r * gw.abs() + s.abs() * r * (r * (gw * s).abs().mean(1, keepdim=True)) * r
    if gs is not None:
        gx, terms = gx + gs.double().cpu(), terms + gs.double().cpu().abs()
    return s * r * w, gx, terms, (gy * (s * r)).sum(0), (gy * (s * r)).abs().sum(0)


def near(got, want, dtype):
    return bool(((got.double().cpu() - want).abs() <= (UNIT[dtype] * 1.0001 + FP32) * want.abs() + LEAST[dtype]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", [(4, 1), (6, 5), (6, 40), (700, 40), (9, 300), (300, 602), (5, 3000), (300, 8200), (3, 16384)])
def test_rows_of_zeros_without_an_epsilon(mqg, ctx, rows, dim, dtype):
    gen = torch.Generator().manual_seed(rows + dim)
    s, gy, gs = (torch.randn((rows, dim), generator=gen).to(dtype).cuda() for _ in range(3))
    s[s == 0] = 1
    s[1] = 0
    s[rows - 1] = 0
    w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
    y64, gx64, terms, gw64, gw_terms = formulas(s, w, gy, gs, 0.0)
    for kind, group in ((torch.float8_e4m3fn, 0), (torch.int8, 64)):
        y = torch.full_like(s, MARK)
        q = torch.full((rows, dim), 3, dtype=torch.uint8, device="cuda").view(kind)
        scale = torch.full((rows, -(-dim // group) if group else 1), MARK, device="cuda")
        mqg.mqg_rms_norm(ctx, s, w, y=y, q=q, q_scale=scale, group=group, eps=0.0)
        torch.cuda.synchronize()
        assert near(y, y64, dtype)
        for row in (1, rows - 1):
            assert bool((y[row] == 0).all()) and bool((q[row].float() == 0).all()) and bool((scale[row] == 2.0 ** -126).all())
        check_q(q, scale, y64, group, kind)
    for add in (gs, None):
        gx, gw = torch.full_like(s, MARK), torch.full((dim,), MARK, device="cuda")
        mqg.mqg_rms_norm_backward(ctx, gy, s, w, gx, grad_weight=gw, grad_sum=add, eps=0.0)
        torch.cuda.synchronize()
        _, gx64, terms, gw64, gw_terms = formulas(s, w, gy, add, 0.0)
        check_backward(gx, gw, (gx64, terms, gw64, gw_terms), dtype, rows)
        for row in (1, rows - 1):
            assert torch.equal(gx[row], torch.zeros_like(gx[row]) if add is None else add[row])
