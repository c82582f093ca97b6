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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,dim", [(3, 1), (7, 40), (700, 64), (5, 300), (300, 602), (3, 3000), (300, 8200), (2, 16384)])
def test_rows_of_any_size(mqg, ctx, rows, dim, dtype):
    """Rows whose squares leave 32 bits at either end, beside others in between: |s| from 2^-120 to 2^120, and sums near the borders of what is added as it is."""
    gen = torch.Generator().manual_seed(rows * 3 + dim)
    size = torch.tensor([-120, -75, -57, -51, -45, 0, 30, 43, 50, 57, 64, 90, 120], dtype=torch.float64)
    exp = size[torch.arange(rows) % len(size)].unsqueeze(1)
    for eps in (0.0, 1e-6, 1e-35):
        s = (torch.randn((rows, dim), generator=gen, dtype=torch.float64) * 2 ** exp).to(dtype).cuda()
        # gradients of a size at which the results are numbers of 32 bits: grad_x has the size of gy / s
        gy = (torch.randn((rows, dim), generator=gen, dtype=torch.float64) * 2 ** (exp / 2)).to(dtype).cuda()
        w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
        y64, gx64, terms, _, _ = formulas(s, w, gy, None, eps)
        y, sums = torch.full_like(s, MARK), torch.full_like(s, MARK)
        q, scale = torch.zeros((rows, dim), dtype=torch.int8, device="cuda"), torch.zeros((rows, 1), device="cuda")
        mqg.mqg_rms_norm(ctx, s, w, sum_out=sums, y=y, q=q, q_scale=scale, eps=eps)
        torch.cuda.synchronize()
        assert torch.equal(sums, s)
        assert near(y, y64, dtype), eps
        check_q(q, scale, y64, 0, torch.int8)
        for start in range(0, min(rows, len(size))):                    # one size at a time: grad_weight's terms are of the size of gy
            pick = torch.arange(start, rows, len(size)).cuda()
            part = [t[pick].contiguous() for t in (s, gy)]
            gx, gw = torch.full_like(part[0], MARK), torch.full((dim,), MARK, device="cuda")
            mqg.mqg_rms_norm_backward(ctx, part[1], part[0], w, gx, grad_weight=gw, eps=eps)
            torch.cuda.synchronize()
            _, gx64, terms, gw64, gw_terms = formulas(part[0], w, part[1], None, eps)
            check_backward(gx, gw, (gx64, terms, gw64, gw_terms), dtype, rows)


@pytest.mark.parametrize("dim", [5, 300, 3000])
def test_rows_of_the_least_numbers(mqg, ctx, dim):
    """Rows about the least number of full precision; those whose factor 1/rms is above the largest number of 32 bits count as zeros, in both directions."""
    gen = torch.Generator().manual_seed(21)
    noise, gy = torch.randn((6, dim), generator=gen, dtype=torch.float64), (torch.randn((6, dim), generator=gen, dtype=torch.float64) * 2.0 ** -40).float().cuda()
    for exp in (-124, -140):
        s = (noise * 2.0 ** exp).float().cuda()
        y, gx, gw = torch.full_like(s, MARK), torch.full_like(s, MARK), torch.full((dim,), MARK, device="cuda")
        q, scale = torch.full((6, dim), 3, dtype=torch.int8, device="cuda"), torch.zeros((6, 1), device="cuda")
        mqg.mqg_rms_norm(ctx, s, None, y=y, q=q, q_scale=scale, eps=0.0)
        mqg.mqg_rms_norm_backward(ctx, gy, s, None, gx, grad_weight=gw, eps=0.0)
        torch.cuda.synchronize()
        if exp == -124:
            y64, gx64, terms, gw64, gw_terms = formulas(s, None, gy, None, 0.0)
            assert near(y, y64, torch.float32)
            check_q(q, scale, y64, 0, torch.int8)
            check_backward(gx, gw, (gx64, terms, gw64, gw_terms), torch.float32, 6)
        else:
            assert bool((y == 0).all()) and bool((q == 0).all()) and bool((scale == 2.0 ** -126).all())
            assert bool((gx == 0).all()) and bool((gw == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dim,group,col", [(66, 64, 62), (130, 128, 126), (602, 64, 575), (2050, 32, 2047), (33, 32, 31), (8194, 128, 8191), (3, 32, 1), (64, 32, 5)])
def test_a_weight_that_is_not_finite_is_its_columns_alone(mqg, ctx, dim, group, col, bad, dtype):
    rows = 5
    gen = torch.Generator().manual_seed(dim)
    x = torch.randn((rows, dim), generator=gen).to(dtype).cuda()
    x[x == 0] = 1
    w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
    w[col] = bad
    others = torch.arange(dim) != col
    y64 = formulas(x, w, x, None, 1e-6)[0]
    for kind in (torch.float8_e4m3fn, torch.int8):
        y = torch.zeros_like(x)
        q = torch.zeros((rows, dim), dtype=torch.uint8, device="cuda").view(kind)
        scale = torch.zeros((rows, -(-dim // group)), device="cuda")
        mqg.mqg_rms_norm(ctx, x, w, y=y, q=q, q_scale=scale, group=group, eps=1e-6)
        torch.cuda.synchronize()
        assert near(y[:, others], y64[:, others], dtype) and not bool(y[:, col].isfinite().any())
        hit = torch.arange(scale.shape[1]) == col // group
        assert bool(scale[:, hit].isnan().all()) and bool(scale[:, ~hit].isfinite().all())
        for g in range(scale.shape[1]):
            if g != col // group:
                lo, hi = g * group, min(dim, (g + 1) * group)
                check_q(q[:, lo:hi], scale[:, g:g + 1], y64[:, lo:hi], 0, kind)
    # backward: the mean has the weight's infinity once, whatever its neighbour's vector repeats; grad_weight does not depend on the weight
    gy = torch.randn((rows, dim), generator=gen).to(dtype).cuda()
    gx, gw = torch.zeros_like(x), torch.zeros(dim, device="cuda")
    mqg.mqg_rms_norm_backward(ctx, gy, x, w, gx, grad_weight=gw, eps=1e-6)
    torch.cuda.synchronize()
    _, gx64, _, gw64, gw_terms = formulas(x, w, gy, None, 1e-6)
    got = gx.double().cpu()
    assert torch.equal(got.isnan(), gx64.isnan()) and torch.equal(got.nan_to_num(), gx64.nan_to_num(posinf=float(got.nan_to_num().max()), neginf=float(got.nan_to_num().min())))
    assert bool(((gw.double().cpu() - gw64).abs() <= (rows + 60) * 2.0 ** -24 * gw_terms + 1e-30).all())
