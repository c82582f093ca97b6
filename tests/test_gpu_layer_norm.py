"""Layer norm with the residual's addition, its output in 8 bits, and its backward, against the formulas in 64 bits.

Tolerances, u = 2^-24.  Sums of a row add at most 45 terms one after the other, in a lane, across lanes and across wavefronts: they are off by 45 u
of their terms' sizes.  The differences' own mean c so is off by 45 u of the spread, the variance, of which c^2 may take half away, by 94 u of itself, its root
by half of that; with the roundings of the square root, the quotient and the products a unit value is off by 55 u of itself and 46 u.  What the
sum of two fp32 inputs loses, u |s|, counts against the spread.  Results are rounded once to their type: 2^-24, 2^-11, 2^-8 relative.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = 1e-5
U = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -140, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -130}
TYPES = [torch.float32, torch.float16, torch.bfloat16]
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


class Padded:
    """[rows, dim] inside a larger buffer filled with a mark: `off` elements before it, `pad` after every row, guard rows at the end."""

    def __init__(self, rows, dim, dtype, pad=0, off=0):
        self.stride = dim + pad
        self.buf = torch.full((off + (rows + 2) * self.stride,), MARK, dtype=torch.float32, device="cuda").to(dtype)
        self.off, self.rows, self.dim = off, rows, dim
        self.t = torch.as_strided(self.buf, (rows, dim), (self.stride, 1), off)

    def untouched(self):
        seen = torch.ones(self.buf.numel(), dtype=torch.bool, device="cuda")
        torch.as_strided(seen, (self.rows, self.dim), (self.stride, 1), self.off).fill_(False)
        return bool((self.buf.float()[seen] == MARK).all())


def filled(rows, dim, dtype, gen, pad=0, off=0, spread=0.0, shift=0.0):
    p = Padded(rows, dim, dtype, pad, off)
    x = torch.randn((rows, dim), generator=gen)
    if spread:
        x = (x + shift * torch.randn((rows, 1), generator=gen)) * torch.exp(spread * torch.randn((rows, 1), generator=gen))
    p.t.copy_(x.to(dtype))
    return p


def norm64(x, r, w, b, eps=EPS):
    """The sum, the norm, and how far fp32 may be from it before it is rounded to its type."""
    s = x.double().cpu()
    lost = torch.zeros_like(s)
    if r is not None:
        s = s + r.double().cpu()
        lost = U * s.abs() if x.dtype == torch.float32 else lost
    d = s - s.mean(1, keepdim=True)
    factor = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + eps)
    unit = d * factor
    w = torch.ones(s.shape[1], dtype=torch.float64) if w is None else w.double().cpu()
    b = torch.zeros(s.shape[1], dtype=torch.float64) if b is None else b.double().cpu()
    off = w.abs() * (55 * U * unit.abs() + 46 * U + (lost + lost.mean(1, keepdim=True)) * factor * (1 + unit.abs())) + U * b.abs()
    return s, unit * w + b, off


def near(got, want, off, dtype):
    got = got.double().cpu()
    return bool(((got - want).abs() <= UNIT[dtype] * 1.0001 * want.abs() + off * 1.01 + LEAST[dtype]).all())


def half_unit(v, kind):
    if kind == torch.int8:
        return torch.full_like(v, 0.5)
    _, e = torch.frexp(v)
    return torch.ldexp(torch.ones_like(v), (e - 1).clamp(min=-6) - 4)


def check_q(q, scale, y64, off, group, kind):
    top = 127.0 if kind == torch.int8 else 448.0
    dim = y64.shape[1]
    width = group or dim
    groups = -(-dim // width)

    def largest(t):
        return torch.nn.functional.pad(t, (0, groups * width - dim)).view(-1, groups, width).amax(2)

    want = (largest(y64.abs()) / top).clamp(min=2.0 ** -126)
    got = scale[:, :groups].double().cpu()
    assert bool(((got - want).abs() <= 3 * U * want + 1.01 * largest(off) / top).all())
    wide = got.repeat_interleave(width, 1)[:, :dim]
    v = y64 / wide
    assert bool(((q.double().cpu() - v).abs() <= half_unit(v, kind) * (1 + 1e-6) + 3 * U * v.abs() + 1.01 * off / wide).all())
    assert float(q.double().abs().max()) <= top


DIMS = [1, 2, 3, 7, 16, 33, 64, 100, 127, 256, 257, 513, 602, 1025, 2049, 4100, 8192, 16384]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_rows_sum_and_8_bits(mqg, ctx, dim, dtype):
    gen = torch.Generator().manual_seed(dim)
    for rows, pad, off, residual, weighted, kind, group in [
            (1, 0, 0, True, True, torch.float8_e4m3fn, 128), (5, 3, 1, True, False, torch.int8, 0), (37, -dim % 16, 0, False, True, torch.float8_e4m3fn, 0),
            (67, 0, 1, True, True, torch.int8, 32), (67, 5, 3, False, False, torch.float8_e4m3fn, 64)]:
        x = filled(rows, dim, dtype, gen, pad, off, spread=1.0, shift=2.0)
        r = filled(rows, dim, dtype, gen, pad, off) if residual else None
        w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda() if weighted else None
        b = torch.randn(dim, generator=gen).cuda() if weighted else None
        s, y = Padded(rows, dim, dtype, pad, off), Padded(rows, dim, dtype, pad, off)
        qb = torch.full((rows + 1, dim + 3), 3, dtype=torch.uint8, device="cuda")
        q = qb.view(kind)[:rows, :dim]
        groups = -(-dim // group) if group else 1
        scale = torch.full((rows, groups + 1), MARK, device="cuda")
        args = dict(residual=None if r is None else r.t, eps=EPS)
        mqg.mqg_layer_norm(ctx, x.t, w, b, sum_out=s.t, y=y.t, q=q, q_scale=scale, group=group, **args)
        torch.cuda.synchronize()
        s64, y64, far = norm64(x.t, None if r is None else r.t, w, b)
        assert near(s.t, s64, U * s64.abs(), dtype), (rows, group)
        assert near(y.t, y64, far, dtype), (rows, group)
        check_q(q, scale, y64, far, group, kind)
        assert s.untouched() and y.untouched()
        assert bool((qb[:rows, dim:] == 3).all()) and bool((qb[rows:] == 3).all()) and bool((scale[:, groups:] == MARK).all())
        # each output alone is the same
        y2 = Padded(rows, dim, dtype, pad, off)
        mqg.mqg_layer_norm(ctx, x.t, w, b, y=y2.t, **args)
        q2, scale2 = torch.zeros((rows, dim), dtype=torch.uint8, device="cuda"), torch.zeros((rows, groups), device="cuda")
        mqg.mqg_layer_norm(ctx, x.t, w, b, q=q2.view(kind), q_scale=scale2, group=group, **args)
        torch.cuda.synchronize()
        assert torch.equal(y2.t, y.t) and torch.equal(q2, qb[:rows, :dim]) and torch.equal(scale2, scale[:, :groups])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", [(3000, 64), (1500, 256), (700, 602), (90_000, 16), (600, 2500), (5000, 8200)])
def test_many_rows_the_device_count_and_buffers_in_place(mqg, ctx, rows, dim, dtype):
    gen = torch.Generator().manual_seed(1)
    x = torch.randn((rows, dim), generator=gen).to(dtype).cuda()
    r = torch.randn((rows, dim), generator=gen).to(dtype).cuda()
    x[5], r[5] = 3.0, 1.0                                          # equal values take the longer way, also in place
    w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
    b = torch.randn(dim, generator=gen).cuda()
    s64, y64, off = norm64(x, r, w, b)
    y = torch.zeros_like(x)
    mqg.mqg_layer_norm(ctx, x, w, b, residual=r, y=y, eps=EPS)
    torch.cuda.synchronize()
    assert near(y, y64, off, dtype) and torch.equal(y[5], b.to(dtype))
    for count, valid in ((rows * 2 // 3, rows * 2 // 3), (rows + 9, rows), (0, 0), (-4, 0)):
        for swap in (False, True):
            xx, rr = x.clone(), r.clone()
            to_sum, to_y = (xx, rr) if swap else (rr, xx)
            mqg.mqg_layer_norm(ctx, xx, w, b, residual=rr, sum_out=to_sum, y=to_y, eps=EPS, num_rows=torch.tensor([count], device="cuda"))
            torch.cuda.synchronize()
            old_sum, old_y = (x, r) if swap else (r, x)
            assert torch.equal(to_y[:valid], y[:valid]) and torch.equal(to_y[valid:], old_y[valid:])
            assert near(to_sum[:valid], s64[:valid], U * s64[:valid].abs(), dtype) and torch.equal(to_sum[valid:], old_sum[valid:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [40, 300, 3000, 9000])
def test_rows_of_equal_values_and_rows_that_are_not_finite(mqg, ctx, dim, dtype):
    rows = 12
    gen = torch.Generator().manual_seed(2)
    x = torch.randn((rows, dim), generator=gen).to(dtype).cuda()
    x[1], x[2], x[4] = 0, 0.1, -30000.0
    x[3, 5] = float("nan")
    x[5, 7] = float("inf")
    x[7, 11] = float("-inf")
    b = torch.randn(dim, generator=gen).cuda()
    fine = [0, 6, 8, 9, 10, 11]
    for eps in (EPS, 0.0):
        for kind in (torch.float8_e4m3fn, torch.int8):
            for group in (0, 32):
                y = torch.zeros_like(x)
                q = torch.zeros((rows, dim), dtype=torch.uint8, device="cuda").view(kind)
                scale = torch.zeros((rows, -(-dim // group) if group else 1), device="cuda")
                mqg.mqg_layer_norm(ctx, x, None, b, y=y, q=q, q_scale=scale, group=group, eps=eps)
                torch.cuda.synchronize()
                for row in (1, 2, 4):
                    assert torch.equal(y[row], b.to(dtype)), (eps, row)
                for row in (3, 5, 7):
                    assert bool(y[row].isnan().all()) and bool(scale[row].isnan().all())
                _, y64, off = norm64(x[fine], None, None, b, eps)
                assert near(y[fine], y64, off, dtype)
                check_q(q[fine], scale[fine], y64, off, group, kind)
        # gradients: no part of a row of equal values reaches it without an epsilon; rows that are not finite keep to themselves
        gy = torch.randn((rows, dim), generator=gen).to(dtype).cuda()
        gs = torch.randn((rows, dim), generator=gen).to(dtype).cuda()
        gx, gw, gb = torch.zeros_like(x), torch.zeros(dim, device="cuda"), torch.zeros(dim, device="cuda")
        mqg.mqg_layer_norm_backward(ctx, gy, x, None, gx, grad_weight=gw, grad_bias=gb, grad_sum=gs, eps=eps)
        torch.cuda.synchronize()
        if eps == 0:
            for row in (1, 2, 4):
                assert torch.equal(gx[row], gs[row])
        assert bool(gx[[3, 5, 7]].isnan().all()) and bool(gx[[1, 2, 4] + fine].isfinite().all()) and bool(gb.isfinite().all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [5, 48, 700, 5000, 9001])
def test_rows_of_any_size_and_mean(mqg, ctx, dim, dtype):
    """Rows whose sums and squares leave fp32, without an epsilon, and rows whose mean is large against their spread: the norm is that of the row times a power of two."""
    gen = torch.Generator().manual_seed(dim)
    base = torch.randn((40, dim), generator=gen).to(dtype)
    gy = torch.randn((40, dim), generator=gen).to(dtype).cuda()
    size = torch.tensor([0, 60, 100, 120, 124, -30, -55, -70, -100, -110] * 4)
    x = torch.ldexp(base.float(), size.view(-1, 1)).to(dtype)
    x[10:20] = x[10:20] + torch.ldexp(torch.full((10, 1), 6.0), size[10:20].view(-1, 1)).to(dtype)
    x = x.cuda()
    w, b = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda(), torch.randn(dim, generator=gen).cuda()
    y, gx = torch.zeros_like(x), torch.zeros_like(x)
    gw, gb = torch.zeros(dim, device="cuda"), torch.zeros(dim, device="cuda")
    mqg.mqg_layer_norm(ctx, x, w, b, y=y, eps=0.0)
    mqg.mqg_layer_norm_backward(ctx, gy, x, w, gx, grad_weight=gw, grad_bias=gb, eps=0.0)
    torch.cuda.synchronize()
    _, y64, off = norm64(x, None, w, b, 0.0)
    assert near(y, y64, off, dtype)
    down = torch.ldexp(torch.ones(1, dtype=torch.float64), -size.double().int()).view(-1, 1)
    want = backward64(gy, x.double().cpu() * down, w, None, 0.0)
    got = gx.double().cpu()
    # gradients go as one over the row's size: those of the smallest rows that are still fp32 numbers are compared
    inside = ((want[0].abs().amax(1, keepdim=True) * down) < 2.0 ** 126) & (size.view(-1, 1) < 100)
    bound = (192 * U * want[1] + UNIT[dtype] * 1.0001 * want[0].abs()) * down + 2.0 ** -126
    assert bool((((got - want[0] * down).abs() <= bound) | ~inside).all())
    assert bool(((gw.double().cpu() - want[2]).abs() <= (40 + 60 + 101) * U * want[3]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [6, 100, 1100])
def test_weight_and_bias_alone(mqg, ctx, dim, dtype):
    gen = torch.Generator().manual_seed(15)
    x = torch.randn((70, dim), generator=gen).to(dtype).cuda()
    w, b = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda(), torch.randn(dim, generator=gen).cuda()
    ones, zeros = torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda")
    for some, full in (((w, None), (w, zeros)), ((None, b), (ones, b)), ((None, None), (ones, zeros))):
        got, want = torch.zeros_like(x), torch.zeros_like(x)
        mqg.mqg_layer_norm(ctx, x, *some, y=got, eps=EPS)
        mqg.mqg_layer_norm(ctx, x, *full, y=want, eps=EPS)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_offsets_beyond_32_bits(mqg, ctx):
    stride, dim = (1 << 31) + 64, 100                              # elements between two rows
    buf = torch.zeros(stride + dim, dtype=torch.float16, device="cuda")
    x = torch.as_strided(buf, (2, dim), (stride, 1))
    x.copy_(torch.randn((2, dim), generator=torch.Generator().manual_seed(3)).half())
    y = torch.zeros((2, dim), dtype=torch.float16, device="cuda")
    gx = torch.zeros_like(y)
    mqg.mqg_layer_norm(ctx, x, None, y=y, eps=EPS)
    mqg.mqg_layer_norm_backward(ctx, y, x, None, gx, eps=EPS)
    want = torch.zeros_like(gx)
    mqg.mqg_layer_norm_backward(ctx, y, x.contiguous(), None, want, eps=EPS)
    torch.cuda.synchronize()
    _, y64, off = norm64(x, None, None, None)
    assert near(y, y64, off, torch.float16) and torch.equal(gx, want)


# ---------------------------------------------------------------------------------------------- backward

def backward64(gy, s, w, gs, eps=EPS):
    """grad_x, what its error is a multiple of, grad_weight and grad_bias with theirs."""
    gy, s = gy.double().cpu(), s.double().cpu()
    d = s - s.mean(1, keepdim=True)
    r = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + eps)
    u = d * r
    h = gy if w is None else gy * w.double().cpu()
    gx = r * (h - h.mean(1, keepdim=True) - u * (h * u).mean(1, keepdim=True))
    far = 1 + u.abs()
    terms = r * (h.abs() + far * (h.abs().mean(1, keepdim=True) + (h * u).abs().mean(1, keepdim=True)))
    if gs is not None:
        gx, terms = gx + gs.double().cpu(), terms + gs.double().cpu().abs()
    return gx, terms, (gy * u).sum(0), (gy.abs() * far).sum(0), gy.sum(0), gy.abs().sum(0)


def check_backward(gx, gw, gb, want, dtype, rows):
    gx64, terms, gw64, gw_terms, gb64, gb_terms = want
    # the means are off by 45 u of their terms' sizes, unit values by 55 u of themselves and 46 u, once more in the mean of products with them; the factor by 52
    assert bool(((gx.double().cpu() - gx64).abs() <= 192 * U * terms + UNIT[dtype] * 1.0001 * gx64.abs() + LEAST[dtype]).all())
    # sums of `rows` terms: no more than that many additions in a row
    if gw is not None:
        assert bool(((gw.double().cpu() - gw64).abs() <= (min(rows, 400) + 60 + 101) * U * gw_terms + 1e-30).all())
    if gb is not None:
        assert bool(((gb.double().cpu() - gb64).abs() <= (min(rows, 400) + 60) * U * gb_terms + 1e-30).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_backward(mqg, ctx, dim, dtype):
    gen = torch.Generator().manual_seed(100 + dim)
    for rows, pad, off, residual, weighted in [(1, 0, 0, True, True), (5, 3, 1, False, True), (67, -dim % 16, 0, True, False), (260, 1, 3, True, True)]:
        s, gy = filled(rows, dim, dtype, gen, pad, off, spread=1.0, shift=2.0), filled(rows, dim, dtype, gen, pad, off)
        gs = filled(rows, dim, dtype, gen, pad, off) if residual else None
        w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda() if weighted else None
        gx = Padded(rows, dim, dtype, pad, off)
        gw, gb = (torch.full((dim + 2,), MARK, device="cuda") for _ in range(2))
        args = dict(grad_sum=None if gs is None else gs.t, eps=EPS)
        mqg.mqg_layer_norm_backward(ctx, gy.t, s.t, w, gx.t, grad_weight=gw[1:-1], grad_bias=gb[1:-1], **args)
        torch.cuda.synchronize()
        check_backward(gx.t, gw[1:-1], gb[1:-1], backward64(gy.t, s.t, w, None if gs is None else gs.t), dtype, rows)
        assert gx.untouched() and bool((gw[[0, -1]] == MARK).all()) and bool((gb[[0, -1]] == MARK).all())
        # each gradient alone is the same
        for weight, bias in ((True, False), (False, True), (False, False)):
            alone, gw2, gb2 = Padded(rows, dim, dtype, pad, off), torch.zeros(dim, device="cuda"), torch.zeros(dim, device="cuda")
            mqg.mqg_layer_norm_backward(ctx, gy.t, s.t, w, alone.t, grad_weight=gw2 if weight else None, grad_bias=gb2 if bias else None, **args)
            torch.cuda.synchronize()
            assert torch.equal(gx.t, alone.t)
            assert not weight or torch.equal(gw2, gw[1:-1])
            assert not bias or torch.equal(gb2, gb[1:-1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", [(90_000, 16), (20_000, 100), (9_000, 602), (3_000, 2500), (1_200, 8200), (700, 16_384)])
def test_backward_many_rows_and_the_device_count(mqg, ctx, rows, dim, dtype):
    gen = torch.Generator().manual_seed(4)
    s, gy, gs = (torch.randn((rows, dim), generator=gen).to(dtype).cuda() for _ in range(3))
    s[3] = 2.0
    w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
    for count, valid in ((rows, rows), (rows - 77, rows - 77), (rows + 5, rows), (0, 0)):
        gx = torch.full_like(s, MARK)
        gw, gb, again, again_b = (torch.full((dim,), MARK, device="cuda") for _ in range(4))
        num = torch.tensor([count], device="cuda")
        mqg.mqg_layer_norm_backward(ctx, gy, s, w, gx, grad_weight=gw, grad_bias=gb, grad_sum=gs, eps=EPS, num_rows=num)
        torch.cuda.synchronize()
        check_backward(gx[:valid], gw, gb, backward64(gy[:valid], s[:valid], w, gs[:valid]), dtype, rows)
        assert bool((gx[valid:] == MARK).all())
        for place in ("gy", "s", "gs"):                                # in place of each input
            at = {"gy": gy.clone(), "s": s.clone(), "gs": gs.clone()}
            mqg.mqg_layer_norm_backward(ctx, at["gy"], at["s"], w, at[place], grad_weight=again, grad_bias=again_b, grad_sum=at["gs"], eps=EPS, num_rows=num)
            torch.cuda.synchronize()
            assert torch.equal(again, gw) and torch.equal(again_b, gb) and torch.equal(at[place][:valid], gx[:valid])
    empty = torch.zeros((0, dim), dtype=dtype, device="cuda")
    gw.fill_(MARK)
    gb.fill_(MARK)
    mqg.mqg_layer_norm_backward(ctx, empty, empty, w, empty, grad_weight=gw, grad_bias=gb, eps=EPS)
    mqg.mqg_layer_norm(ctx, empty, w, y=empty, eps=EPS)
    torch.cuda.synchronize()
    assert bool((gw == 0).all()) and bool((gb == 0).all())


def test_backward_against_differences(mqg, ctx):
    rows, dim = 6, 50
    gen = torch.Generator().manual_seed(5)
    s, gy, gs = (torch.randn((rows, dim), generator=gen) for _ in range(3))
    w, b = 1 + 0.3 * torch.randn(dim, generator=gen), torch.randn(dim, generator=gen)
    gx, gw, gb = torch.zeros((rows, dim), device="cuda"), torch.zeros(dim, device="cuda"), torch.zeros(dim, device="cuda")
    mqg.mqg_layer_norm_backward(ctx, gy.cuda(), s.cuda(), w.cuda(), gx, grad_weight=gw, grad_bias=gb, grad_sum=gs.cuda(), eps=EPS)
    torch.cuda.synchronize()

    def loss(s, w, b):
        d = s - s.mean(1, keepdim=True)
        y = d / torch.sqrt((d * d).mean(1, keepdim=True) + EPS) * w + b
        return float((gy.double() * y).sum() + (gs.double() * s).sum())

    h = 1e-5                                                       # the difference is off by h^2 of the third derivative, and 1e-15 / h
    s, w, b = s.double(), w.double(), b.double()
    for k in range(20):
        ds, dw, db = (torch.randn(t.shape, generator=gen).double() for t in (s, w, b))
        slope = (loss(s + h * ds, w + h * dw, b + h * db) - loss(s - h * ds, w - h * dw, b - h * db)) / (2 * h)
        parts = [(g.double().cpu() * t) for g, t in ((gx, ds), (gw, dw), (gb, db))]
        assert abs(sum(float(p.sum()) for p in parts) - slope) <= 1e-5 * sum(float(p.abs().sum()) for p in parts)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [5, 64, 250, 1023, 4100, 8200])
def test_backward_of_a_few_rows(mqg, ctx, dim, dtype):
    """Rows that one workgroup takes by itself, the first that it does not, and device counts of less."""
    gen = torch.Generator().manual_seed(11)
    w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
    for rows in (1, 2, 3, 4, 5, 16, 17, 64, 65, 256, 257):
        s, gy, gs = (torch.randn((rows, dim), generator=gen).to(dtype).cuda() for _ in range(3))
        for count, valid in ((rows, rows), (rows // 2, rows // 2), (0, 0)):
            gx = torch.full_like(s, MARK)
            gw, gb = torch.full((dim,), MARK, device="cuda"), torch.full((dim,), MARK, device="cuda")
            mqg.mqg_layer_norm_backward(ctx, gy, s, w, gx, grad_weight=gw, grad_bias=gb, grad_sum=gs, eps=EPS, num_rows=torch.tensor([count], device="cuda"))
            torch.cuda.synchronize()
            check_backward(gx[:valid], gw, gb, backward64(gy[:valid], s[:valid], w, gs[:valid]), dtype, rows)
            assert bool((gx[valid:] == MARK).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_backward_of_few_columns_call_after_call(mqg, ctx, dtype):
    """Shares that the last workgroup adds: any number of workgroups, the same bits in every call, and what the device counts in between."""
    gen = torch.Generator().manual_seed(14)
    for dim, rows in ((1, 300), (3, 9000), (64, 1400), (64, 2048), (100, 700), (128, 1100), (128, 5000), (129, 1100)):
        s, gy = (torch.randn((rows, dim), generator=gen).to(dtype).cuda() for _ in range(2))
        w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
        first = None
        for call in range(6):
            count = rows if call != 3 else rows // 3
            gx, gw, gb = torch.zeros_like(s), torch.full((dim,), MARK, device="cuda"), torch.full((dim,), MARK, device="cuda")
            mqg.mqg_layer_norm_backward(ctx, gy, s, w, gx, grad_weight=gw, grad_bias=gb, eps=EPS, num_rows=torch.tensor([count], device="cuda"))
            torch.cuda.synchronize()
            if call in (0, 3):
                check_backward(gx[:count], gw, gb, backward64(gy[:count], s[:count], w, None), dtype, rows)
                first = (gw, gb) if call == 0 else first
            else:
                assert torch.equal(gw, first[0]) and torch.equal(gb, first[1]), (dim, rows, call)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_weight_that_is_not_finite_stays_its_own_columns(mqg, ctx, bad):
    for dim in (10, 250, 3000):
        rows, col = 9, dim - 1
        gen = torch.Generator().manual_seed(12)
        x = torch.randn((rows, dim), generator=gen).half().cuda()
        for which in (0, 1):
            w, b = torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda")
            (w, b)[which][col] = bad
            y, scale = torch.zeros_like(x), torch.zeros((rows, -(-dim // 32)), device="cuda")
            q = torch.zeros((rows, dim), dtype=torch.int8, device="cuda")
            mqg.mqg_layer_norm(ctx, x, w, b, y=y, q=q, q_scale=scale, group=32, eps=EPS)
            torch.cuda.synchronize()
            assert not bool(y[:, col].isfinite().any()) and bool(y[:, :col].isfinite().all())
            assert bool(scale[:, -1].isnan().all()) and bool(scale[:, :-1].isfinite().all())


def test_recorded_and_replayed(mqg, ctx):
    rows, dim = 3000, 96
    own = mqg.Context(mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda")), 1, [1])
    gen = torch.Generator().manual_seed(13)
    x, gy = torch.randn((rows, dim), generator=gen).cuda(), torch.randn((rows, dim), generator=gen).cuda()
    w, b = torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda")
    got, want = ([torch.zeros_like(x), torch.zeros_like(x), torch.zeros(dim, device="cuda"), torch.zeros(dim, device="cuda")] for _ in range(2))

    def step(c, out):
        mqg.mqg_layer_norm(c, x, w, b, y=out[0], eps=EPS)
        mqg.mqg_layer_norm_backward(c, gy, x, w, out[1], grad_weight=out[2], grad_bias=out[3], eps=EPS)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with pytest.raises(mqg.MqgError) as refused:                    # nothing is allocated while a stream is recorded
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=side):
            step(own, got)
    assert refused.value.code == mqg.MQG_ERR_UNSUPPORTED
    torch.cuda.synchronize()
    own.reserve_layer(norm_dim=dim)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(own, got)
    for k in range(4):
        x.add_(0.1 * k)
        w.add_(0.1)
        graph.replay()
        step(ctx, want)
        torch.cuda.synchronize()
        for g, t in zip(got, want):
            assert torch.equal(g, t), k


# ---------------------------------------------------------------------------------------------- refusals

def test_refusals(mqg, ctx):
    x = torch.zeros((4, 8), device="cuda")
    w = torch.ones(8, device="cuda")
    q, scale = torch.zeros((4, 8), dtype=torch.int8, device="cuda"), torch.zeros((4, 1), device="cuda")

    def forward(xs=8, dim=8, dtype=0, eps=1e-6, rows=4, y=x.data_ptr(), qp=None, qs=8, qt=0, group=0, sp=scale.data_ptr(), ss=1, xp=x.data_ptr()):
        return mqg.lib.mqg_layer_norm(ctx.h, xp, xs, None, 0, w.data_ptr(), None, eps, None, rows, dim, dtype, None, 0, y, 8, qp, qs, qt, group, sp, ss, None)

    bad, limit = mqg.MQG_ERR_INVALID_ARG, mqg.MQG_ERR_UNSUPPORTED
    assert forward(xs=7) == bad and b"mqg_layer_norm: stride" in mqg.lib.mqg_last_error(ctx.h)
    assert forward(dim=0) == bad and forward(dtype=3) == bad and forward(rows=-1) == bad and forward(xp=None) == bad
    assert forward(eps=-1.0) == bad and forward(eps=float("nan")) == bad and forward(eps=float("inf")) == bad
    assert forward(y=None) == bad and b"neither" in mqg.lib.mqg_last_error(ctx.h)
    assert forward(dim=mqg.MQG_NORM_MAX_DIM + 1, xs=1 << 20) == limit
    qp = q.data_ptr()
    assert forward(qp=qp, qs=7) == bad and forward(qp=qp, qt=2) == bad and forward(qp=qp, group=16) == bad and forward(qp=qp, sp=None) == bad
    assert forward(qp=qp, ss=0) == bad

    def backward(strides=(8, 8, 8), dim=8, gx=x.data_ptr(), s=x.data_ptr(), eps=1e-6):
        return mqg.lib.mqg_layer_norm_backward(ctx.h, x.data_ptr(), strides[0], s, strides[1], w.data_ptr(), None, 0, eps, None, 4, dim, 0, gx,
                                               strides[2], None, None, None)

    for k in range(3):
        assert backward(strides=[7 if i == k else 8 for i in range(3)]) == bad
    assert backward(gx=None) == bad and backward(s=None) == bad and backward(eps=-1.0) == bad and backward(dim=0) == bad
    with pytest.raises(TypeError):
        mqg.mqg_layer_norm(ctx, x.double(), None, y=x.double())
    with pytest.raises(AssertionError):
        mqg.mqg_layer_norm(ctx, x, w, w[:7], y=x)
    with pytest.raises(AssertionError):
        mqg.mqg_layer_norm(ctx, x, w, residual=x.half(), y=x)
    with pytest.raises(AssertionError):
        mqg.mqg_layer_norm_backward(ctx, x, x, w, x, grad_bias=w[:7])
