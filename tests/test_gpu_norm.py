"""Root-mean-square norm with the residual's addition, its output in 8 bits, and its backward, against the formulas in 64 bits.

Tolerances.  A value is computed in fp32 and rounded once to its type: half a unit of its last place (u = 2^-24, 2^-11, 2^-8
relative; fp16 below 2^-14: 2^-25 absolute) plus the error of the computation.  A row's sum of squares adds at most 32 terms in a lane
and 10 levels across lanes, so it is off by at most 45 * 2^-24; its root by half of that, and four more roundings follow: 32 * 2^-24 < 2e-6.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = 1e-6
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -140, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -130}
FP32 = 2e-6
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

    def untouched(self, rows=None):
        """Everything outside the first `rows` rows' columns still holds the mark."""
        rows = self.rows if rows is None else rows
        seen = torch.ones(self.buf.numel(), dtype=torch.bool, device="cuda")
        torch.as_strided(seen, (rows, self.dim), (self.stride, 1), self.off).fill_(False)
        return bool((self.buf.float()[seen] == MARK).all())


def filled(rows, dim, dtype, gen, pad=0, off=0, spread=0.0):
    p = Padded(rows, dim, dtype, pad, off)
    x = torch.randn((rows, dim), generator=gen)
    if spread:
        x *= torch.exp(spread * torch.randn((rows, 1), generator=gen))
    p.t.copy_(x.to(dtype))
    return p


def norm64(x, r, w):
    s = x.double().cpu()
    if r is not None:
        s = s + r.double().cpu()
    y = s / torch.sqrt((s * s).mean(1, keepdim=True) + EPS)
    return s, y if w is None else y * w.double().cpu()


def near(got, want, dtype, extra=FP32):
    got, want = got.double().cpu(), want
    return bool(((got - want).abs() <= (UNIT[dtype] * 1.0001 + extra) * want.abs() + LEAST[dtype]).all())


def half_unit(v, kind):
    """Half the distance between neighbouring 8-bit values around v (in scaled units)."""
    if kind == torch.int8:
        return torch.full_like(v, 0.5)
    _, e = torch.frexp(v)
    return torch.ldexp(torch.ones_like(v), (e - 1).clamp(min=-6) - 4)


def check_q(q, scale, y64, group, kind):
    top = 127.0 if kind == torch.int8 else 448.0
    dim = y64.shape[1]
    width = group or dim
    groups = -(-dim // width)
    padded = torch.nn.functional.pad(y64, (0, groups * width - dim)).view(-1, groups, width)
    want = (padded.abs().amax(2) / top).clamp(min=2.0 ** -126)
    got = scale[:, :groups].double().cpu()
    assert bool(((got - want).abs() <= (FP32 + 2.0 ** -23) * want).all())
    wide = got.repeat_interleave(width, 1)[:, :dim]
    v = y64 / wide
    # nearest: half a unit, and what the computation in fp32 is off by
    assert bool(((q.double().cpu() - v).abs() <= half_unit(v, kind) * (1 + 1e-6) + 4 * FP32 * v.abs()).all())
    assert float(q.double().abs().max()) <= top


DIMS = [1, 3, 16, 33, 64, 100, 127, 256, 257, 513, 602, 1025, 2049, 4100, 8192, 16384]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_rows_sum_and_8_bits(mqg, ctx, dim, dtype):
    gen = torch.Generator().manual_seed(dim)
    for rows, pad, off, residual, weighted, kind, group in [
            (1, 0, 0, True, True, torch.float8_e4m3fn, 128), (5, 3, 1, True, False, torch.int8, 0), (37, -dim % 16, 0, False, True, torch.float8_e4m3fn, 0),
            (67, 0, 1, True, True, torch.int8, 32), (67, 5, 3, False, False, torch.float8_e4m3fn, 64)]:
        x = filled(rows, dim, dtype, gen, pad, off, spread=1.0)
        r = filled(rows, dim, dtype, gen, pad, off) if residual else None
        w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda() if weighted else None
        s, y = Padded(rows, dim, dtype, pad, off), Padded(rows, dim, dtype, pad, off)
        qb = torch.full((rows + 1, dim + 3), 3, dtype=torch.uint8, device="cuda")
        q = qb.view(kind)[:rows, :dim]
        groups = -(-dim // group) if group else 1
        scale = torch.full((rows, groups + 1), MARK, device="cuda")
        mqg.mqg_rms_norm(ctx, x.t, w, residual=None if r is None else r.t, sum_out=s.t, y=y.t, q=q, q_scale=scale, group=group, eps=EPS)
        torch.cuda.synchronize()
        s64, y64 = norm64(x.t, None if r is None else r.t, w)
        assert near(s.t, s64, dtype), (rows, group)
        assert near(y.t, y64, dtype), (rows, group)
        check_q(q, scale, y64, group, kind)
        for p in (x, s, y) + ((r,) if r else ()):
            assert p.untouched() or p in (x, r)
        assert s.untouched() and y.untouched()
        assert bool((qb[:rows, dim:] == 3).all()) and bool((qb[rows:] == 3).all()) and bool((scale[:, groups:] == MARK).all())
        # each output alone is the same
        y2 = Padded(rows, dim, dtype, pad, off)
        mqg.mqg_rms_norm(ctx, x.t, w, residual=None if r is None else r.t, y=y2.t, eps=EPS)
        q2, scale2 = torch.zeros((rows, dim), dtype=torch.uint8, device="cuda"), torch.zeros((rows, groups), device="cuda")
        mqg.mqg_rms_norm(ctx, x.t, w, residual=None if r is None else r.t, q=q2.view(kind), q_scale=scale2, group=group, eps=EPS)
        torch.cuda.synchronize()
        assert torch.equal(y2.t, y.t) and torch.equal(q2, qb[:rows, :dim]) and torch.equal(scale2, scale[:, :groups])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", [(3000, 64), (1500, 256), (700, 602), (90_000, 16), (600, 2500), (5000, 8200)])
def test_many_rows_the_device_count_and_buffers_in_place(mqg, ctx, rows, dim, dtype):
    gen = torch.Generator().manual_seed(1)
    x = torch.randn((rows, dim), generator=gen).to(dtype).cuda()
    r = torch.randn((rows, dim), generator=gen).to(dtype).cuda()
    w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
    s64, y64 = norm64(x, r, w)
    y = torch.zeros_like(x)
    mqg.mqg_rms_norm(ctx, x, w, residual=r, y=y, eps=EPS)
    torch.cuda.synchronize()
    assert near(y, y64, dtype)
    for count, valid in ((rows * 2 // 3, rows * 2 // 3), (rows + 9, rows), (0, 0), (-4, 0)):
        a, b = x.clone(), r.clone()
        num = torch.tensor([count], device="cuda")
        mqg.mqg_rms_norm(ctx, a, w, residual=b, sum_out=b, y=a, eps=EPS, num_rows=num)
        torch.cuda.synchronize()
        assert torch.equal(a[:valid], y[:valid]) and torch.equal(a[valid:], x[valid:])
        assert near(b[:valid], s64[:valid], dtype) and torch.equal(b[valid:], r[valid:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [40, 300, 3000])
def test_rows_of_zeros_and_rows_that_are_not_finite(mqg, ctx, dim, dtype):
    rows = 12
    x = torch.randn((rows, dim), generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    x[1] = 0
    x[3, 5] = float("nan")
    x[5, 7] = float("inf")
    x[7, 11] = float("-inf")
    for kind in (torch.float8_e4m3fn, torch.int8):
        for group in (0, 32):
            y = torch.zeros_like(x)
            q = torch.zeros((rows, dim), dtype=torch.uint8, device="cuda").view(kind)
            scale = torch.zeros((rows, -(-dim // group) if group else 1), device="cuda")
            mqg.mqg_rms_norm(ctx, x, None, y=y, q=q, q_scale=scale, group=group, eps=EPS)
            torch.cuda.synchronize()
            assert bool((y[1] == 0).all()) and bool((q[1].float() == 0).all()) and bool((scale[1] == 2.0 ** -126).all())
            assert bool(y[3].isnan().all()) and bool(scale[3].isnan().all())
            for row, col in ((5, 7), (7, 11)):                     # infinity over infinity, and zeros elsewhere
                assert bool(y[row, col].isnan()) and int(y[row].isnan().sum()) == 1
                assert bool(scale[row, col // (group or dim)].isnan()) and int(scale[row].isnan().sum()) == 1
            fine = [0, 2, 4, 6, 8, 9, 10, 11]
            _, y64 = norm64(x[fine], None, None)
            assert near(y[fine], y64, dtype)
            check_q(q[fine], scale[fine], y64, group, kind)


def test_offsets_beyond_32_bits(mqg, ctx):
    stride, dim = (1 << 31) + 64, 100                              # elements between two rows
    buf = torch.zeros(stride + dim, dtype=torch.float16, device="cuda")
    x = torch.as_strided(buf, (2, dim), (stride, 1))
    x.copy_(torch.randn((2, dim), generator=torch.Generator().manual_seed(3)).half())
    y = torch.zeros((2, dim), dtype=torch.float16, device="cuda")
    gx = torch.zeros_like(y)
    mqg.mqg_rms_norm(ctx, x, None, y=y, eps=EPS)
    mqg.mqg_rms_norm_backward(ctx, y, x, None, gx, eps=EPS)
    want = torch.zeros_like(gx)
    mqg.mqg_rms_norm_backward(ctx, y, x.contiguous(), None, want, eps=EPS)
    torch.cuda.synchronize()
    assert near(y, norm64(x, None, None)[1], torch.float16) and torch.equal(gx, want)


# ---------------------------------------------------------------------------------------------- backward

def backward64(gy, s, w, gs):
    gy, s = gy.double().cpu(), s.double().cpu()
    dim = s.shape[1]
    r = 1 / torch.sqrt((s * s).mean(1, keepdim=True) + EPS)
    gw = gy if w is None else gy * w.double().cpu()
    gx = r * gw - s * r ** 3 * (gw * s).mean(1, keepdim=True)
    terms = r * gw.abs() + s.abs() * r ** 3 * (gw * s).abs().mean(1, keepdim=True)
    if gs is not None:
        gx, terms = gx + gs.double().cpu(), terms + gs.double().cpu().abs()
    return gx, terms, (gy * s * r).sum(0), (gy * s * r).abs().sum(0)


def check_backward(gx, gw, want, dtype, rows):
    gx64, terms, gw64, gw_terms = want
    # the means are off by 45 * 2^-24 of their terms' sizes, as the sum of squares is; four factors of R and four more roundings
    bound = (45 + 4 * 25 + 8) * 2.0 ** -24 * terms + UNIT[dtype] * 1.0001 * gx64.abs() + LEAST[dtype]
    assert bool(((gx.double().cpu() - gx64).abs() <= bound).all())
    if gw is not None:
        # a sum of `rows` terms, each off by 30 * 2^-24 of its size: no more than that many additions in a row
        assert bool(((gw.double().cpu() - gw64).abs() <= (min(rows, 400) + 60) * 2.0 ** -24 * gw_terms + 1e-30).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_backward(mqg, ctx, dim, dtype):
    gen = torch.Generator().manual_seed(100 + dim)
    for rows, pad, off, residual, weighted in [(1, 0, 0, True, True), (5, 3, 1, False, True), (67, -dim % 16, 0, True, False), (260, 1, 3, True, True)]:
        s, gy = filled(rows, dim, dtype, gen, pad, off, spread=1.0), filled(rows, dim, dtype, gen, pad, off)
        gs = filled(rows, dim, dtype, gen, pad, off) if residual else None
        w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda() if weighted else None
        gx, gw = Padded(rows, dim, dtype, pad, off), torch.full((dim,), MARK, device="cuda")
        mqg.mqg_rms_norm_backward(ctx, gy.t, s.t, w, gx.t, grad_weight=gw, grad_sum=None if gs is None else gs.t, eps=EPS)
        alone = Padded(rows, dim, dtype, pad, off)
        mqg.mqg_rms_norm_backward(ctx, gy.t, s.t, w, alone.t, grad_sum=None if gs is None else gs.t, eps=EPS)
        torch.cuda.synchronize()
        check_backward(gx.t, gw, backward64(gy.t, s.t, w, None if gs is None else gs.t), dtype, rows)
        assert gx.untouched() and torch.equal(gx.t, alone.t)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", [(90_000, 16), (20_000, 100), (9_000, 602), (3_000, 2500), (1_200, 8200)])
def test_backward_many_rows_and_the_device_count(mqg, ctx, rows, dim, dtype):
    gen = torch.Generator().manual_seed(4)
    s, gy, gs = (torch.randn((rows, dim), generator=gen).to(dtype).cuda() for _ in range(3))
    w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
    for count, valid in ((rows, rows), (rows - 77, rows - 77), (rows + 5, rows), (0, 0)):
        gx, gw, again = torch.full_like(s, MARK), torch.full((dim,), MARK, device="cuda"), torch.full((dim,), MARK, device="cuda")
        num = torch.tensor([count], device="cuda")
        mqg.mqg_rms_norm_backward(ctx, gy, s, w, gx, grad_weight=gw, grad_sum=gs, eps=EPS, num_rows=num)
        torch.cuda.synchronize()
        check_backward(gx[:valid], gw, backward64(gy[:valid], s[:valid], w, gs[:valid]), dtype, rows)
        assert bool((gx[valid:] == MARK).all())
        place = gs.clone()                                             # in place of the gradient that it adds
        mqg.mqg_rms_norm_backward(ctx, gy, s, w, place, grad_weight=again, grad_sum=place, eps=EPS, num_rows=num)
        torch.cuda.synchronize()
        assert torch.equal(again, gw) and torch.equal(place[:valid], gx[:valid])
    empty = torch.zeros((0, dim), dtype=dtype, device="cuda")
    gw.fill_(MARK)
    mqg.mqg_rms_norm_backward(ctx, empty, empty, w, empty, grad_weight=gw, eps=EPS)
    mqg.mqg_rms_norm(ctx, empty, w, y=empty, eps=EPS)
    torch.cuda.synchronize()
    assert bool((gw == 0).all())


def test_backward_against_differences(mqg, ctx):
    rows, dim = 6, 50
    gen = torch.Generator().manual_seed(5)
    s, gy, gs = (torch.randn((rows, dim), generator=gen) for _ in range(3))
    w = 1 + 0.3 * torch.randn(dim, generator=gen)
    gx, gw = torch.zeros((rows, dim), device="cuda"), torch.zeros(dim, device="cuda")
    mqg.mqg_rms_norm_backward(ctx, gy.cuda(), s.cuda(), w.cuda(), gx, grad_weight=gw, grad_sum=gs.cuda(), eps=EPS)
    torch.cuda.synchronize()

    def loss(s, w):
        y = s / torch.sqrt((s * s).mean(1, keepdim=True) + EPS) * w
        return float((gy.double() * y).sum() + (gs.double() * s).sum())

    h = 1e-5                                                       # the difference is off by h^2 of the third derivative, and 1e-15 / h
    for k in range(20):
        ds, dw = torch.randn((rows, dim), generator=gen).double(), torch.randn(dim, generator=gen).double()
        slope = (loss(s.double() + h * ds, w.double() + h * dw) - loss(s.double() - h * ds, w.double() - h * dw)) / (2 * h)
        got = float((gx.double().cpu() * ds).sum() + (gw.double().cpu() * dw).sum())
        size = float((gx.double().cpu() * ds).abs().sum() + (gw.double().cpu() * dw).abs().sum())
        assert abs(got - slope) <= 1e-5 * size


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [5, 64, 250, 1023, 4100, 8200])
def test_backward_of_a_few_rows(mqg, ctx, dim, dtype):
    """Rows that one workgroup takes by itself, the first that it does not, and device counts of less."""
    gen = torch.Generator().manual_seed(11)
    w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
    for rows in (1, 2, 3, 4, 5, 16, 17, 64, 65, 256, 257):
        s, gy, gs = (torch.randn((rows, dim), generator=gen).to(dtype).cuda() for _ in range(3))
        for count, valid in ((rows, rows), (rows // 2, rows // 2), (rows + 1, rows), (0, 0)):
            gx, gw = torch.full_like(s, MARK), torch.full((dim + 2,), MARK, device="cuda")
            mqg.mqg_rms_norm_backward(ctx, gy, s, w, gx, grad_weight=gw[1:-1], grad_sum=gs, eps=EPS, num_rows=torch.tensor([count], device="cuda"))
            torch.cuda.synchronize()
            check_backward(gx[:valid], gw[1:-1], backward64(gy[:valid], s[:valid], w, gs[:valid]), dtype, rows)
            assert bool((gx[valid:] == MARK).all()) and bool((gw[[0, -1]] == MARK).all())


# ---------------------------------------------------------------------------------------------- refusals

def test_refusals(mqg, ctx):
    x = torch.zeros((4, 8), device="cuda")
    w = torch.ones(8, device="cuda")
    q, scale = torch.zeros((4, 8), dtype=torch.int8, device="cuda"), torch.zeros((4, 1), device="cuda")

    def forward(xs=8, dim=8, dtype=0, eps=1e-6, rows=4, y=x.data_ptr(), qp=None, qs=8, qt=0, group=0, sp=scale.data_ptr(), ss=1, xp=x.data_ptr()):
        return mqg.lib.mqg_rms_norm(ctx.h, xp, xs, None, 0, w.data_ptr(), eps, None, rows, dim, dtype, None, 0, y, 8, qp, qs, qt, group, sp, ss, None)

    bad, limit = mqg.MQG_ERR_INVALID_ARG, mqg.MQG_ERR_UNSUPPORTED
    assert mqg.lib.mqg_rms_norm(None, None, 0, None, 0, None, 0.0, None, 0, 1, 0, None, 0, None, 0, None, 0, 0, 0, None, 0, None) == bad
    assert forward(xs=7) == bad and b"stride" in mqg.lib.mqg_last_error(ctx.h)
    assert forward(dim=0) == bad and forward(dtype=3) == bad and forward(rows=-1) == bad and forward(xp=None) == bad
    assert forward(eps=-1.0) == bad and forward(eps=float("nan")) == bad and forward(eps=float("inf")) == bad
    assert forward(y=None) == bad and b"neither" in mqg.lib.mqg_last_error(ctx.h)
    assert forward(dim=mqg.MQG_NORM_MAX_DIM + 1, xs=1 << 20) == limit
    qp = q.data_ptr()
    assert forward(qp=qp, qs=7) == bad and forward(qp=qp, qt=2) == bad and forward(qp=qp, group=16) == bad and forward(qp=qp, sp=None) == bad
    assert forward(qp=qp, ss=0) == bad

    def backward(strides=(8, 8, 8), dim=8, gx=x.data_ptr(), s=x.data_ptr(), eps=1e-6):
        return mqg.lib.mqg_rms_norm_backward(ctx.h, x.data_ptr(), strides[0], s, strides[1], w.data_ptr(), None, 0, eps, None, 4, dim, 0, gx,
                                             strides[2], None, None)

    for k in range(3):
        assert backward(strides=[7 if i == k else 8 for i in range(3)]) == bad
    assert backward(gx=None) == bad and backward(s=None) == bad and backward(eps=-1.0) == bad and backward(dim=0) == bad
    assert mqg.lib.mqg_rms_norm_backward(None, None, 0, None, 0, None, None, 0, 0.0, None, 0, 1, 0, None, 0, None, None) == bad
    with pytest.raises(TypeError):
        mqg.mqg_rms_norm(ctx, x.double(), None, y=x.double())
    with pytest.raises(AssertionError):
        mqg.mqg_rms_norm(ctx, x, w[:7], y=x)
    with pytest.raises(AssertionError):
        mqg.mqg_rms_norm(ctx, x, w, residual=x.half(), y=x)
    # the aggregation of rows in features' types keeps to those
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    b = mqg.Blocks(g, 1, [1])
    rows = torch.zeros((2, 8), device="cuda")
    import ctypes
    assert mqg.lib.mqg_sage_mean_aggregate(ctx.h, ctypes.byref(b.c[0]), rows.data_ptr(), 8, rows.data_ptr(), 8, 8, mqg.MQG_BF16, None) == bad
