"""Orthogonalised updates and the weights' step, against the same polynomial in 64 bits.

Tolerance.  Step i rounds X_i and what is made of it: c * 2^-22 of its Frobenius norm |X_i|, c = 8 for the terms that two f16 hold (2^-22), the
products of low terms that are left out (2^-22) and sums in fp32 in each of three products.  The polynomial takes a difference between two
matrices to one that is at most max |p'| = D times as large (D = a at 0 for the usual coefficients, 3.4445), so that the result is off by at most
c * 2^-22 * sum_i |X_i| D^(steps - i) in Frobenius norm, and by its own rounding to the output's type.
"""
import ctypes
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

USUAL = (3.4445, -4.775, 2.0315)
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
EPS = 1e-7


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    assert torch.cuda.is_available()
    return m


@pytest.fixture(scope="module")
def ctx(mqg):
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    return mqg.Context(g, 1, [1])


def slope(k, r):
    a, b, c = k
    t = torch.linspace(0, r, 2001, dtype=torch.float64) ** 2
    return float((a + 3 * b * t + 5 * c * t * t).abs().max())


def orth64(u, coeffs, eps=EPS):
    """(result, bound of the error's Frobenius norm) of one matrix."""
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T
    x = x / (x.norm() + eps)
    off = 0.0
    for k in coeffs:
        r = float(torch.linalg.matrix_norm(x, 2)) if x.numel() else 0.0
        off = (off + 8 * 2.0 ** -22 * float(x.norm())) * max(slope(k, max(1.0, r)), 1.0)
        g = x @ x.T
        x = k[0] * x + (k[1] * g + k[2] * g @ g) @ x
    off += 8 * 2.0 ** -22 * float(x.norm())
    return (x.T if tall else x), off


def check(got, u, dtype, coeffs):
    want, off = orth64(u.cpu(), coeffs)
    err = float((got.double().cpu() - want).norm())
    bound = off + UNIT[dtype] * float(want.norm()) + 2.0 ** -25 * math.sqrt(want.numel())
    assert err <= bound, (tuple(u.shape), err, bound)
    return want


SIZES = [(1, 1), (1, 9), (9, 1), (5, 3), (16, 16), (17, 40), (64, 64), (33, 130), (130, 33), (128, 128), (129, 257), (300, 100), (256, 602), (520, 520), (700, 150)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_matrices_of_all_shapes(mqg, ctx, rows, cols, dtype):
    gen = torch.Generator().manual_seed(rows * 1000 + cols)
    for mats, pad in ((1, 0), (3, 5)):
        buf = torch.zeros((mats, rows + 1, cols + pad), dtype=dtype, device="cuda")
        u = buf[:, :rows, :cols]
        u.copy_((1e-3 * torch.randn((mats, rows, cols), generator=gen)).to(dtype))
        whole = torch.full((mats, rows + 1, cols + pad), 7.0, device="cuda").to(dtype)
        out = whole[:, :rows, :cols]
        mqg.mqg_orthogonalize(ctx, u, out, eps=EPS)
        torch.cuda.synchronize()
        for i in range(mats):
            check(out[i], u[i], dtype, [USUAL] * 5)
        assert bool((whole[:, rows:] == 7).all()) and bool((whole[:, :, cols:] == 7).all())
    if mats > 1:                                                       # one matrix alone is the same, and in its own place
        alone = u[1].clone()
        mqg.mqg_orthogonalize(ctx, alone, alone, eps=EPS)
        torch.cuda.synchronize()
        assert torch.equal(alone, out[1])


@pytest.mark.parametrize("rows,cols", [(100, 300), (300, 100), (200, 200)])
def test_singular_values_of_a_known_matrix(mqg, ctx, rows, cols):
    """Singular vectors are kept and every singular value goes through the polynomial: from a matrix built from them."""
    gen = torch.Generator().manual_seed(9)
    n = min(rows, cols)
    a, _ = torch.linalg.qr(torch.randn((rows, n), generator=gen, dtype=torch.float64))
    b, _ = torch.linalg.qr(torch.randn((cols, n), generator=gen, dtype=torch.float64))
    sigma = torch.exp(-torch.arange(n, dtype=torch.float64) * 6 / n)
    u = (a * sigma) @ b.T
    x = sigma / (sigma.norm() + EPS)
    for _ in range(5):
        x = USUAL[0] * x + USUAL[1] * x ** 3 + USUAL[2] * x ** 5
    out = torch.zeros((rows, cols), device="cuda")
    mqg.mqg_orthogonalize(ctx, u.float().cuda(), out, eps=EPS)
    torch.cuda.synchronize()
    _, off = orth64(u, [USUAL] * 5)
    assert float((out.double().cpu() - (a * x) @ b.T).norm()) <= off + 2 * 2.0 ** -24 * 3.4445 ** 5
    found = torch.linalg.svdvals(out.double().cpu())
    assert float(found.max()) < 1.21


def test_steps_and_coefficients(mqg, ctx):
    u = torch.randn((90, 140), generator=torch.Generator().manual_seed(10)).cuda()
    for coeffs in ([(1.5, -0.5, 0.0)] * 12, [(3.0, -16 / 5, 6 / 5)] * 3, [(2.0, -1.5, 0.5), (1.875, -1.25, 0.375)], [(4.0, 0.0, 0.0)], [(0.5, 0.0, 0.0)] * 3,
                   [(3.4445, -4.775, 2.0315)]):
        out = torch.zeros_like(u)
        mqg.mqg_orthogonalize(ctx, u, out, steps=len(coeffs), coeffs=coeffs, eps=EPS)
        torch.cuda.synchronize()
        check(out, u, torch.float32, coeffs)


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e15, 1e30])
def test_updates_of_any_size(mqg, ctx, size):
    u = (size * torch.randn((60, 50), generator=torch.Generator().manual_seed(11), dtype=torch.float64)).float().cuda()
    out = torch.zeros_like(u)
    mqg.mqg_orthogonalize(ctx, u, out, eps=0.0 if size < 1e-6 else EPS)
    torch.cuda.synchronize()
    want, off = orth64(u.cpu(), [USUAL] * 5, 0.0 if size < 1e-6 else EPS)
    assert float((out.double().cpu() - want).norm()) <= off + 1e-6


def test_zeros_and_values_that_are_not_finite(mqg, ctx):
    u = torch.randn((4, 70, 50), generator=torch.Generator().manual_seed(12)).cuda()
    u[0] = 0
    u[1, 3] = 0
    u[1, :, 8] = 0
    u[2, 4, 4] = float("nan")
    u[3, 5, 5] = float("inf")
    out = torch.zeros_like(u)
    mqg.mqg_orthogonalize(ctx, u, out, eps=EPS)
    torch.cuda.synchronize()
    assert bool((out[0] == 0).all())
    check(out[1], u[1], torch.float32, [USUAL] * 5)
    assert bool((out[1, 3] == 0).all()) and bool((out[1, :, 8] == 0).all())
    assert not bool(out[2:].isfinite().any())


def test_a_deterministic_result_on_another_stream_and_after_other_sizes(mqg, ctx):
    u = torch.randn((2, 200, 333), generator=torch.Generator().manual_seed(13)).cuda()
    first, other, again = torch.zeros_like(u), torch.zeros((40, 1000), device="cuda"), torch.zeros_like(u)
    mqg.mqg_orthogonalize(ctx, u, first)
    mqg.mqg_orthogonalize(ctx, torch.randn_like(other), other)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mqg.mqg_orthogonalize(ctx, u, again, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(first, again)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("rows,cols", [(1, 5), (30, 44), (256, 120), (128, 256)])
def test_steps_of_the_weights(mqg, ctx, rows, cols, nesterov, dtype):
    gen = torch.Generator().manual_seed(14)
    lr, beta, decay = 0.02, 0.9, 0.1
    scale = math.sqrt(max(1.0, rows / cols))
    for shape, pad in (((rows, cols), 0), ((2, rows, cols), 3)):
        def padded(t):
            buf = torch.full(tuple(shape[:-1]) + (cols + pad,), 7.0, device="cuda").to(t.dtype)
            buf[..., :cols] = t.cuda()
            return buf, buf[..., :cols]
        gbuf, g = padded(torch.randn(shape, generator=gen).to(dtype))
        mbuf, m = padded(torch.randn(shape, generator=gen))
        wbuf, w = padded(torch.randn(shape, generator=gen))
        for step in range(3):
            g64, m64, w64 = g.double().cpu(), m.double().cpu(), w.double().cpu()
            mqg.mqg_muon_step(ctx, g, m, w, lr=lr, beta=beta, nesterov=nesterov, weight_decay=decay)
            torch.cuda.synchronize()
            m64 = beta * m64 + g64
            assert bool(((m.double().cpu() - m64).abs() <= 3 * 2.0 ** -24 * (m64.abs() + g64.abs() + 1)).all())
            u64 = g64 + beta * m64 if nesterov else m64
            for i, (got, u, before) in enumerate(zip(w.view(-1, rows, cols) if pad == 0 else w, u64.reshape(-1, rows, cols), w64.reshape(-1, rows, cols))):
                o, off = orth64(u, [USUAL] * 5)
                want = (1 - lr * decay) * before - lr * scale * o
                # the update itself is off by the rounding of its two products and sums: 4 * 2^-24 of it, through the polynomials as a step's error is
                off = off * 1.5
                err = float((got.double().cpu() - want).norm())
                assert err <= lr * scale * off + 4 * 2.0 ** -24 * float(want.norm() + before.norm())
        assert bool((gbuf[..., cols:] == 7).all()) and bool((mbuf[..., cols:] == 7).all()) and bool((wbuf[..., cols:] == 7).all())


def test_recorded_and_replayed_beside_eager_calls(mqg):
    gr = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    ctx = mqg.Context(gr, 1, [1])
    gen = torch.Generator().manual_seed(15)
    rows, cols, n = 96, 160, 300
    grad, w0 = torch.randn((rows, cols), generator=gen).cuda(), torch.randn((rows, cols), generator=gen).cuda()
    x, gy = torch.randn((n, 64), generator=gen).cuda(), torch.randn((n, 64), generator=gen).cuda()
    weight = torch.ones(64, device="cuda")
    state = [torch.zeros_like(grad), w0.clone(), torch.zeros_like(x), torch.zeros_like(x), torch.zeros(64, device="cuda")]

    def step(c, m, w, y, gx, gw):
        mqg.mqg_rms_norm(c, x, weight, y=y)
        mqg.mqg_rms_norm_backward(c, gy, x, weight, gx, grad_weight=gw)
        mqg.mqg_muon_step(c, grad, m, w, lr=0.05)

    eager = mqg.Context(gr, 1, [1])
    want = [t.clone() for t in state]
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with pytest.raises(mqg.MqgError) as refused:                    # nothing is allocated while a stream is recorded
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=side):
            step(ctx, *state)
    assert refused.value.code == mqg.MQG_ERR_UNSUPPORTED
    torch.cuda.synchronize()
    ctx.reserve_layer(norm_dim=64, num_mats=1, rows=rows, cols=cols)
    with torch.cuda.graph(graph, stream=side):
        step(ctx, *state)
    for t, f in zip(state, want):
        t.copy_(f)
    for k in range(4):
        x.add_(0.1 * k)
        graph.replay()
        step(eager, *want)
        torch.cuda.synchronize()
        for t, f in zip(state, want):
            assert torch.equal(t, f), k


def test_refusals(mqg, ctx):
    u, f16 = torch.zeros((2, 6, 4), device="cuda"), torch.zeros((2, 6, 4), device="cuda").half()
    good = mqg._matrices(u)
    bad, limit = mqg.MQG_ERR_INVALID_ARG, mqg.MQG_ERR_UNSUPPORTED

    def orth(a=good, b=good, plan=None):
        r = lambda s: ctypes.byref(s) if s is not None else None  # noqa: E731
        return mqg.lib.mqg_orthogonalize(ctx.h, r(a), r(b), r(plan), None)

    def changed(**kw):
        m = mqg._matrices(u)
        for k, v in kw.items():
            setattr(m, k, v)
        return m

    assert orth() == mqg.MQG_OK
    assert mqg.lib.mqg_orthogonalize(None, None, None, None, None) == bad
    assert orth(a=None) == bad and orth(b=None) == bad
    for wrong in (dict(rows=-1), dict(cols=-1), dict(num_mats=-1), dict(dtype=3), dict(data=None), dict(row_stride=3), dict(mat_stride=23)):
        assert orth(a=changed(**wrong)) == bad and orth(b=changed(**wrong)) == bad, wrong
    assert orth(b=changed(rows=5)) == bad and b"different sizes" in mqg.lib.mqg_last_error(ctx.h)
    big = dict(rows=mqg.MQG_ORTH_MAX_SIDE + 1, mat_stride=1 << 40)
    assert orth(a=changed(**big), b=changed(**big)) == limit
    assert orth(plan=mqg.COrth(0, 0.0, None)) == bad and orth(plan=mqg.COrth(33, 0.0, None)) == bad
    assert orth(plan=mqg.COrth(5, -1.0, None)) == bad and orth(plan=mqg.COrth(5, float("nan"), None)) == bad
    for k in ((300.0, 0.0, 0.0), (float("nan"), 0.0, 0.0), (1.0, 1e9, 0.0), (float("inf"), 0.0, 0.0)):
        assert orth(plan=mqg._orth(1, k, 0.0)) == limit, k
    assert orth(plan=mqg._orth(20, (3.4445, 4.775, 2.0315), 0.0)) == limit      # each step makes them larger
    empty = changed(num_mats=0, data=None)
    assert orth(a=empty, b=empty) == mqg.MQG_OK

    m, w, g = (torch.zeros((6, 4), device="cuda") for _ in range(3))

    def muon(grad=g, mom=m, weight=w, lr=0.1, beta=0.9, decay=0.0, scale=1.0):
        cs = [mqg._matrices(t) for t in (grad, mom, weight)]
        return mqg.lib.mqg_muon_step(ctx.h, *[ctypes.byref(c) for c in cs], lr, beta, 1, decay, scale, None, None)

    assert muon() == mqg.MQG_OK
    assert muon(mom=m.half()) == bad and b"MQG_F32" in mqg.lib.mqg_last_error(ctx.h) and muon(weight=w.bfloat16()) == bad
    for k in ("lr", "beta", "decay", "scale"):
        assert muon(**{k: float("nan")}) == bad and muon(**{k: float("inf")}) == bad
    assert mqg.lib.mqg_muon_step(ctx.h, ctypes.byref(good), None, ctypes.byref(good), 0.1, 0.9, 1, 0.0, 1.0, None, None) == bad
    assert mqg.lib.mqg_ctx_reserve_layer(None, 0, 0, 0, 0) == bad and mqg.lib.mqg_ctx_reserve_layer(ctx.h, -1, 0, 0, 0) == bad
    assert mqg.lib.mqg_ctx_reserve_layer(ctx.h, mqg.MQG_NORM_MAX_DIM + 1, 0, 0, 0) == limit
    with pytest.raises(AssertionError):
        mqg.mqg_orthogonalize(ctx, u, f16[:1])
    with pytest.raises(AssertionError):
        mqg.mqg_orthogonalize(ctx, u, u.transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(TypeError):
        mqg.mqg_orthogonalize(ctx, u.double(), u.double())
    with pytest.raises(AssertionError):
        mqg.mqg_orthogonalize(ctx, u, u, steps=2, coeffs=[(1.5, -0.5, 0.0)] * 3)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mats,rows,cols", [(1, 70, 900), (3, 900, 70), (1, 40, 700), (2, 700, 40), (1, 128, 4000), (1, 4000, 100), (40, 128, 1000), (9, 100, 130), (500, 20, 30),
                                            (1, 1, 3000), (3, 100, 160), (1, 160, 96), (1, 1030, 1100), (3, 600, 1300), (1, 2200, 2200), (4, 2000, 2040), (1, 4000, 4090)])
def test_matrices_by_every_kernel(mqg, ctx, mats, rows, cols, dtype):
    """One launch, few rows or columns, single blocks, tiles of 64, of 128 and of 256 and the last tiles of a round."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(mats + rows * 7 + cols)
    u = torch.randn((mats, rows, cols), generator=gen, device="cuda") + torch.randn((mats, rows, 3), generator=gen, device="cuda") @ torch.randn((mats, 3, cols), generator=gen, device="cuda")
    u = u.to(dtype)
    out = torch.full_like(u, 7.0)
    mqg.mqg_orthogonalize(ctx, u, out, eps=EPS)
    torch.cuda.synchronize()
    for i in sorted({0, mats // 2, mats - 1}):
        want, off = orth64(u[i], [USUAL] * 5)
        err = float((out[i].double() - want).norm())
        assert err <= off + UNIT[dtype] * float(want.norm()), (i, err, off)
