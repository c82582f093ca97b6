"""Which buffers the norm and its backward write: inputs stay as they are, and every buffer that may be an input's gives the bits that separate ones give."""
import pytest
import torch

from test_gpu_norm import TYPES, Padded, filled

pytestmark = pytest.mark.gpu

EPS = 1e-6
# widths whose last vector repeats columns of the lane before, within a wavefront and between two, and whole ones
SHAPES = [(5, 3), (70, 33), (3, 250), (300, 602), (40, 1000), (7, 2049), (300, 3001), (4, 8191), (260, 8200), (300, 1024), (3, 16383)]


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    assert torch.cuda.is_available()
    return m


@pytest.fixture(scope="module")
def ctx(mqg):
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    return mqg.Context(g, 1, [1])


def copy_of(p):
    q = Padded(p.rows, p.dim, p.buf.dtype, p.stride - p.dim, p.off)
    q.buf.copy_(p.buf)
    return q


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", SHAPES)
def test_forward(mqg, ctx, rows, dim, dtype):
    gen = torch.Generator().manual_seed(dim)
    for pad, off in ((0, 0), (3, 1)):
        x, r = filled(rows, dim, dtype, gen, pad, off), filled(rows, dim, dtype, gen, pad, off)
        w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
        before = [t.clone() for t in (x.buf, r.buf, w)]
        s, y = Padded(rows, dim, dtype, pad, off), Padded(rows, dim, dtype, pad, off)
        q, scale = torch.zeros((rows, dim), dtype=torch.int8, device="cuda"), torch.zeros((rows, -(-dim // 32)), device="cuda")
        mqg.mqg_rms_norm(ctx, x.t, w, residual=r.t, sum_out=s.t, y=y.t, q=q, q_scale=scale, group=32, eps=EPS)
        torch.cuda.synchronize()
        for t, b in zip((x.buf, r.buf, w), before):
            assert torch.equal(t, b)
        for sum_in, y_in in (("x", "r"), ("r", "x"), ("x", None), (None, "x"), ("r", None), (None, "r")):
            a = {"x": copy_of(x), "r": copy_of(r), None: Padded(rows, dim, dtype, pad, off)}
            q2, scale2 = torch.zeros_like(q), torch.zeros_like(scale)
            mqg.mqg_rms_norm(ctx, a["x"].t, w, residual=a["r"].t, sum_out=a[sum_in].t, y=a[y_in].t, q=q2, q_scale=scale2, group=32, eps=EPS)
            torch.cuda.synchronize()
            assert torch.equal(a[sum_in].t, s.t) and torch.equal(a[y_in].t, y.t) and torch.equal(q2, q) and torch.equal(scale2, scale), (sum_in, y_in)
            assert all(p.untouched() for p in a.values())
            for name, was in (("x", x), ("r", r)):
                if name not in (sum_in, y_in):
                    assert torch.equal(a[name].buf, was.buf)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", SHAPES + [(9_000, 602), (2_000, 1001)])
def test_backward(mqg, ctx, rows, dim, dtype):
    gen = torch.Generator().manual_seed(dim + 1)
    for pad, off in ((0, 0), (3, 1)):
        ins = {k: filled(rows, dim, dtype, gen, pad, off) for k in ("gy", "s", "gs")}
        w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
        before = [t.clone() for t in [p.buf for p in ins.values()] + [w]]
        gx, gw = Padded(rows, dim, dtype, pad, off), torch.zeros(dim, device="cuda")
        mqg.mqg_rms_norm_backward(ctx, ins["gy"].t, ins["s"].t, w, gx.t, grad_weight=gw, grad_sum=ins["gs"].t, eps=EPS)
        torch.cuda.synchronize()
        for t, b in zip([p.buf for p in ins.values()] + [w], before):
            assert torch.equal(t, b)
        for place in ins:
            a = {k: copy_of(p) for k, p in ins.items()}
            again = torch.zeros_like(gw)
            mqg.mqg_rms_norm_backward(ctx, a["gy"].t, a["s"].t, w, a[place].t, grad_weight=again, grad_sum=a["gs"].t, eps=EPS)
            torch.cuda.synchronize()
            assert torch.equal(a[place].t, gx.t) and torch.equal(again, gw), place
            assert all(p.untouched() for p in a.values())
            for k, p in ins.items():
                if k != place:
                    assert torch.equal(a[k].buf, p.buf), (place, k)
