"""The backward of few rows of few columns, whose shares the last workgroup adds: 5 to 32 workgroups, and 33, which have a launch of their own for it; one gradient or both, call after
call on one context, with what the device counts.

Tolerances as in test_gpu_layer_norm.py, u = 2^-24: sums of n rows are off by n + 60 u of their terms' sizes, unit values by 101 u more.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
EPS = 1e-5
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


def rows_of_a_workgroup(dim, dtype):
    """256 threads; a row has the least power of two of lanes, four at least, that hold it with 16 bytes each."""
    vecs = -(-dim // (4 if dtype == F32 else 8))
    lanes = 4
    while lanes < vecs:
        lanes *= 2
    return 256 // lanes


def sums64(gy, s):
    gy, s = gy.double().cpu(), s.double().cpu()
    d = s - s.mean(1, keepdim=True)
    u = d / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    return (gy * u).sum(0), (gy.abs() * (1 + u.abs())).sum(0), gy.sum(0), gy.abs().sum(0)


@pytest.mark.parametrize("groups", [5, 6, 31, 32, 33])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", [1, 3, 17, 64, 100, 127, 128, 129])
def test_call_after_call(mqg, ctx, dim, dtype, groups):
    each = rows_of_a_workgroup(dim, dtype)
    gen = torch.Generator().manual_seed(dim)
    w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
    for rows in ((groups - 1) * each + 1, groups * each):
        s, gy = (torch.randn((rows, dim), generator=gen).to(dtype).cuda() for _ in range(2))
        seen = {}
        for call, (weight, bias, count) in enumerate([(True, True, rows), (True, False, rows), (False, True, rows), (True, True, rows // 3), (False, True, rows // 3), (True, True, rows),
                                                      (True, True, 0), (True, False, rows // 3), (True, True, rows + 9), (False, True, rows)]):
            gx = torch.full_like(s, MARK)
            gw, gb = (torch.full((dim + 2,), MARK, device="cuda") for _ in range(2))
            mqg.mqg_layer_norm_backward(ctx, gy, s, w, gx, grad_weight=gw[1:-1] if weight else None, grad_bias=gb[1:-1] if bias else None, eps=EPS,
                                        num_rows=torch.tensor([count], device="cuda"))
            torch.cuda.synchronize()
            valid = min(count, rows)
            want = sums64(gy[:valid], s[:valid])
            got_w, got_b = gw[1:-1].double().cpu(), gb[1:-1].double().cpu()
            assert not weight or bool(((got_w - want[0]).abs() <= (valid + 161) * U * want[1]).all()), call
            assert not bias or bool(((got_b - want[2]).abs() <= (valid + 60) * U * want[3]).all()), call
            assert bool((gw[[0, -1]] == MARK).all()) and bool((gb[[0, -1]] == MARK).all()) and bool((gx[valid:] == MARK).all())
            assert (weight or bool((gw == MARK).all())) and (bias or bool((gb == MARK).all()))
            for k, t, there in (("gw", gw, weight), ("gb", gb, bias), ("gx", gx, True)):         # the same bits as the calls before, whatever else they wrote
                if there:
                    assert torch.equal(seen.setdefault((k, valid), t), t), (k, call)


def test_between_calls_of_the_norm_of_gradients(mqg, ctx):
    """Both count the workgroups that are done, on one context; recorded and replayed with other sizes between."""
    gen = torch.Generator().manual_seed(1)
    s, gy = (torch.randn((300, 64), generator=gen).cuda() for _ in range(2))
    grads = [torch.randn(n, generator=gen).cuda() for n in (20_000, 100, 9)]
    params = mqg.Params(grads=grads)
    total = float(torch.cat(grads).double().norm())
    outs = [[torch.zeros_like(s), torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda"), torch.zeros(1, device="cuda")] for _ in range(2)]

    def both(out):
        mqg.mqg_layer_norm_backward(ctx, gy, s, None, out[0], grad_weight=out[1], grad_bias=out[2], eps=EPS)
        mqg.mqg_grad_norm(ctx, params, norm=out[3])

    both(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        both(outs[1])
    for k in range(4):
        for t in outs[1]:
            t.fill_(MARK)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*outs)), k
        assert abs(float(outs[1][3]) - total) <= 10 * U * total
        mqg.mqg_layer_norm_backward(ctx, gy[:40 + 70 * k], s[:40 + 70 * k], None, torch.zeros_like(s[:40 + 70 * k]), grad_weight=torch.zeros(64, device="cuda"), eps=EPS)
        mqg.mqg_grad_norm(ctx, mqg.Params(grads=grads[:1 + k % 3]), norm=torch.zeros(1, device="cuda"))
        torch.cuda.synchronize()
