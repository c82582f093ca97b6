"""Infinities in the mean aggregation of 8-bit rows: what the sum in 64 bits has, and what leaves 32 bits on its way."""
import numpy as np
import pytest
import torch

from test_gpu_aggregate_q8 import block

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    assert torch.cuda.is_available()
    return m


@pytest.fixture(scope="module")
def ctx(mqg):
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    return mqg.Context(g, 1, [1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("kind", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("dim,group", [(5, 0), (64, 32), (100, 0), (602, 128), (1030, 0)])
def test_infinite_scales(mqg, ctx, dim, group, kind, dtype):
    rng = np.random.default_rng(dim)
    rows, sources, fanout = 90, 60, 14
    b, indptr, indices = block(mqg, rng, rows, fanout, sources)
    q = torch.from_numpy(rng.integers(-3, 4, (sources, dim))).float().cuda().to(kind)       # (zeros among them: 0 times infinity is no number)
    scale = torch.from_numpy(np.exp(rng.normal(size=(sources, -(-dim // (group or dim)))))).float().cuda()
    scale[rng.permutation(sources)[:8]] = INF
    scale[rng.permutation(sources)[:4]] = -INF
    out = torch.full((rows, dim), 7.0, device="cuda").to(dtype)
    mqg.mqg_sage_mean_aggregate_q8(ctx, b, 0, q, scale, out, group=group)
    torch.cuda.synchronize()
    wide = q.double().cpu() * scale.double().cpu().repeat_interleave(group or dim, 1)[:, :dim]
    seen = set()
    for i in range(rows):
        n = indptr[i + 1] - indptr[i]
        want = wide[indices[indptr[i]:indptr[i + 1]]].sum(0) / max(n, 1)
        got = out[i].double().cpu()
        assert torch.equal(got.isnan(), want.isnan()), i
        for v in (INF, -INF):
            assert torch.equal(got == v, want == v), i
            if bool((want == v).any()):
                seen.add(v)
        fine = want.isfinite()
        assert bool(((got - want)[fine].abs() <= 2.0 ** -7 * (want[fine].abs() + 20)).all())
    assert seen == {INF, -INF}


def test_sums_that_leave_32_bits(mqg, ctx):
    indptr = torch.tensor([0, 1, 3, 6, 6, 8], dtype=torch.int32, device="cuda")
    indices = torch.tensor([0, 0, 0, 1, 1, 1, 0, 1], dtype=torch.int32, device="cuda")
    b = mqg.BlockView(indptr, indices, torch.tensor([5, 2, 8, 0], device="cuda"), 2)
    q = torch.tensor([[100], [-100]], dtype=torch.int8, device="cuda").expand(2, 40).contiguous()
    scale = torch.full((2, 1), 3e36, device="cuda")
    out = torch.zeros((5, 40), device="cuda")
    mqg.mqg_sage_mean_aggregate_q8(ctx, b, 0, q, scale, out)
    torch.cuda.synchronize()
    assert bool(((out[0].double() - 3e38).abs() <= 2.0 ** -22 * 3e38).all())
    assert bool((out[1] == INF).all()) and bool((out[2] == -INF).all()) and bool((out[3] == 0).all())
    # the sum of a number and its opposite: the first is rounded, the second is added as it is (n + 8 roundings of the terms' sizes, as in test_gpu_aggregate_q8.py)
    assert bool((out[4].abs() <= 10 * 2.0 ** -24 * 3e38).all())
