"""Mean aggregation of 8-bit source rows with scales, against the sum in 64 bits.

Tolerance.  Terms scale * q are exact to 2^-24 each (a fused multiply-add rounds the sum alone); a row of n entries is added in at most
n + 6 additions, so |error| <= (n + 8) 2^-24 sum |terms| / n, and half a unit of the output's type.
"""
import ctypes

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -140, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -130}
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


def block(mqg, rng, rows, fanout, sources, cap_rows=None):
    count = rng.integers(0, fanout + 1, rows)
    count[rng.random(rows) < 0.3] = 0
    if rows:
        count[-1] = fanout
    indptr = np.zeros((cap_rows or rows) + 1, np.int32)
    indptr[1:rows + 1] = np.cumsum(count)
    indptr[rows + 1:] = indptr[rows]
    indices = rng.integers(0, sources, max(1, int(indptr[rows]))).astype(np.int32)
    sizes = torch.tensor([rows, sources, int(indptr[rows]), 0], device="cuda")
    b = mqg.BlockView(torch.from_numpy(indptr).cuda(), torch.from_numpy(indices).cuda(), sizes, sources)
    return b, indptr, indices


def rows8(rng, sources, dim, kind, group, pad, off=0):
    width = group or dim
    groups = -(-dim // width)
    v = torch.from_numpy(rng.integers(-127, 128, (sources, dim))).to(torch.float32) * (1 if kind == torch.int8 else 448 / 127)
    buf = torch.zeros(off + sources * (dim + pad), dtype=torch.uint8, device="cuda").view(kind)
    q = torch.as_strided(buf, (sources, dim), (dim + pad, 1), off)
    q.copy_(v.to(kind))
    scale = torch.from_numpy(np.exp(rng.normal(size=(sources, groups + 1)))).float().cuda()
    return q, scale


def check(out, q, scale, indptr, indices, group, dtype):
    rows = out.shape[0]
    width = group or q.shape[1]
    wide = q.double().cpu() * scale.double().cpu().repeat_interleave(width, 1)[:, :q.shape[1]]
    got = out.double().cpu()
    for i in range(rows):
        terms = wide[indices[indptr[i]:indptr[i + 1]]]
        n = max(1, terms.shape[0])
        want = terms.sum(0) / n
        bound = (n + 8) * 2.0 ** -24 * terms.abs().sum(0) / n + UNIT[dtype] * 1.0001 * want.abs() + LEAST[dtype]
        assert bool(((got[i] - want).abs() <= bound).all()), i


@pytest.mark.parametrize("kind", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("dim", [1, 7, 16, 31, 33, 64, 100, 130, 256, 500, 602, 1024, 1030, 2100])
def test_against_the_sum(mqg, ctx, dim, kind):
    rng = np.random.default_rng(dim)
    for rows, fanout, sources, group, pad, dtype in [(1, 1, 3, 0, 0, torch.float32), (70, 25, 300, 0, -dim % 16, torch.float32),
                                                     (130, 9, 200, 32, 1, torch.float16), (33, 70, 500, 128, 3, torch.bfloat16),
                                                     (40, 3, 90, 64, -dim % 16, torch.float16)]:
        b, indptr, indices = block(mqg, rng, rows, fanout, sources)
        q, scale = rows8(rng, sources, dim, kind, group, pad, off=pad)
        buf = torch.full((rows + 1, dim + 3), MARK, device="cuda").to(dtype)
        out = buf[:rows, :dim]
        mqg.mqg_sage_mean_aggregate_q8(ctx, b, 0, q, scale, out, group=group)
        torch.cuda.synchronize()
        check(out, q, scale, indptr, indices, group, dtype)
        assert bool((buf[:, dim:] == MARK).all()) and bool((buf[rows:] == MARK).all())
        again = torch.zeros((rows, dim), dtype=dtype, device="cuda")
        mqg.mqg_sage_mean_aggregate_q8(ctx, b, 0, q, scale, again, group=group)
        torch.cuda.synchronize()
        assert torch.equal(again, out)


def test_rows_are_the_same_wherever_they_lie(mqg, ctx):
    rng = np.random.default_rng(3)
    q, scale = rows8(rng, 400, 100, torch.float8_e4m3fn, 0, 12)
    entries = rng.integers(0, 400, 23).astype(np.int32)
    outs = []
    for rows, at in ((1, 0), (50, 17), (3000, 2999)):
        count = rng.integers(0, 40, rows)
        count[at] = 23
        indptr = np.zeros(rows + 1, np.int32)
        indptr[1:] = np.cumsum(count)
        indices = rng.integers(0, 400, int(indptr[-1])).astype(np.int32)
        indices[indptr[at]:indptr[at + 1]] = entries
        b = mqg.BlockView(torch.from_numpy(indptr).cuda(), torch.from_numpy(indices).cuda(),
                          torch.tensor([rows, 400, int(indptr[-1]), 0], device="cuda"), 400)
        out = torch.zeros((rows, 100), device="cuda")
        mqg.mqg_sage_mean_aggregate_q8(ctx, b, 0, q, scale, out)
        outs.append(out[at].clone())
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_device_count_empty_blocks_and_scales_that_are_not_numbers(mqg, ctx):
    rng = np.random.default_rng(4)
    b, indptr, indices = block(mqg, rng, 60, 8, 50, cap_rows=80)
    for kind in (torch.float8_e4m3fn, torch.int8):
        q, scale = rows8(rng, 50, 96, kind, 32, 0)
        scale[7, 1] = float("nan")
        out = torch.full((80, 96), MARK, device="cuda")
        mqg.mqg_sage_mean_aggregate_q8(ctx, b, 0, q, scale, out, group=32)
        torch.cuda.synchronize()
        assert bool((out[60:] == MARK).all())
        reads = torch.tensor([7 in indices[indptr[i]:indptr[i + 1]] for i in range(60)], device="cuda")
        assert bool(reads.any()) and torch.equal(out[:60, 32:64].isnan().all(1), reads) and not bool(out[:60, :32].isnan().any())
        assert not bool(out[:60, 64:].isnan().any())
    none = mqg.BlockView(torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"),
                         torch.zeros(4, dtype=torch.int64, device="cuda"), 0)
    mqg.mqg_sage_mean_aggregate_q8(ctx, none, 0, q, scale, torch.zeros((0, 96), device="cuda"), group=32)
    torch.cuda.synchronize()


def test_offsets_beyond_32_bits(mqg, ctx):
    sources, dim = 9_000_000, 256                                  # 2.3 GB of rows
    q = torch.zeros((sources, dim), dtype=torch.int8, device="cuda")
    q[-1], q[0] = 5, 1
    scale = torch.ones((sources, 1), device="cuda")
    b = mqg.BlockView(torch.tensor([0, 2], dtype=torch.int32, device="cuda"), torch.tensor([0, sources - 1], dtype=torch.int32, device="cuda"),
                      torch.tensor([1, sources, 2, 0], device="cuda"), sources)
    out = torch.zeros((1, dim), device="cuda")
    mqg.mqg_sage_mean_aggregate_q8(ctx, b, 0, q, scale, out)
    torch.cuda.synchronize()
    assert bool((out == 3).all())


def test_what_the_norm_writes_is_what_the_aggregation_reads(mqg, ctx):
    """The two calls one after the other, against the fp32 aggregation of the values that the 8 bits stand for; and the existing backward."""
    rng = np.random.default_rng(6)
    dim, sources = 96, 700
    x = torch.randn((sources, dim), generator=torch.Generator().manual_seed(6)).cuda()
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    for kind, group in ((torch.float8_e4m3fn, 0), (torch.int8, 32)):
        b, indptr, indices = block(mqg, rng, 200, 12, sources)
        q = torch.zeros((sources, dim), dtype=kind, device="cuda")
        scale = torch.zeros((sources, -(-dim // group) if group else 1), device="cuda")
        mqg.mqg_rms_norm(ctx, x, None, q=q, q_scale=scale, group=group)
        out = torch.zeros((200, dim), device="cuda")
        mqg.mqg_sage_mean_aggregate_q8(ctx, b, 0, q, scale, out, group=group)
        torch.cuda.synchronize()
        check(out, q, scale, indptr, indices, group, torch.float32)
        values = q.float() * scale.repeat_interleave(group or dim, 1)[:, :dim]
        plain = torch.zeros_like(out)
        mqg.mqg_sage_mean_aggregate(ctx, b, 0, values, plain)
        torch.cuda.synchronize()
        assert float((plain - out).abs().max()) <= 20 * 2.0 ** -24 * float(values.abs().max())


def test_refusals(mqg, ctx):
    rng = np.random.default_rng(7)
    b, _, _ = block(mqg, rng, 5, 3, 9)
    q, scale = rows8(rng, 9, 40, torch.int8, 32, 0)
    out = torch.zeros((5, 40), device="cuda")

    def call(block=b.c[0], qp=q.data_ptr(), qs=40, qt=1, group=32, sp=scale.data_ptr(), ss=3, op=out.data_ptr(), os_=40, dim=40, dtype=0):
        return mqg.lib.mqg_sage_mean_aggregate_q8(ctx.h, ctypes.byref(block) if block is not None else None, qp, qs, qt, group, sp, ss, op, os_, dim, dtype, None)

    bad = mqg.MQG_ERR_INVALID_ARG
    assert call() == mqg.MQG_OK
    for wrong in (dict(block=None), dict(qp=None), dict(op=None), dict(sp=None), dict(qs=39), dict(os_=39), dict(ss=1), dict(qt=2), dict(group=33),
                  dict(group=-32), dict(dim=0), dict(dtype=3), dict(dtype=-1)):
        assert call(**wrong) == bad, wrong
    assert call(dim=(1 << 24) + 1, qs=1 << 25, os_=1 << 25, ss=1 << 25) == mqg.MQG_ERR_UNSUPPORTED
    empty = mqg.CBlock(5, 9, 3, None, None, None, None)
    assert call(block=empty) == bad
    assert mqg.lib.mqg_sage_mean_aggregate_q8(None, None, None, 0, 0, 0, None, 0, None, 0, 1, 0, None) == bad
    with pytest.raises(TypeError):
        mqg.mqg_sage_mean_aggregate_q8(ctx, b, 0, q.view(torch.uint8), scale, out, group=32)
    with pytest.raises(AssertionError):
        mqg.mqg_sage_mean_aggregate_q8(ctx, b, 0, q[:8], scale, out, group=32)
    with pytest.raises(AssertionError):
        mqg.mqg_sage_mean_aggregate_q8(ctx, b, 0, q, scale[:, :1], out, group=32)
    torch.cuda.synchronize()
