"""Calls that move more than the memory-side cache holds have kernels of their own, which go past the caches: the same bits as the kernels of smaller calls on parts of the
same buffers, of every layout, type and alignment; and nothing outside the buffers is written.

Gradients of weight and bias are sums over all rows, which the workgroups share another way: against 64 bits, u = 2^-24, at most 400 additions in a row, 60 of the joins, and
101 of a unit value (as in test_gpu_layer_norm.py).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
SIZE = {F32: 4, F16: 2, BF16: 2, E4M3: 1}
LAYER_PAST, STEP_PAST = 256 << 20, 128 << 20
BLOCK = 128
EPS = 1e-5


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    assert torch.cuda.is_available()
    return m


@pytest.fixture(scope="module")
def ctx(mqg):
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    return mqg.Context(g, 1, [1])


def normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=F32).to(dtype)


def padded(rows, dim, dtype, pad, off):
    """A buffer of bytes of one, and rows of dim columns in it, `off` elements from its beginning and `pad` apart."""
    buf = torch.ones((off + rows * (dim + pad) + 16) * SIZE[dtype], dtype=torch.uint8, device="cuda")
    return buf, torch.as_strided(buf.view(dtype), (rows, dim), (dim + pad, 1), off)


def untouched(buf, t, off):
    seen = buf.view(t.dtype).view(torch.uint8).clone()
    torch.as_strided(seen.view(t.dtype), t.shape, t.stride(), off).view(torch.uint8 if SIZE[t.dtype] == 1 else torch.int16 if SIZE[t.dtype] == 2 else torch.int32).fill_(
        {1: 0x01, 2: 0x0101, 4: 0x01010101}[SIZE[t.dtype]])
    return bool((seen == 1).all())


# a dim of every layout: lanes of 4 to 64, one to four vectors of these, workgroups of 512 and 1,024
DIMS = {F32: [13, 30, 61, 127, 250, 500, 602, 1000, 2047, 4001, 8003, 16_383], F16: [31, 61, 127, 250, 500, 1000, 1500, 2001, 4099, 8003, 16_383]}
DIMS[BF16] = DIMS[F16]
ROWS = [(dtype, dim) for dtype in (F32, F16, BF16) for dim in DIMS[dtype]]


@pytest.mark.parametrize("dtype,dim", ROWS)
def test_layer_norm(mqg, ctx, dtype, dim):
    gen = torch.Generator(device="cuda").manual_seed(dim)
    rows = LAYER_PAST // (dim * (4 * SIZE[dtype] + 1)) + 5
    part = rows // 3 + 1                                                   # a third is below the border, and more than a few rows where the rows are
    pad, off = dim % 3, dim % 5
    x, r = normal(gen, (rows, dim), dtype), normal(gen, (rows, dim), dtype)
    x[7], r[7] = 3.0, 1.0
    w, b = 1 + 0.3 * normal(gen, (dim,), F32), normal(gen, (dim,), F32)
    sums, y, q = padded(rows, dim, dtype, pad, off), padded(rows, dim, dtype, pad, off), padded(rows, dim, E4M3, pad, off)
    scale = torch.zeros((rows, -(-dim // 32)), device="cuda")
    for group, kind in ((0, E4M3), (32, torch.int8)):
        mqg.mqg_layer_norm(ctx, x, w, b, residual=r, sum_out=sums[1], y=y[1], q=q[1].view(kind), q_scale=scale, group=group, eps=EPS)
        for at in range(0, rows, part):
            xx, rr = x[at:at + part], r[at:at + part]
            s2, y2 = torch.zeros_like(xx), torch.zeros_like(xx)
            q2, scale2 = torch.zeros(xx.shape, dtype=kind, device="cuda"), torch.zeros((xx.shape[0], scale.shape[1]), device="cuda")
            mqg.mqg_layer_norm(ctx, xx, w, b, residual=rr, sum_out=s2, y=y2, q=q2, q_scale=scale2, group=group, eps=EPS)
            torch.cuda.synchronize()
            groups = scale.shape[1] if group else 1
            assert torch.equal(sums[1][at:at + part], s2) and torch.equal(y[1][at:at + part], y2), (group, at)
            assert torch.equal(q[1][at:at + part].view(torch.uint8), q2.view(torch.uint8)) and torch.equal(scale[at:at + part, :groups], scale2[:, :groups]), (group, at)
    for buf, t in (sums, y, q):
        assert untouched(buf, t, off)


@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("dtype,dim", ROWS)
def test_layer_norm_backward(mqg, ctx, dtype, dim, residual):
    gen = torch.Generator(device="cuda").manual_seed(dim)
    arrays = 4 if residual else 3
    rows = LAYER_PAST // (dim * arrays * SIZE[dtype]) + 5
    part = rows // 3 + 1
    pad, off = dim % 3, dim % 5
    s, gy = normal(gen, (rows, dim), dtype), normal(gen, (rows, dim), dtype)
    gs = normal(gen, (rows, dim), dtype) if residual else None
    s[7] = 2.0
    w = 1 + 0.3 * normal(gen, (dim,), F32)
    gx = padded(rows, dim, dtype, pad, off)
    gw, gb = torch.zeros(dim, device="cuda"), torch.zeros(dim, device="cuda")
    mqg.mqg_layer_norm_backward(ctx, gy, s, w, gx[1], grad_weight=gw, grad_bias=gb, grad_sum=gs, eps=EPS)
    want = [torch.zeros(dim, dtype=torch.float64, device="cuda") for _ in range(4)]
    for at in range(0, rows, part):
        cut = slice(at, at + part)
        gx2 = torch.zeros_like(s[cut])
        mqg.mqg_layer_norm_backward(ctx, gy[cut], s[cut], w, gx2, grad_sum=gs[cut] if residual else None, eps=EPS)
        torch.cuda.synchronize()
        assert torch.equal(gx[1][cut], gx2), at
        g64, s64 = gy[cut].double(), s[cut].double()
        s64 -= s64.mean(1, keepdim=True)
        u64 = s64 / torch.sqrt(s64.square().mean(1, keepdim=True) + EPS)
        for t, add in zip(want, (g64 * u64, g64.abs() * (1 + u64.abs()), g64, g64.abs())):
            t += add.sum(0)
    assert untouched(*gx, off)
    assert bool(((gw.double() - want[0]).abs() <= (400 + 60 + 101) * U * want[1]).all())
    assert bool(((gb.double() - want[2]).abs() <= (400 + 60) * U * want[3]).all())
    again = [torch.zeros(dim, device="cuda") for _ in range(2)]
    mqg.mqg_layer_norm_backward(ctx, gy, s, w, s, grad_weight=again[0], grad_bias=again[1], grad_sum=gs, eps=EPS)      # in place
    torch.cuda.synchronize()
    assert torch.equal(s, gx[1]) and torch.equal(again[0], gw) and torch.equal(again[1], gb)


def blocks_of(n):
    return -(-n // BLOCK)


class Tensors:
    """A tensor with its gradient, moments and copy, each `off` elements into a buffer, and an equal one beside it."""

    def __init__(self, gen, n, weight, grad, bits, copy, off):
        state = E4M3 if bits == 8 else F32
        types = {"weight": weight, "grad": grad, "m": state, "v": state, "copy": copy}
        self.n, self.bits, self.off = n, bits, off
        self.bufs, self.t = {}, {}
        for k, dtype in types.items():
            if dtype:
                buf, t = padded(1, n, dtype, 0, off)
                self.bufs[k], self.t[k] = buf, t.view(-1)
        unit = torch.exp(normal(gen, (n,), F32))
        self.t["weight"].copy_(normal(gen, (n,), F32))
        self.t["grad"].copy_(0.01 * unit * normal(gen, (n,), F32))
        m, v = 0.003 * unit * normal(gen, (n,), F32), 1e-4 * (unit * normal(gen, (n,), F32)).square()
        if bits == 8:
            for k, x in (("m", m), ("v", v.sqrt())):
                blocks = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
                scale = (blocks.abs().amax(1) / 448).clamp(min=2.0 ** -126)
                self.t[k].copy_((blocks / scale.unsqueeze(1)).view(-1)[:n])
                self.bufs[k + "_scale"], t = padded(1, blocks_of(n), F32, 0, off)
                self.t[k + "_scale"] = t.view(-1)
                self.t[k + "_scale"].copy_(scale)
        else:
            self.t["m"].copy_(m)
            self.t["v"].copy_(v)
        self.same = {k: t.clone() for k, t in self.t.items()}

    def bytes(self):
        return sum(t.numel() * SIZE[t.dtype] * (1 if k in ("grad", "copy") else 2) for k, t in self.t.items() if not k.endswith("scale"))


def params_of(mqg, t, lo, hi):
    cut = {k: [x[lo // BLOCK:blocks_of(hi)] if k.endswith("scale") else x[lo:hi]] for k, x in t.items()}
    return mqg.Params(cut["weight"], cut["grad"], m=cut["m"], v=cut["v"], m_scale=cut.get("m_scale"), v_scale=cut.get("v_scale"), copies=cut.get("copy"))


PLAN = dict(lr=3e-3, step=5, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)


@pytest.mark.parametrize("off", [0, 1, 128])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("weight,grad,copy", [(F32, BF16, BF16), (F32, F32, None), (F32, F16, F16), (F32, BF16, F32), (BF16, BF16, None), (F16, F16, None), (BF16, F32, BF16)])
def test_adamw_step(mqg, ctx, weight, grad, copy, bits, off):
    gen = torch.Generator(device="cuda").manual_seed(off)
    each = 2 * SIZE[weight] + SIZE[grad] + (SIZE[copy] if copy else 0) + (4 if bits == 8 else 16)
    n = STEP_PAST // each + 77
    a = Tensors(gen, n, weight, grad, bits, copy, off)
    assert a.bytes() >= STEP_PAST
    scale = torch.full((1,), 0.37, device="cuda")
    mqg.mqg_adamw_step(ctx, params_of(mqg, a.t, 0, n), grad_scale=scale, **PLAN)
    part = n // 3 // BLOCK * BLOCK
    for lo in range(0, n, part):
        mqg.mqg_adamw_step(ctx, params_of(mqg, a.same, lo, min(n, lo + part)), grad_scale=scale, **PLAN)
    torch.cuda.synchronize()
    for k, t in a.t.items():
        assert torch.equal(t.view(torch.uint8), a.same[k].view(torch.uint8)), k
        assert untouched(a.bufs[k], t.view(1, -1), off), k


@pytest.mark.parametrize("off", [0, 3])
def test_adamw_step_of_more_than_2_to_the_31_elements_with_32_bit_moments(mqg, ctx, off):
    """A tensor that goes in two launches, each of which begins at a cache line of the weight; against steps of its parts."""
    n = (1 << 31) + 1000
    gen = torch.Generator(device="cuda").manual_seed(1)
    bufs = {k: torch.zeros(off + n + 64, dtype=t, device="cuda") for k, t in (("weight", BF16), ("grad", BF16), ("m", F32), ("v", F32))}
    chunk = 1 << 28
    for lo in range(0, n, chunk):
        hi = min(n, lo + chunk)
        for k, buf in bufs.items():
            x = torch.randn(hi - lo, generator=gen, device="cuda")
            buf[off + lo:off + hi] = x.square() if k == "v" else x
    t = {k: buf[off:off + n] for k, buf in bufs.items()}
    same = {k: x.clone() for k, x in t.items()}
    norm = torch.zeros(1, device="cuda")
    mqg.mqg_grad_norm(ctx, params_of(mqg, t, 0, n), norm=norm)
    mqg.mqg_adamw_step(ctx, params_of(mqg, t, 0, n), **PLAN)
    squares = 0.0
    part = 3 << 20                                                         # 72 MB a call: below the border
    for lo in range(0, n, part):
        mqg.mqg_adamw_step(ctx, params_of(mqg, same, lo, min(n, lo + part)), **PLAN)
    torch.cuda.synchronize()
    for lo in range(0, n, chunk):
        hi = min(n, lo + chunk)
        for k in t:
            assert torch.equal(t[k][lo:hi], same[k][lo:hi]), (k, lo)
        squares += float(t["grad"][lo:hi].float().square().sum(dtype=torch.float64))
    assert abs(float(norm) - math.sqrt(squares)) <= 10 * U * math.sqrt(squares)
    for buf in bufs.values():
        assert not bool(buf[:off].any()) and not bool(buf[off + n:].any())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("off", [0, 1])
def test_norm_of_gradients(mqg, ctx, dtype, off):
    """In one tensor and in many, above the border and below it: sixteen squares in fp32 lose 16 u of them, half of that in the root, and one rounding."""
    n = (256 << 20) // SIZE[dtype] + 99
    gen = torch.Generator(device="cuda").manual_seed(2)
    g = normal(gen, (off + n,), dtype)[off:]
    total = math.sqrt(sum(float(p.double().square().sum()) for p in g.split(1 << 26)))
    for grads in ([g], list(g.split(n // 400 + 1)), list(g.split(n // 3 + 1))):
        norm = torch.zeros(1, device="cuda")
        mqg.mqg_grad_norm(ctx, mqg.Params(grads=grads), norm=norm)
        torch.cuda.synchronize()
        assert abs(float(norm) - total) <= 10 * U * total
