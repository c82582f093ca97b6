"""Matrices taller than wide and the weights' steps by every kernel of the products, against the same polynomial in 64 bits.

Tolerance as in test_gpu_orthogonal.py: step i adds 8 * 2^-22 |X_i| in Frobenius norm, which the polynomial makes at most D times as large, D the largest slope
between 0 and 1.21, above which no singular value gets; for the weights' step half as much again for the update's own rounding, and four roundings of the weights.
"""
import math

import pytest
import torch

from test_gpu_orthogonal import EPS, UNIT, USUAL, slope

pytestmark = pytest.mark.gpu

# mats, rows, cols: X by tiles of 64; of 128, a side of an odd number of them; the last tiles of a round (525 of 128) by single blocks; tiles of 256.
# G and B by single blocks, by tiles of 64, of 64, of 128
SIZES = [(3, 1300, 600), (3, 600, 1300), (1, 2200, 2100), (1, 2100, 2200), (1, 3200, 2688), (1, 2688, 3200), (1, 4090, 4000), (1, 4000, 4090)]


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    assert torch.cuda.is_available()
    return m


@pytest.fixture(scope="module")
def ctx(mqg):
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    return mqg.Context(g, 1, [1])


def orth64(u):
    """(result, bound of the error's Frobenius norm) of one matrix, on the GPU."""
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T.contiguous()
    x = x / (x.norm() + EPS)
    a, b, c = USUAL
    most, off = slope(USUAL, 1.21), 0.0
    for _ in range(5):
        off = (off + 8 * 2.0 ** -22 * float(x.norm())) * most
        g = x @ x.T.contiguous()
        x = a * x + (b * g + c * (g @ g)) @ x
    off += 8 * 2.0 ** -22 * float(x.norm())
    return (x.T if tall else x), off


class Guarded:
    """[mats, rows, cols] of a larger buffer of sevens: a row more per matrix and `pad` columns more per row."""

    def __init__(self, values, pad):
        mats, rows, cols = values.shape
        self.buf = torch.full((mats, rows + 1, cols + pad), 7.0, dtype=values.dtype, device="cuda")
        self.t = self.buf[:, :rows, :cols]
        self.t.copy_(values)

    def untouched(self):
        return bool((self.buf[:, self.t.shape[1]:] == 7).all()) and bool((self.buf[:, :, self.t.shape[2]:] == 7).all())


def inputs(mats, rows, cols, dtype, pad):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(mats + rows * 7 + cols)

    def noise(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    grad = noise(mats, rows, cols)
    for i in range(mats):
        grad[i] += noise(rows, 3) @ noise(3, cols)
    return Guarded(grad.to(dtype), pad), noise


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mats,rows,cols", SIZES)
def test_orthogonalised(mqg, ctx, mats, rows, cols, dtype):
    u, _ = inputs(mats, rows, cols, dtype, 3)
    out = Guarded(torch.zeros((mats, rows, cols), dtype=dtype, device="cuda"), 5)
    mqg.mqg_orthogonalize(ctx, u.t, out.t, eps=EPS)
    torch.cuda.synchronize()
    assert u.untouched() and out.untouched()
    for i in range(mats):
        want, off = orth64(u.t[i])
        err = float((out.t[i].double() - want).norm())
        assert err <= off + UNIT[dtype] * float(want.norm()), (i, err, off)


@pytest.mark.parametrize("dtype,nesterov", [(torch.float32, True), (torch.bfloat16, False)])
@pytest.mark.parametrize("mats,rows,cols", SIZES)
def test_steps_of_the_weights(mqg, ctx, mats, rows, cols, nesterov, dtype):
    lr, beta, decay, scale = 0.02, 0.9, 0.1, math.sqrt(max(1.0, rows / cols))
    g, noise = inputs(mats, rows, cols, dtype, 1)
    m, w = Guarded(0.5 * noise(mats, rows, cols), 3), Guarded(noise(mats, rows, cols), 5)
    g64, m64, w64 = g.t.double(), m.t.double(), w.t.double()
    mqg.mqg_muon_step(ctx, g.t, m.t, w.t, lr=lr, beta=beta, nesterov=nesterov, weight_decay=decay)
    torch.cuda.synchronize()
    assert g.untouched() and m.untouched() and w.untouched() and torch.equal(g.t.double(), g64)
    m64 = beta * m64 + g64
    assert bool(((m.t.double() - m64).abs() <= 3 * 2.0 ** -24 * (m64.abs() + g64.abs() + 1)).all())
    u64 = g64 + beta * m64 if nesterov else m64
    for i in range(mats):
        o, off = orth64(u64[i])
        want = (1 - lr * decay) * w64[i] - lr * scale * o
        err = float((w.t[i].double() - want).norm())
        assert err <= lr * scale * 1.5 * off + 4 * 2.0 ** -24 * float(want.norm() + w64[i].norm()), (i, err, off)
