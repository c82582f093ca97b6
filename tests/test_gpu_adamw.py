"""The norm of all gradients and the AdamW step of many tensors, against the formulas in 64 bits.

Tolerances, u = 2^-24 (half a unit of fp32's last place).  m is two products and a sum with two rounded coefficients and, where gradients are scaled, a
rounded product before: 4 u of its terms; v, whose terms are all positive, 5 u, its root 4 u; the divisor 4 + 3 u; the step, with its rounded size, product and
quotient, 7 + 3 u and what m is off by; the weight's kept part u.  Each result is rounded once to its type: 2^-24, 2^-11, 2^-8 relative.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
UNIT = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
LEAST = {F32: 2.0 ** -140, F16: 2.0 ** -25, BF16: 2.0 ** -130}
TYPES = [F32, F16, BF16]
BLOCK = 128
MARK = 3.0


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    assert torch.cuda.is_available()
    return m


def context(mqg):
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    return mqg.Context(g, 1, [1])


@pytest.fixture(scope="module")
def ctx(mqg):
    return context(mqg)


class Guarded:
    """n elements `off` elements into a buffer filled with a mark (bytes of one for 8 bits)."""

    def __init__(self, n, dtype, off=0, values=None):
        self.n, self.off = n, off
        if dtype == E4M3:
            self.buf = torch.ones(off + n + 40, dtype=torch.uint8, device="cuda")
            self.t = self.buf[off:off + n].view(E4M3)
        else:
            self.buf = torch.full((off + n + 40,), MARK, device="cuda").to(dtype)
            self.t = self.buf[off:off + n]
        self.t.copy_(torch.zeros(n) if values is None else values.to(dtype))

    def untouched(self):
        rest = torch.cat([self.buf[:self.off], self.buf[self.off + self.n:]])
        return bool((rest == (1 if rest.dtype == torch.uint8 else MARK)).all())


def blocks_of(n):
    return -(-n // BLOCK)


def spread_out(scale, n):
    return scale.repeat_interleave(BLOCK)[:n]


def quantised(x, least=0.0):
    """e4m3 values and scales of a flat tensor."""
    n = x.numel()
    flat = torch.nn.functional.pad(x.float(), (0, -n % BLOCK)).view(-1, BLOCK)
    scale = (flat.abs().amax(1) / 448).clamp(min=2.0 ** -126)
    q = (flat / scale.unsqueeze(1)).view(-1)[:n]
    return torch.where((q > 0) & (q < least), torch.full_like(q, least), q).to(E4M3), scale


class Case:
    """One tensor with its gradient, moments and copy, and what a step makes of them in 64 bits."""

    def __init__(self, n, gen, weight=F32, grad=F32, bits=32, copy=None, off=0, lr_scale=1.0, decay_scale=1.0, fresh=False):
        rand = lambda: torch.randn(n, generator=gen)  # noqa: E731
        unit = torch.exp(rand())
        self.n, self.bits, self.lr_scale, self.decay_scale = n, bits, float(torch.tensor(lr_scale)), decay_scale
        self.weight = Guarded(n, weight, off, rand())
        self.grad = Guarded(n, grad, off, 0.01 * unit * rand() * (torch.rand(n, generator=gen) > 0.1))
        self.copy = Guarded(n, copy, off) if copy else None
        m, v = 0.003 * unit * rand(), 1e-4 * unit * unit * torch.rand(n, generator=gen)
        if fresh:
            m, v = torch.zeros(n), torch.zeros(n)
        if bits == 8:
            (m, ms), (v, vs) = quantised(m), quantised(v.sqrt(), 2.0 ** -9)
            self.m_scale, self.v_scale = Guarded(blocks_of(n), F32, off, ms), Guarded(blocks_of(n), F32, off, vs)
        self.m, self.v = (Guarded(n, E4M3 if bits == 8 else F32, off, t) for t in (m, v))

    def buffers(self):
        return [b for b in (self.weight, self.grad, self.copy, self.m, self.v, getattr(self, "m_scale", None), getattr(self, "v_scale", None)) if b]

    def moments64(self):
        m, v = self.m.t.double().cpu(), self.v.t.double().cpu()
        if self.bits == 8:
            return m * spread_out(self.m_scale.t.double().cpu(), self.n), (v * spread_out(self.v_scale.t.double().cpu(), self.n)) ** 2
        return m, v

    def expect(self, lr, step, beta1, beta2, eps, decay, scale=1.0):
        lr = lr * self.lr_scale
        g, w = scale * self.grad.t.double().cpu(), self.weight.t.double().cpu()
        m0, v0 = self.moments64()
        self.m64, self.v64 = beta1 * m0 + (1 - beta1) * g, beta2 * v0 + (1 - beta2) * g * g
        self.m_off = 4 * U * ((beta1 * m0).abs() + ((1 - beta1) * g).abs()) + 1e-44
        under = (self.v64 / (1 - beta2 ** step)).sqrt() + eps
        size = lr / (1 - beta1 ** step)
        change = torch.where(under == 0, torch.zeros_like(under), size * self.m64 / under)
        off = torch.where(under == 0, torch.zeros_like(under), abs(size) / under * (self.m_off + 17 * U * self.m64.abs()))
        self.w64 = w * (1 - lr * decay * self.decay_scale) - change
        self.w_off = 2 * U * w.abs() + off

    def check(self):
        dtype = self.weight.t.dtype
        got = self.weight.t.double().cpu()
        assert bool(((got - self.w64).abs() <= UNIT[dtype] * 1.0001 * self.w64.abs() + self.w_off + LEAST[dtype]).all())
        if self.copy:
            dtype = self.copy.t.dtype
            got = self.copy.t.double().cpu()
            assert bool(((got - self.w64).abs() <= UNIT[dtype] * 1.0001 * self.w64.abs() + self.w_off + LEAST[dtype]).all())
        if self.bits == 32:
            assert bool(((self.m.t.double().cpu() - self.m64).abs() <= self.m_off).all())
            assert bool(((self.v.t.double().cpu() - self.v64).abs() <= 5 * U * self.v64 + 1e-44).all())
        else:
            self.check8(self.m.t, self.m_scale.t, self.m64, self.m_off, 0.0)
            root = self.v64.sqrt()
            self.check8(self.v.t, self.v_scale.t, root, 4 * U * root + 1e-22, 2.0 ** -9)
        for b in self.buffers():
            assert b.untouched()

    def check8(self, q, scale, want, off, least):
        def largest(t):
            return torch.nn.functional.pad(t, (0, -self.n % BLOCK)).view(-1, BLOCK).amax(1)

        scale = scale.double().cpu()
        top = (largest(want.abs()) / 448).clamp(min=2.0 ** -126)
        assert bool(((scale - top).abs() <= 3 * U * top + largest(off) / 448).all())
        wide = spread_out(scale, self.n)
        v, q = want / wide, q.double().cpu()
        _, e = torch.frexp(v)
        half = torch.ldexp(torch.ones_like(v), (e - 1).clamp(min=-6) - 4)
        near = (q - v).abs() <= half * (1 + 1e-6) + 3 * U * v.abs() + off / wide
        if least:
            near |= (q == least) & (v < least)
            assert bool((q[want > 0] >= least).all()) and bool((q[want == 0] == 0).all())
        assert bool(near.all()) and float(q.abs().max()) <= 448


def params_of(mqg, cases):
    lists = {k: [getattr(c, k).t for c in cases] for k in ("weight", "grad", "m", "v")}
    eight = cases[0].bits == 8
    return mqg.Params(lists["weight"], lists["grad"], m=lists["m"], v=lists["v"], m_scale=[c.m_scale.t for c in cases] if eight else None,
                      v_scale=[c.v_scale.t for c in cases] if eight else None, copies=[c.copy.t if c.copy else None for c in cases],
                      lr_scale=[c.lr_scale for c in cases], decay_scale=[c.decay_scale for c in cases])


PLAN = dict(lr=3e-3, step=5, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)
SIZES = [1, 2, 7, 8, 9, 127, 128, 129, 1023, 2047, 2048, 2049, 5000, 100_003]


def expect(cases, plan, scale=1.0):
    for c in cases:
        c.expect(plan["lr"], plan["step"], plan["beta1"], plan["beta2"], plan["eps"], plan["weight_decay"], scale)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", TYPES)
@pytest.mark.parametrize("weight", TYPES)
def test_a_step_of_tensors_of_all_sizes(mqg, ctx, weight, grad, bits):
    for copy, off, plan, fresh in ((None, 0, PLAN, False), (BF16, 1, dict(PLAN, step=1, weight_decay=0.0), True), (F16, 3, dict(PLAN, beta1=0.0, beta2=0.0), False),
                                   (F32, 5, dict(PLAN, step=10 ** 7, lr=-1e-3, eps=1e-3), False)):
        gen = torch.Generator().manual_seed(off)
        cases = [Case(n, gen, weight, grad, bits, copy, off, 1.0 + (i % 3), float(i % 2), fresh) for i, n in enumerate(SIZES)]
        expect(cases, plan)
        mqg.mqg_adamw_step(ctx, params_of(mqg, cases), **plan)
        torch.cuda.synchronize()
        for c in cases:
            c.check()


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_a_launch_takes_of_mixed_types_and_some_left_alone(mqg, ctx, bits):
    gen = torch.Generator().manual_seed(1)
    cases = [Case(int(torch.randint(0, 3000, (1,), generator=gen)), gen, TYPES[i % 2], TYPES[i % 3], bits, BF16 if i % 4 == 0 else None, i % 5)
             for i in range(170)]
    params = params_of(mqg, cases)
    alone = set(range(5, 170, 7))
    params.set_grads([None if i in alone else c.grad.t for i, c in enumerate(cases)])
    before = [[b.buf.clone() for b in c.buffers()] for c in cases]
    norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    total = math.sqrt(sum(float((c.grad.t.double() ** 2).sum()) for i, c in enumerate(cases) if i not in alone))
    mqg.mqg_grad_norm(ctx, params, max_norm=0.5 * total, norm=norm, scale=scale)
    torch.cuda.synchronize()
    # sixteen squares in fp32 lose 16 u of them, half of that in the root, and one rounding
    assert abs(float(norm) - total) <= 10 * U * total and abs(float(scale) - 0.5) <= 10 * U
    expect(cases, PLAN, float(scale))
    mqg.mqg_adamw_step(ctx, params, grad_scale=scale, **PLAN)
    torch.cuda.synchronize()
    for i, c in enumerate(cases):
        if i in alone or c.n == 0:
            assert all(torch.equal(b.buf, t) for b, t in zip(c.buffers(), before[i]))
        else:
            c.check()


@pytest.mark.parametrize("grad", TYPES)
def test_8_bit_moments_are_those_of_elementary_operations(mqg, ctx, grad):
    """Bit for bit, step after step: products, sums, roots and quotients are each rounded to nearest in fp32, as torch's are one by one."""
    n = 50_000
    gen = torch.Generator().manual_seed(13)
    weight = torch.randn(n, generator=gen).cuda()
    params = mqg.Params([weight], [torch.zeros(n, dtype=grad, device="cuda")], state_dtype=E4M3)
    unit = torch.exp(2 * torch.randn(n, generator=gen))
    unit[:1000] = 0
    m, v = torch.zeros(n, dtype=E4M3, device="cuda"), torch.zeros(n, dtype=E4M3, device="cuda")
    ms, vs = torch.zeros(blocks_of(n), device="cuda"), torch.zeros(blocks_of(n), device="cuda")
    scale = torch.full((1,), 0.37, device="cuda")
    for step in range(1, 9):
        g16 = (1e-3 * unit * torch.randn(n, generator=gen)).to(grad).cuda()
        params.set_grads([g16])
        mqg.mqg_adamw_step(ctx, params, grad_scale=scale, **dict(PLAN, step=step))
        g = g16.float() * scale
        m32 = 0.9 * (m.float() * spread_out(ms, n)) + (1 - 0.9) * g
        root = (0.999 * (v.float() * spread_out(vs, n)).square() + (1 - 0.999) * g * g).sqrt()
        (m, ms), (v, vs) = quantised(m32), quantised(root, 2.0 ** -9)
        torch.cuda.synchronize()
        assert torch.equal(params.m_scale[0], ms) and torch.equal(params.v_scale[0], vs), step
        # (zeros of either sign are the same value)
        assert torch.equal(params.m[0].float(), m.float()) and torch.equal(params.v[0].float(), v.float()), step


@pytest.mark.parametrize("bits", [32, 8])
def test_a_rate_of_its_own_for_every_tensor(mqg, ctx, bits):
    gen = torch.Generator().manual_seed(12)
    cases = [Case(50 + 37 * i, gen, bits=bits, lr_scale=0.9 ** i, decay_scale=float(i % 4)) for i in range(40)]
    expect(cases, PLAN)
    mqg.mqg_adamw_step(ctx, params_of(mqg, cases), **PLAN)
    torch.cuda.synchronize()
    for c in cases:
        c.check()


def test_one_list_of_both_kinds_of_moments(mqg, ctx):
    """The C call takes them together: the lists of two Params, one after the other."""
    gen = torch.Generator().manual_seed(2)
    cases = [Case(n, gen, bits=bits) for bits in (32, 8) for n in (500, 4000, 77)]
    lists = [params_of(mqg, cases[:3]), params_of(mqg, cases[3:])]
    both = (mqg.CParam * 6)(*lists[0].c, *lists[1].c)
    import ctypes
    plan = mqg.CAdamw(lr=PLAN["lr"], beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, step=5)
    expect(cases, PLAN)
    ctx.check(mqg.lib.mqg_adamw_step(ctx.h, both, 6, ctypes.byref(plan), mqg._stream(None)))
    torch.cuda.synchronize()
    for c in cases:
        c.check()


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_in_a_row_from_nothing(mqg, ctx, bits):
    """Moments that the binding made, ten steps, each against 64 bits from what the one before left."""
    gen = torch.Generator().manual_seed(3)
    c = Case(3001, gen, bits=bits, fresh=True)
    params = mqg.Params([c.weight.t], [c.grad.t], state_dtype=E4M3 if bits == 8 else F32)
    # the case's views of the binding's own moments
    for k in ("m", "v") + (("m_scale", "v_scale") if bits == 8 else ()):
        held = getattr(c, k)
        held.t = getattr(params, k)[0]
        held.untouched = lambda: True
    for step in range(1, 11):
        c.grad.t.copy_(0.01 * torch.randn(3001, generator=gen))
        plan = dict(PLAN, step=step)
        expect([c], plan)
        mqg.mqg_adamw_step(ctx, params, **plan)
        torch.cuda.synchronize()
        c.check()


def test_no_step_where_nothing_is_known_and_without_an_epsilon(mqg, ctx):
    for bits in (32, 8):
        for eps in (0.0, 1e-42):                                         # the second one is below fp32's normal numbers
            c = Case(300, torch.Generator().manual_seed(4), bits=bits, fresh=True)
            c.grad.t[::3] = 0
            plan = dict(PLAN, eps=eps, step=1)
            expect([c], dict(plan, eps=0.0))
            mqg.mqg_adamw_step(ctx, params_of(mqg, [c]), **plan)
            torch.cuda.synchronize()
            assert bool(c.weight.t.isfinite().all())
            c.check()


def test_a_block_of_zeros_and_the_smallest_roots_in_8_bits(mqg, ctx):
    n = 5 * BLOCK
    gen = torch.Generator().manual_seed(5)
    c = Case(n, gen, bits=8, fresh=True)
    g = torch.zeros(n)
    g[BLOCK] = 1.0
    g[BLOCK + 1:2 * BLOCK] = torch.logspace(-8, 0, BLOCK - 1)            # far below the block's least value: their roots become that one
    g[2 * BLOCK:3 * BLOCK] = 1e-30                                       # squares below fp32's numbers
    g[3 * BLOCK:4 * BLOCK] = 1e18                                        # and near their end
    g[4 * BLOCK:] = torch.randn(BLOCK, generator=gen)
    c.grad.t.copy_(g)
    plan = dict(PLAN, step=1)
    expect([c], plan)
    c.v64[2 * BLOCK:3 * BLOCK] = 0
    c.w64[2 * BLOCK:3 * BLOCK] = c.weight.t.double().cpu()[2 * BLOCK:3 * BLOCK] * (1 - PLAN["lr"] * 0.1)     # 1e-30 over the epsilon: nothing
    mqg.mqg_adamw_step(ctx, params_of(mqg, [c]), **plan)
    torch.cuda.synchronize()
    c.check()
    assert float(c.m_scale.t[0]) == 2.0 ** -126 and float(c.v_scale.t[0]) == 2.0 ** -126
    assert bool((c.v.t.float()[BLOCK:2 * BLOCK] >= 2.0 ** -9).all())


def test_gradients_that_are_not_finite(mqg, ctx):
    for bad in (float("nan"), float("inf"), float("-inf")):
        for bits in (32, 8):
            cases = [Case(1000, torch.Generator().manual_seed(6 + i), bits=bits) for i in range(2)]
            cases[0].grad.t[200] = bad
            params = params_of(mqg, cases)
            before = [[b.buf.clone() for b in c.buffers()] for c in cases]
            norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
            mqg.mqg_grad_norm(ctx, params, max_norm=1.0, norm=norm, scale=scale)
            mqg.mqg_adamw_step(ctx, params, grad_scale=scale, **PLAN)
            torch.cuda.synchronize()
            assert not math.isfinite(float(norm)) and math.isnan(float(scale))
            for c, was in zip(cases, before):                            # not stepped
                assert all(torch.equal(b.buf.view(torch.uint8), t.view(torch.uint8)) for b, t in zip(c.buffers(), was))
            expect(cases[1:], PLAN)
            mqg.mqg_adamw_step(ctx, params, **PLAN)                       # stepped all the same: the element's own, and its block's moments
            torch.cuda.synchronize()
            cases[1].check()
            w = cases[0].weight.t
            assert bool(w[:200].isfinite().all()) and bool(w[201:].isfinite().all())
            if bits == 8:
                finite = cases[0].m_scale.t.isfinite()
                assert not bool(finite[1]) and int(finite.sum()) == 7


@pytest.mark.parametrize("bits", [32, 8])
def test_recorded_steps_read_their_numbers_on_the_device(mqg, ctx, bits):
    """A recorded norm and step, replayed with other gradients, learning rates and step numbers, against calls that have these from the host."""
    own = context(mqg)
    sizes = [64, 3000, 129] * 25                                          # several launches
    pairs = [[Case(n, torch.Generator().manual_seed(n + i), bits=bits, copy=BF16) for i, n in enumerate(sizes)] for _ in range(2)]
    params = [params_of(mqg, cases) for cases in pairs]
    step, lr = torch.ones(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")
    results = [[torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")] for _ in range(2)]

    def call(k, c, **now):
        mqg.mqg_grad_norm(c, params[k], max_norm=2.0, norm=results[k][0], scale=results[k][1])
        mqg.mqg_adamw_step(c, params[k], beta1=0.9, beta2=0.99, weight_decay=0.1, grad_scale=results[k][1], **now)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        call(0, own, lr=lr, step=step)
    for k in range(1, 6):
        rate = 2.0 ** -(6 + k)
        lr.fill_(rate)
        step.fill_(k * k)
        for a, b in zip(*pairs):
            a.grad.t.mul_(1.0 + 0.1 * k)
            b.grad.t.mul_(1.0 + 0.1 * k)
        graph.replay()
        call(1, ctx, lr=rate, step=k * k)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*results))
        for a, b in zip(*pairs):
            assert all(torch.equal(x.buf, y.buf) for x, y in zip(a.buffers(), b.buffers())), k
    step.fill_(-3)                                                        # below the first: the first
    graph.replay()
    call(1, ctx, lr=rate, step=1)
    torch.cuda.synchronize()
    for a, b in zip(*pairs):
        assert all(torch.equal(x.buf, y.buf) for x, y in zip(a.buffers(), b.buffers()))


def test_on_another_stream(mqg):
    own = context(mqg)
    c = Case(50_000, torch.Generator().manual_seed(7), bits=8)
    params = params_of(mqg, [c])
    expect([c], PLAN)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mqg.mqg_adamw_step(own, params, stream=side, **PLAN)
    side.synchronize()
    c.check()


@pytest.mark.parametrize("grad", [F16, BF16])
def test_a_tensor_of_more_than_2_to_the_31_elements(mqg, ctx, grad):
    n = (1 << 31) + 2 * BLOCK + 5
    tail = 70_000
    weight, g = (torch.zeros(n, dtype=grad, device="cuda") for _ in range(2))
    params = mqg.Params([weight], [g], state_dtype=E4M3)
    gen = torch.Generator().manual_seed(8)
    at = n // BLOCK * BLOCK - tail // BLOCK * BLOCK                       # a block's beginning, on both sides of 2^31 elements
    small = Case(n - at, gen, grad, grad, 8)
    first = Case(1000, gen, grad, grad, 8)
    for c, lo in ((small, at), (first, 0)):
        weight[lo:lo + c.n], g[lo:lo + c.n] = c.weight.t, c.grad.t
        params.m[0].view(torch.uint8)[lo:lo + c.n], params.v[0].view(torch.uint8)[lo:lo + c.n] = c.m.t.view(torch.uint8), c.v.t.view(torch.uint8)
        params.m_scale[0][lo // BLOCK:lo // BLOCK + blocks_of(c.n)], params.v_scale[0][lo // BLOCK:lo // BLOCK + blocks_of(c.n)] = c.m_scale.t, c.v_scale.t
    norm = torch.zeros(1, device="cuda")
    mqg.mqg_grad_norm(ctx, params, norm=norm)
    mqg.mqg_adamw_step(ctx, params, **PLAN)
    mqg.mqg_adamw_step(ctx, params_of(mqg, [small, first]), **PLAN)
    torch.cuda.synchronize()
    total = math.sqrt(sum(float((c.grad.t.double() ** 2).sum()) for c in (small, first)))
    assert abs(float(norm) - total) <= 10 * U * total
    for c, lo in ((small, at), (first, 0)):
        assert torch.equal(weight[lo:lo + c.n], c.weight.t)
        assert torch.equal(params.m[0].view(torch.uint8)[lo:lo + c.n], c.m.t.view(torch.uint8))
        assert torch.equal(params.v[0].view(torch.uint8)[lo:lo + c.n], c.v.t.view(torch.uint8))
        assert torch.equal(params.m_scale[0][lo // BLOCK:lo // BLOCK + blocks_of(c.n)], c.m_scale.t)
    assert not bool(weight[5000:at].any())


# ---------------------------------------------------------------------------------------------- the norm

def norm_of(mqg, ctx, grads, **args):
    norm, scale = torch.full((3,), MARK, device="cuda"), torch.full((3,), MARK, device="cuda")
    mqg.mqg_grad_norm(ctx, mqg.Params(grads=grads), norm=norm[1:], scale=scale[1:], **args)
    torch.cuda.synchronize()
    assert norm[[0, 2]].tolist() == [MARK] * 2 and scale[[0, 2]].tolist() == [MARK] * 2
    return float(norm[1]), float(scale[1])


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_of_lists(mqg, ctx, dtype):
    gen = torch.Generator().manual_seed(9)
    for count, most in ((1, 3), (1, 100_000), (5, 5000), (64, 300), (65, 9000), (200, 2000), (700, 90), (1, 5_000_000)):
        grads = [Guarded(int(torch.randint(0 if count > 1 else most, most + 1, (1,), generator=gen)), dtype, i % 4) for i in range(count)]
        for g in grads:
            g.t.copy_(torch.randn(g.n, generator=gen))
        grads = [g.t for g in grads]
        total = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
        for mul, limit in ((1.0, float("inf")), (0.125, 0.01 * total), (3.0, 5.0 * total)):
            norm, scale = norm_of(mqg, ctx, grads, mul=mul, max_norm=limit)
            want = mul * min(1.0, limit / (mul * total))
            assert abs(norm - mul * total) <= 10 * U * mul * total and abs(scale - want) <= 12 * U * want
            assert (norm, scale) == norm_of(mqg, ctx, grads, mul=mul, max_norm=limit)      # the same bits every time


def test_norm_of_gradients_of_any_size(mqg, ctx):
    gen = torch.Generator().manual_seed(10)
    for size in (-149, -140, -100, -70, -30, 50, 70, 100, 110):
        g = torch.ldexp(torch.randn(30_000, generator=gen), torch.tensor(size)).cuda()
        total = math.sqrt(float((g.double() ** 2).sum()))
        norm, scale = norm_of(mqg, ctx, [g, torch.zeros(5000, device="cuda")], max_norm=1.0)
        assert abs(norm - total) <= 10 * U * total + 2.0 ** -149 and abs(scale - min(1.0, 1 / total)) <= 12 * U * scale
    assert norm_of(mqg, ctx, [torch.full((100,), 3e38, device="cuda")])[0] == float("inf")
    for bad in (float("inf"), float("nan")):
        g = torch.ones(10_000, device="cuda")
        g[7777] = bad
        norm, scale = norm_of(mqg, ctx, [g])
        assert not math.isfinite(norm) and math.isnan(scale)


def test_norm_of_nothing(mqg, ctx):
    for grads in ([], [torch.zeros(0, device="cuda")], [None, torch.zeros(1000, device="cuda")]):
        assert norm_of(mqg, ctx, grads, mul=0.5, max_norm=1.0) == (0.0, 0.5)
    # what an earlier call left does not count
    norm_of(mqg, ctx, [torch.ones(3_000_000, device="cuda")])
    assert norm_of(mqg, ctx, [torch.ones(4, device="cuda")]) == (2.0, 1.0)
    mqg.mqg_adamw_step(ctx, mqg.Params([], []), **PLAN)


# ---------------------------------------------------------------------------------------------- refusals

def test_refusals(mqg, ctx):
    import ctypes
    bad = mqg.MQG_ERR_INVALID_ARG
    gen = torch.Generator().manual_seed(11)

    def step(change=lambda p: None, bits=32, count=2, plan=None, num=None, **plan_args):
        cases = [Case(300, gen, bits=bits) for _ in range(count)]
        params = params_of(mqg, cases)
        change(params.c)
        fields = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, step=1)
        fields.update(plan_args)
        rc = mqg.lib.mqg_adamw_step(ctx.h, params.c, count if num is None else num, ctypes.byref(mqg.CAdamw(**fields)) if plan is None else None, mqg._stream(None))
        torch.cuda.synchronize()
        return rc

    def setting(field, value, index=1):
        return lambda c: setattr(c[index], field, value)

    assert step() == mqg.MQG_OK and step(bits=8) == mqg.MQG_OK
    for name in ("lr", "beta1", "beta2", "eps", "weight_decay"):
        assert step(**{name: float("nan")}) == bad and step(**{name: float("inf")}) == bad
    assert step(beta1=1.0) == bad and step(beta2=-0.1) == bad and step(eps=-1e-8) == bad and step(step=0) == bad and step(plan=False) == bad
    assert step(num=-1) == bad
    assert mqg.lib.mqg_adamw_step(ctx.h, None, 1, ctypes.byref(mqg.CAdamw(step=1)), None) == bad
    for field in ("weight", "m", "v"):
        assert step(setting(field, None)) == bad
    for field in ("weight_type", "grad_type", "copy_type"):
        assert step(lambda c: (setting("copy", c[0].grad)(c), setting(field, 3)(c))) == bad
    assert step(setting("numel", -1)) == bad and step(setting("state_type", 2)) == bad
    assert step(setting("m_scale", None), bits=8) == bad and step(setting("v_scale", None), bits=8) == bad
    assert step(setting("lr_scale", float("inf"))) == bad and step(setting("decay_scale", float("nan"))) == bad
    # the same tensor twice, or overlapping ones
    for field in ("weight", "m", "v"):
        assert step(lambda c: setattr(c[1], field, getattr(c[0], field))) == bad and b"share" in mqg.lib.mqg_last_error(ctx.h)
        assert step(lambda c: setattr(c[0], field, getattr(c[1], field) + 4 * 299)) == bad
    for field in ("m_scale", "v_scale"):
        assert step(lambda c: setattr(c[1], field, getattr(c[0], field)), bits=8) == bad
    # one buffer in two places of the same tensor
    for a, b in (("m", "v"), ("weight", "m"), ("v", "grad"), ("weight", "grad"), ("copy", "weight"), ("copy", "grad")):
        assert step(lambda c: setattr(c[1], a, getattr(c[1], b))) == bad and b"share" in mqg.lib.mqg_last_error(ctx.h)
    # what has no gradient is not looked at
    assert step(lambda c: (setting("grad", None)(c), setting("weight", None)(c))) == mqg.MQG_OK

    g = torch.ones(8, device="cuda")
    one = mqg.Params(grads=[g]).c

    def norm(mul=1.0, most=1.0, out=g.data_ptr(), num=1, params=one):
        return mqg.lib.mqg_grad_norm(ctx.h, params, num, mul, most, out, None, mqg._stream(None))

    assert norm() == mqg.MQG_OK
    for value in (0.0, -1.0, float("nan")):
        assert norm(mul=value) == bad and norm(most=value) == bad
    assert norm(mul=float("inf")) == bad and norm(most=float("inf")) == mqg.MQG_OK
    assert norm(out=None) == bad and norm(num=-1) == bad and norm(params=None) == bad
    torch.cuda.synchronize()

    w = torch.zeros((4, 8), device="cuda")
    with pytest.raises(AssertionError):
        mqg.Params([w.t()], [w.t()])
    with pytest.raises(AssertionError):
        mqg.Params([w], [w[:3]])
    with pytest.raises(AssertionError):
        mqg.Params([w], [w], m=[w], v=[w.half()])
    with pytest.raises(AssertionError):
        mqg.Params([w], [w], m=[w.clone()], v=[w.clone()], lr_scale=[1.0, 2.0])
    with pytest.raises(TypeError):
        mqg.Params([w.double()], [w])
    with pytest.raises(AssertionError):
        mqg.mqg_adamw_step(ctx, mqg.Params([w], [w.clone()]), lr=torch.zeros(1), step=1)
