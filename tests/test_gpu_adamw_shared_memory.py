"""The step refuses lists of which a buffer that is written shares memory with any other one, of the same tensor or of another, before it launches anything."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

N = 300
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    assert torch.cuda.is_available()
    return m


@pytest.fixture(scope="module")
def ctx(mqg):
    g = mqg.Graph(torch.tensor([0, 1, 2], device="cuda"), torch.tensor([1, 0], device="cuda"))
    return mqg.Context(g, 1, [1])


def test_refused_before_anything_is_launched(mqg, ctx):
    bad = mqg.MQG_ERR_INVALID_ARG
    fields = ["weight", "copy", "m", "v", "m_scale", "v_scale", "grad"]
    size = {"weight": 4 * N, "copy": 2 * N, "m": N, "v": N, "m_scale": 12, "v_scale": 12, "grad": 4 * N}
    weights = [torch.ones(N, device="cuda") for _ in range(2)]
    grads = [torch.ones(N, device="cuda") for _ in range(2)]
    params = mqg.Params(weights, grads, state_dtype=E4M3, copies=[torch.zeros(N, dtype=torch.bfloat16, device="cuda") for _ in range(2)])
    held = [t for k in (params.weights, params.grads, params.copies, params.m, params.v, params.m_scale, params.v_scale) for t in k]
    before = [t.clone() for t in held]

    def step(changes, **plan):
        c = (mqg.CParam * 2)(*params.c)
        for index, field, value in changes:
            setattr(c[index], field, value)
        args = mqg.CAdamw(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, **plan)
        return mqg.lib.mqg_adamw_step(ctx.h, c, 2, ctypes.byref(args), mqg._stream(None))

    for k in range(2):                                                     # in the tensor itself, and in the other
        for to in fields:
            for of in fields:
                if to == of:
                    continue
                begin = getattr(params.c[0], of)
                for place in (begin, begin + size[of] - 1):
                    assert step([(k, to, place)]) == bad and b"shares memory" in mqg.lib.mqg_last_error(ctx.h), (k, to, of)
    for to in fields[:-1]:                                                 # the same buffer of both
        assert step([(1, to, getattr(params.c[0], to))]) == bad
    for name in ("lr_dev", "step_dev", "grad_scale_dev"):
        assert step([], **{name: weights[1].data_ptr() + 8}) == bad and step([], **{name: params.v_scale[0].data_ptr()}) == bad
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(held, before))
    # one gradient of two tensors is read twice
    assert step([(1, "grad", params.c[0].grad)]) == mqg.MQG_OK
    torch.cuda.synchronize()
    assert torch.equal(weights[0], weights[1]) and not torch.equal(weights[0], before[0])
