"""Params keeps the tensors whose addresses it passes to the library, without a GPU (its check that tensors are the GPU's is replaced)."""
import gc
import weakref

import pytest
import torch


@pytest.fixture
def mqg(monkeypatch):
    from paper_2601_04707_amd import mqg as m

    def data(t, shape, dtype=None):
        assert t.is_contiguous() and t.shape == shape and (dtype is None or t.dtype is dtype)
        return t.data_ptr()

    monkeypatch.setattr(m.Params, "_data", staticmethod(data))
    return m


@pytest.mark.parametrize("eight", [False, True])
def test_lists_that_the_caller_changes(mqg, eight):
    state = torch.float8_e4m3fn if eight else torch.float32
    lists = {k: [torch.zeros(200) for _ in range(3)] for k in ("weights", "copies")}
    lists.update({k: [torch.zeros(200, dtype=state) for _ in range(3)] for k in ("m", "v")})
    if eight:
        lists.update({k: [torch.zeros(2) for _ in range(3)] for k in ("m_scale", "v_scale")})
    alive = {k: weakref.ref(ts[1]) for k, ts in lists.items()}
    at = {k: ts[1].data_ptr() for k, ts in lists.items()}
    params = mqg.Params(**lists)
    for ts in lists.values():
        ts[1] = None
        ts.append(None)
    gc.collect()
    c = params.c[1]
    for k, field in (("weights", "weight"), ("copies", "copy"), ("m", "m"), ("v", "v")) + ((("m_scale", "m_scale"), ("v_scale", "v_scale")) if eight else ()):
        held = getattr(params, k)
        assert alive[k]() is held[1] and len(held) == 3 and getattr(c, field) == at[k] == held[1].data_ptr(), k
    # the checks of the gradients go by the tensors that are kept
    params.set_grads([None, torch.zeros(200), None])
    with pytest.raises(AssertionError):
        params.set_grads([None, torch.zeros(199), None])


def test_gradients_that_are_refused_leave_those_before(mqg):
    params = mqg.Params([torch.zeros(8) for _ in range(2)])
    first = [torch.ones(8), torch.ones(8, dtype=torch.float16)]
    params.set_grads(first)
    for wrong in ([torch.ones(8, dtype=torch.bfloat16), torch.ones(7)], [None, torch.ones(8, dtype=torch.float64)], [torch.ones(8)]):
        with pytest.raises((AssertionError, TypeError)):
            params.set_grads(wrong)
        assert [(p.grad, p.grad_type) for p in params.c] == [(first[0].data_ptr(), mqg.MQG_F32), (first[1].data_ptr(), mqg.MQG_F16)]
        assert all(a is b for a, b in zip(params.grads, first))
