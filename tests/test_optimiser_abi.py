"""Layer norm, the gradients' norm and the AdamW step without a GPU: struct layouts, refusals that need no context, and the binding's own."""
import ctypes
import os
import re

import pytest
import torch


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    return m


def test_struct_layouts_match_the_header(mqg):
    assert ctypes.sizeof(mqg.CParam) == 8 + 7 * 8 + 4 * 4 + 2 * 4
    assert mqg.CParam.weight.offset == 8 and mqg.CParam.grad.offset == 16 and mqg.CParam.copy.offset == 24 and mqg.CParam.v_scale.offset == 56
    assert mqg.CParam.state_type.offset == 76 and mqg.CParam.decay_scale.offset == 84
    assert ctypes.sizeof(mqg.CAdamw) == 9 * 8 and mqg.CAdamw.step.offset == 40 and mqg.CAdamw.grad_scale_dev.offset == 64


def test_no_context_is_refused(mqg):
    bad = mqg.MQG_ERR_INVALID_ARG
    assert mqg.lib.mqg_layer_norm(None, None, 0, None, 0, None, None, 0.0, None, 0, 1, 0, None, 0, None, 0, None, 0, 0, 0, None, 0, None) == bad
    assert mqg.lib.mqg_layer_norm_backward(None, None, 0, None, 0, None, None, 0, 0.0, None, 0, 1, 0, None, 0, None, None, None) == bad
    assert mqg.lib.mqg_grad_norm(None, None, 0, 1.0, 1.0, None, None, None) == bad
    assert mqg.lib.mqg_adamw_step(None, None, 0, None, None) == bad


def test_the_numbers_of_the_header_and_of_the_binding_are_the_same(mqg):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mqg.h")).read()
    assert int(re.search(r"#define MQG_ADAMW_BLOCK (\d+)", text)[1]) == mqg.MQG_ADAMW_BLOCK
    for name in ("MQG_STATE_F32", "MQG_STATE_E4M3"):
        assert int(re.search(rf"{name} = (\d+)", text)[1]) == getattr(mqg, name)


def test_tensors_of_the_host_are_refused(mqg):
    w = torch.zeros(4)
    with pytest.raises(AssertionError):
        mqg.Params([w], [w])
    with pytest.raises(AssertionError):
        mqg.Params(grads=[w])
    with pytest.raises(AssertionError):
        mqg.Params()
    assert len(mqg.Params(grads=[None, None]).c) == 2
