"""The calls of a layer without a GPU: struct layouts, refusals that need no context, and the binding's own arguments."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def mqg():
    from paper_2601_04707_amd import mqg as m
    return m


def test_struct_layouts_match_the_header(mqg):
    assert ctypes.sizeof(mqg.CMatrices) == 4 * 4 + 8 + 8 + 8
    assert mqg.CMatrices.data.offset == 16 and mqg.CMatrices.mat_stride.offset == 32
    assert ctypes.sizeof(mqg.COrth) == 16 and mqg.COrth.coeffs.offset == 8


def test_no_context_is_refused(mqg):
    bad = mqg.MQG_ERR_INVALID_ARG
    assert mqg.lib.mqg_rms_norm(None, None, 0, None, 0, None, 0.0, None, 0, 1, 0, None, 0, None, 0, None, 0, 0, 0, None, 0, None) == bad
    assert mqg.lib.mqg_rms_norm_backward(None, None, 0, None, 0, None, None, 0, 0.0, None, 0, 1, 0, None, 0, None, None) == bad
    assert mqg.lib.mqg_sage_mean_aggregate_q8(None, None, None, 0, 0, 0, None, 0, None, 0, 1, 0, None) == bad
    assert mqg.lib.mqg_orthogonalize(None, None, None, None, None) == bad
    assert mqg.lib.mqg_muon_step(None, None, None, None, 0.1, 0.9, 1, 0.0, 1.0, None, None) == bad
    assert mqg.lib.mqg_ctx_reserve_layer(None, 1, 1, 1, 1) == bad


def test_coefficients_for_one_step_or_for_all(mqg):
    p = mqg._orth(3, (1.5, -0.5, 0.0), 1e-7)
    assert p.steps == 3 and [p.coeffs[i] for i in range(9)] == [1.5, -0.5, 0.0] * 3
    p = mqg._orth(2, [(2.0, -1.5, 0.5), (1.875, -1.25, 0.375)], 1e-7)
    assert [p.coeffs[i] for i in range(6)] == [2.0, -1.5, 0.5, 1.875, -1.25, 0.375]
    assert not mqg._orth(5, None, 1e-7).coeffs
    with pytest.raises(AssertionError):
        mqg._orth(2, [(1.5, -0.5, 0.0)], 1e-7)


def test_the_limits_of_the_header_and_of_the_binding_are_the_same(mqg):
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mqg.h")).read()
    for name in ("MQG_NORM_MAX_DIM", "MQG_ORTH_MAX_STEPS", "MQG_ORTH_MAX_SIDE", "MQG_ORTH_MAX_MATS"):
        assert int(re.search(rf"#define {name} (\d+)", text)[1]) == getattr(mqg, name)
    for name in ("MQG_BF16", "MQG_Q_E4M3", "MQG_Q_INT8"):
        assert int(re.search(rf"{name} = (\d+)", text)[1]) == getattr(mqg, name)
