"""Refusals of the optimiser's step at the ends of what its arguments may be
(no kernel is launched)."""
import ctypes

import pytest

import paper_2607_01164_amd as gs
from test_optim_oracle import params, plan


@pytest.mark.parametrize("bad", [dict(lr_scale=1e39), dict(eps=1e39), dict(lr_scale=1.7e308), dict(eps=3.5e38)], ids=str)
def test_settings_that_float32_does_not_hold(bad):
    """An infinite factor would make NaN of a rate of 0."""
    L = gs.load_library()
    assert L.gs_adamw(ctypes.byref(plan()), ctypes.byref(params(**bad)), 1, None, None) == gs.GS_ERR_INVALID_ARGUMENT
    assert b"float32" in L.gs_last_error()
