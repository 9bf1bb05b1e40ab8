"""Refusals of the optimiser's step at the ends of what its arguments may be,
and of tensors on several devices (no kernel is launched)."""
import ctypes

import pytest
import torch

import paper_2607_01164_amd as gs
from test_optim_oracle import params, plan


@pytest.mark.parametrize("bad", [dict(lr_scale=1e39), dict(eps=1e39), dict(lr_scale=1.7e308), dict(eps=3.5e38)], ids=str)
def test_settings_that_float32_does_not_hold(bad):
    """An infinite factor would make NaN of a rate of 0."""
    L = gs.load_library()
    assert L.gs_adamw(ctypes.byref(plan()), ctypes.byref(params(**bad)), 1, None, None) == gs.GS_ERR_INVALID_ARGUMENT
    assert b"float32" in L.gs_last_error()


class Tensor:
    """Stands for a contiguous tensor of a device."""

    def __init__(self, dtype, device, n=64):
        self.dtype, self.index, self.n = dtype, device, n
        self.is_cuda, self.device = device >= 0, ("cuda", device)

    def get_device(self):
        return self.index

    def numel(self):
        return self.n

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


def arrays(names, form, other=None, where=1):
    dt = torch.float32 if form == "f32" else torch.uint8
    return {k: Tensor(torch.float32 if k in ("param", "grad") else dt, where if k == other else 0) for k in names
            if form == "mxfp8" or "scale" not in k}


TENSOR = ("param", "grad", "m", "v", "m_scale", "v_scale")
ROWS = ("m", "v", "m_out", "v_out", "m_scale", "v_scale", "m_scale_out", "v_scale_out")


@pytest.mark.parametrize("where", [1, -1], ids=["another", "host"])
@pytest.mark.parametrize("form", ["f32", "mxfp8"])
def test_arrays_on_several_devices(form, where):
    gs.AdamTensor(**arrays(TENSOR, form)).c()
    for k in arrays(TENSOR, form):
        with pytest.raises(ValueError):
            gs.AdamTensor(**arrays(TENSOR, form, k, where)).c()
    carry = gs.AdamCarry([gs.AdamRows(2, **arrays(ROWS, form)), gs.AdamRows(1, **arrays(ROWS, form))])
    for k in arrays(ROWS, form):
        for first in (arrays(ROWS, form), None):
            rows = [gs.AdamRows(1, **first)] if first else []
            with pytest.raises(ValueError):
                gs.AdamCarry(rows + [gs.AdamRows(2, **arrays(ROWS, form, k, where))])
    with pytest.raises(ValueError):
        gs.gs_adamw_carry(carry, 4, Tensor(torch.int32, where), 4)


@pytest.mark.parametrize("where", [1, -1], ids=["another", "host"])
def test_control_on_another_device(where):
    class Plan:
        c, device = plan(), 0

        def on(self, stream):
            return 0

    with pytest.raises(ValueError):
        gs.gs_grad_norm(Plan(), Tensor(torch.uint8, where))
    with pytest.raises(ValueError):
        gs.gs_adamw(Plan(), control=Tensor(torch.uint8, where))


def test_moment_values_are_the_oracles():
    """What codes and scales stand for, from an empty tensor to blocks that end
    early, with the scale of a new tensor (byte 0) and both signs of NaN."""
    import numpy as np
    import optim_oracle as oo
    r = np.random.default_rng(1)
    for n in (0, 1, 31, 32, 33, 1000):
        codes = r.integers(0, 256, n).astype(np.uint8)
        scales = r.integers(1, 247, gs.moment_scales(n)).astype(np.uint8)
        got = gs.moment_values(torch.from_numpy(codes), torch.from_numpy(scales))
        assert got.dtype == torch.float32 and got.shape == (n,)
        want = oo.values(codes, scales).astype(np.float32)
        np.testing.assert_array_equal(got.numpy(), want)
    zero = gs.moment_values(torch.zeros(40, dtype=torch.uint8), torch.zeros(2, dtype=torch.uint8))
    assert zero.shape == (40,) and not zero.any()
    rows = torch.full((2, 32), 0x38, dtype=torch.uint8)  # 1.0, of any shape
    assert gs.moment_values(rows, torch.tensor([0, 130], dtype=torch.uint8)).tolist() == [2.0 ** -127] * 32 + [8.0] * 32
