"""The float64 optimiser of the tests against closed forms: AdamW's first
step, a long run's average, E4M3's table, the grid's rounding against
torch's cast, and the random bits. Also the gs_optim.h entry points'
refusals (no kernel is launched)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import optim_oracle as oo
import paper_2607_01164_amd as gs
from paper_2607_01164_amd import gsq

FAKE = 1 << 20  # a non-null, aligned address that validation never dereferences


def test_first_step_moves_by_the_learning_rate():
    g = np.array([3.0, -1e-3, 0.5])
    p, m, v, s, *_ = oo.step(np.ones(3), g, 0 * g, 0 * g, lr=0.01, wd=0.0, beta1=0.9, beta2=0.999, eps=0.0, t=1)
    assert np.allclose(p, 1 - oo.f32(0.01) * np.sign(g), rtol=1e-12)
    assert np.allclose(m, 0.1 * g) and np.allclose(v, 1e-3 * g * g) and np.allclose(s * s, v)


def test_decay_leaves_the_moments():
    p, m, v, *_ = oo.step([2.0], [0.0], [0.0], [0.0], lr=0.5, wd=0.25, beta1=0.9, beta2=0.999, eps=1e-8, t=7)
    assert p[0] == 2.0 - 0.5 * 0.25 * 2.0 and m[0] == 0 and v[0] == 0


def test_constant_gradient_reaches_its_average():
    p = m = v = np.zeros(1)
    for t in range(1, 400):
        p, m, v, *_ = oo.step(p, [0.3], m, v, lr=0.01, wd=0.0, beta1=0.9, beta2=0.99, eps=0.0, t=t)
    assert math.isclose(m[0], 0.3, rel_tol=1e-12) and math.isclose(v[0], 0.09 * (1 - 0.99 ** 399), rel_tol=1e-9)
    assert math.isclose(p[0], -399 * oo.f32(0.01), rel_tol=1e-9)  # every bias-corrected step has the rate's length


def test_e4m3_table_is_torchs():
    codes = np.arange(256)
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(oo.e4m3(codes), want)
    fine = np.arange(0x7F)
    np.testing.assert_array_equal(oo.magnitude_code(oo.e4m3(fine)), fine)


def test_nearest_rounding_is_torchs_cast():
    r = np.random.default_rng(1)
    x = np.exp2(r.uniform(-14, 8.8, 4096)) * np.sign(r.normal(size=4096))
    x[:64] = oo.e4m3(r.integers(0, 0x7E, 64)) + oo.e4m3(r.integers(0, 8, 64)) / 2  # ties among them
    x[::32] = 448.0  # every block's scale is 1
    x = np.clip(x, -448, 448).astype(np.float32)
    codes = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    oo.check_mxfp8(codes, np.full(128, 127), x.astype(np.float64), 0.0 * x, label="cast")
    wrong = codes.copy()
    wrong[5] ^= 1
    with pytest.raises(AssertionError):
        oo.check_mxfp8(wrong, np.full(128, 127), x.astype(np.float64), 0.0 * x)


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.0001, 1), (256.0, 0), (255.9, 0), (224.0, -1), (1.0, -8),
                                   (2.0 ** -149, -126), (0.0, -126), (3.0e38, 120)])
def test_block_exponent(top, e):
    got = int(oo.exponents(np.array([top]))[0])
    assert got == e or (top == 3.0e38 and top <= 448.0 * 2.0 ** got and top > 448.0 * 2.0 ** (got - 1))


def test_random_bits_are_even_and_differ_by_step_and_place():
    n = 1 << 16
    a = oo.random_bits(np.arange(n), 3, 17, 0x123456789)
    for b in (oo.random_bits(np.arange(n), 4, 17, 0x123456789), oo.random_bits(np.arange(n), 3, 18, 0x123456789),
              oo.random_bits(np.arange(n), 3, 17, 0x123456788),
              oo.random_bits(np.arange(n) + (1 << 32), 3, 17, 0x123456789)):
        assert np.mean(a == b) < 1e-3
        x, y = (a & np.uint64(0xFFFF)).astype(float), (b & np.uint64(0xFFFF)).astype(float)
        assert abs(np.corrcoef(x, y)[0, 1]) < 6 / math.sqrt(n)  # six standard deviations of independent draws
    for half in (a & np.uint64(0xFFFF), a >> np.uint64(16)):
        u = (half.astype(float) + 0.5) / 65536
        assert abs(u.mean() - 0.5) < 6 * math.sqrt(1 / 12 / n)
        assert abs(np.mean(u[1:] * u[:-1]) - 0.25) < 6 * math.sqrt(7 / 144 / n)


# ---- refusals -------------------------------------------------------------

def tensor(**k):
    d = dict(param=FAKE, grad=FAKE, m=FAKE, v=FAKE, m_scale=FAKE, v_scale=FAKE, n=100, param_type=0, grad_type=0,
             moments=0, lr=0.1, weight_decay=0.0)
    d.update(k)
    return gsq.GsAdamwTensor(*[d[f] for f, _ in gsq.GsAdamwTensor._fields_])


def plan(work=FAKE, work_bytes=1 << 20, n_items=4, updatable=1):
    return gsq.GsAdamwPlan(work, work_bytes, n_items, 1, 100, 100, 1, updatable)


def params(beta1=0.9, beta2=0.999, eps=1e-8, lr_scale=1.0, max_norm=1.0):
    return gsq.GsAdamwParams(beta1, beta2, eps, lr_scale, max_norm, 0)


def test_plan_bytes():
    L = gs.load_library()
    a, b = L.gs_adamw_plan_bytes(ctypes.byref(tensor(n=1)), 1), L.gs_adamw_plan_bytes(ctypes.byref(tensor(n=10 ** 6)), 1)
    assert 0 < L.gs_adamw_plan_bytes(None, 0) < a < b and a % 256 == 0
    err = ctypes.c_size_t(-1).value
    assert L.gs_adamw_plan_bytes(None, 1) == err
    assert L.gs_adamw_plan_bytes(ctypes.byref(tensor()), -1) == err
    assert L.gs_adamw_plan_bytes(ctypes.byref(tensor()), (1 << 20) + 1) == err
    assert L.gs_adamw_plan_bytes(ctypes.byref(tensor(n=-1)), 1) == err
    assert L.gs_adamw_plan_bytes(ctypes.byref(tensor(n=1 << 40)), 1) == err


@pytest.mark.parametrize("bad", [dict(n=-1), dict(param_type=2), dict(grad_type=-1), dict(param_type=1, grad_type=0),
                                 dict(moments=2), dict(lr=float("nan")), dict(lr=-1.0),
                                 dict(weight_decay=float("inf")), dict(weight_decay=-0.5), dict(grad=None),
                                 dict(grad=FAKE + 2), dict(param=FAKE + 2), dict(m=None), dict(v=None),
                                 dict(m=FAKE + 1), dict(moments=1, m_scale=None), dict(moments=1, v_scale=None),
                                 dict(grad_type=1, grad=FAKE + 1)])
def test_plan_refuses(bad):
    L = gs.load_library()
    p = plan()
    assert L.gs_plan_adamw(ctypes.byref(tensor(**bad)), 1, ctypes.byref(p), None) == gs.GS_ERR_INVALID_ARGUMENT
    assert b"gs_plan_adamw" in L.gs_last_error() and p.n_items == -1
    assert L.gs_adamw(ctypes.byref(p), ctypes.byref(params()), 1, None, None) == gs.GS_ERR_INVALID_ARGUMENT


def test_plan_refuses_workspaces():
    L = gs.load_library()
    t = tensor()
    for p in (plan(work=None), plan(work_bytes=16), plan(work=FAKE + 8)):
        assert L.gs_plan_adamw(ctypes.byref(t), 1, ctypes.byref(p), None) == gs.GS_ERR_WORKSPACE
    assert L.gs_plan_adamw(ctypes.byref(t), 1, None, None) == gs.GS_ERR_INVALID_ARGUMENT
    assert L.gs_plan_adamw(None, 1, ctypes.byref(plan()), None) == gs.GS_ERR_INVALID_ARGUMENT


@pytest.mark.parametrize("case", ["null_plan", "null_params", "unmade", "short", "beta1", "beta2", "nan_beta", "eps", "no_eps",
                                  "lr_scale", "step", "control", "no_param"])
def test_step_refuses(case):
    L = gs.load_library()
    p, s, t, c = plan(), params(), 1, None
    if case == "unmade":
        p = plan(n_items=-1)
    elif case == "short":
        p = plan(work_bytes=100)
    elif case == "beta1":
        s = params(beta1=1.0)
    elif case == "beta2":
        s = params(beta2=-0.1)
    elif case == "nan_beta":
        s = params(beta1=float("nan"))
    elif case == "eps":
        s = params(eps=-1e-8)
    elif case == "no_eps":
        s = params(eps=0.0)
    elif case == "lr_scale":
        s = params(lr_scale=float("inf"))
    elif case == "step":
        t = 0
    elif case == "control":
        c = FAKE + 4
    elif case == "no_param":
        p = plan(updatable=0)
    st = L.gs_adamw(None if case == "null_plan" else ctypes.byref(p),
                    None if case == "null_params" else ctypes.byref(s), t, c, None)
    assert st == gs.GS_ERR_INVALID_ARGUMENT and b"gs_adamw" in L.gs_last_error()


@pytest.mark.parametrize("case", ["null_plan", "beta2", "max_norm", "nan_norm", "null_control", "control"])
def test_norm_refuses(case):
    L = gs.load_library()
    p, s, c = plan(), params(), FAKE
    if case == "beta2":
        s = params(beta2=1.0)
    elif case == "max_norm":
        s = params(max_norm=0.0)
    elif case == "nan_norm":
        s = params(max_norm=float("nan"))
    elif case == "null_control":
        c = None
    elif case == "control":
        c = FAKE + 4
    st = L.gs_grad_norm(None if case == "null_plan" else ctypes.byref(p), ctypes.byref(s), c, None)
    assert st == gs.GS_ERR_INVALID_ARGUMENT and b"gs_grad_norm" in L.gs_last_error()


@pytest.mark.parametrize("bad", [dict(width=0), dict(width=65), dict(moments=7), dict(m=None), dict(v_out=None),
                                 dict(moments=1, m_scale=None), dict(moments=1, v_scale_out=None),
                                 dict(m_out=FAKE + 2), dict(count=-1), dict(count=17), dict(n_in=-1),
                                 dict(n_out=1 << 31), dict(source=None), dict(source=FAKE + 2), dict(arrays=None)])
def test_carry_refuses(bad):
    L = gs.load_library()
    d = {f: FAKE for f, _ in gsq.GsAdamwRows._fields_}
    d.update(width=3, moments=0)
    d.update({k: v for k, v in bad.items() if k in d})
    r = gsq.GsAdamwRows(*[d[f] for f, _ in gsq.GsAdamwRows._fields_])
    st = L.gs_adamw_carry(None if "arrays" in bad else ctypes.byref(r), bad.get("count", 1), bad.get("n_in", 10),
                          bad.get("source", FAKE), bad.get("n_out", 10), None)
    assert st == gs.GS_ERR_INVALID_ARGUMENT and b"gs_adamw_carry" in L.gs_last_error()


def test_binding_refuses():
    x = torch.zeros(64)
    with pytest.raises(ValueError):
        gs.AdamTensor(x, x).c()  # not on the device
    with pytest.raises(ValueError):
        gs.gs_adamw(None)
    with pytest.raises(ValueError):
        gs.gs_adamw(None, step=1, control=x)
    with pytest.raises(ValueError):
        gs.AdamTensor.new(x, x, 0.1, moments=5)
    with pytest.raises(ValueError):
        gs.AdamCarry([gs.AdamRows(0, x, x, x, x)])
    assert [gs.moment_scales(n) for n in (0, 1, 32, 33)] == [0, 1, 1, 2]
