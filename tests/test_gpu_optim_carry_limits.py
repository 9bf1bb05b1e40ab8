"""Moments in 8 bits through a densification, at the ends of what the call
takes: inputs of about 2^32 elements, and codes that are NaN with either sign
beside zeros and beside values that a new scale makes small."""
import numpy as np
import pytest

import optim_oracle as oo
from harness import log
from test_gpu_optim import host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def carry(width, a, n_in, source):
    """Rows `source` of the arrays a (m, v and their scales, on the device):
    the outputs on the host."""
    import torch
    import paper_2607_01164_amd as gs
    n = len(source) * width
    z = lambda k: torch.full((k,), 9, dtype=torch.uint8, device="cuda")  # noqa: E731
    out = {"m": z(n), "v": z(n), "m_scale": z(gs.moment_scales(n)), "v_scale": z(gs.moment_scales(n))}
    rows = gs.AdamRows(width, a["m"], a["v"], out["m"], out["v"], a["m_scale"], a["v_scale"], out["m_scale"],
                       out["v_scale"])
    gs.gs_adamw_carry(gs.AdamCarry([rows]), n_in, torch.from_numpy(np.asarray(source, np.int32)).cuda(), len(source))
    return {k: host(x) for k, x in out.items()}


# (width, rows): 32 elements below 2^32, 26 to 2 below it, where the count of
# the blocks must not be formed past 32 bits, 1 below it, and 2^32
NEAR = [(4, 2 ** 30 - 8), (3, 1431655757), (5, 858993454), (7, 613566753), (2, 2 ** 31 - 2),
        (5, 858993458), (3, 1431655764), (4, 2 ** 30 - 1), (2, 2 ** 31 - 1), (3, 1431655765), (4, 2 ** 30)]


@pytest.mark.parametrize("width,n_in", NEAR, ids=[f"{w}x{n}" for w, n in NEAR])
def test_inputs_of_about_2_to_32_elements(width, n_in):
    """Rows at the start, the middle and the end, whose blocks have scales of
    their own."""
    import torch
    import paper_2607_01164_amd as gs
    free, _ = torch.cuda.mem_get_info()
    if free < 20 << 30:
        pytest.skip("needs 20 GiB")
    n, part = n_in * width, 4096
    log(f"case: carry from {n_in} rows of {width}, 2^32 {n - 2 ** 32:+d} elements")
    r = np.random.default_rng(n_in)
    a = {k: torch.zeros(n, dtype=torch.uint8, device="cuda") for k in "mv"}
    a.update({k + "_scale": torch.zeros(gs.moment_scales(n), dtype=torch.uint8, device="cuda") for k in "mv"})
    starts = [0, n // 64 * 32, (n - part) // 32 * 32]
    ends = [part, starts[1] + part, n]
    for at, end in zip(starts, ends):
        for k in "mv":
            codes = r.integers(0, 0x7F, end - at) | (r.integers(0, 2, end - at) * 128 if k == "m" else 0)
            a[k][at:end] = torch.from_numpy(codes.astype(np.uint8)).cuda()
            a[k + "_scale"][at // 32:(end + 31) // 32] = torch.from_numpy(
                r.integers(100, 150, (end + 31) // 32 - at // 32).astype(np.uint8)).cuda()
    take = part // width - 20
    near = [np.arange(take), starts[1] // width + 8 + r.permutation(take), n_in - 1 - np.arange(take)]
    source = np.concatenate(near + [np.array([-1, n_in - 1, 0, -7])])
    out = carry(width, a, n_in, source)
    live = source >= 0
    index = np.where(live, source, 0)[:, None] * width + np.arange(width)
    for k in "mv":
        at = torch.from_numpy(index.reshape(-1)).cuda()
        x = oo.e4m3(host(a[k][at])) * oo.scale_value(host(a[k + "_scale"][at // 32]))
        want = np.where(np.repeat(live, width), x, 0.0)
        oo.check_mxfp8(out[k], out[k + "_scale"], want, 0.0 * want, positive=k == "v", label=f"{width} x {n_in} {k}")


@pytest.mark.parametrize("width", [1, 3, 4, 7])
@pytest.mark.parametrize("nan", [0x7F, 0xFF])
def test_nan_beside_zeros_and_small_values(nan, width):
    """A NaN in any place of its word, either sign, in m and v: zeros beside it
    stay zeros, and values of sqrt(v) that the new block's scale takes below
    half its smallest number stay positive."""
    import torch
    r = np.random.default_rng(width)
    n_in = 512
    n = n_in * width
    kinds = r.integers(0, 4, n)
    small = np.repeat(np.arange((n + 31) // 32) % 2 == 1, 32)[:n]  # every other block has a far smaller scale
    codes = np.where(kinds == 0, 0, np.where(kinds == 1, nan, np.where(small, r.integers(1, 8, n),
                                                                       r.integers(0x70, 0x7F, n))))
    scales = np.where(np.arange((n + 31) // 32) % 2 == 1, 100, 130)
    dev = lambda x: torch.from_numpy(x.astype(np.uint8)).cuda()  # noqa: E731
    a = {"m": dev(codes), "v": dev(codes), "m_scale": dev(scales), "v_scale": dev(scales)}
    source = np.concatenate([r.permutation(n_in), -1 - np.arange(9), r.permutation(n_in)])
    out = carry(width, a, n_in, source)
    x = np.concatenate([oo.values(codes, scales).reshape(n_in, width), np.zeros((1, width))])
    want = x[np.where(source >= 0, source, n_in)].reshape(-1)
    assert ((want > 0) & (want < 2.0 ** -20)).sum() > 100
    for k in "mv":
        oo.check_mxfp8(out[k], out[k + "_scale"], want, np.zeros_like(want), positive=k == "v",
                       label=f"{k}, NaN {nan:#x}, width {width}")


def test_a_gradient_that_is_not_a_number_then_a_carry():
    """NaN gradients of either sign, a step, and the moments' carry: the same
    elements are NaN, every other keeps its kind."""
    import torch
    import paper_2607_01164_amd as gs
    n = 4096
    r = np.random.default_rng(2)
    g = np.where(r.random(n) < 0.5, 0.0, np.exp(r.normal(size=n) * 6 - 10)).astype(np.float32)
    bits = g.view(np.uint32)
    bits[::5] = 0x7FC00000
    bits[2::5] = 0xFFC00000
    t = gs.AdamTensor.new(torch.zeros(n, device="cuda"), torch.from_numpy(g).cuda(), 0.01,
                          moments=gs.GS_MOMENTS_MXFP8)
    gs.gs_adamw(gs.AdamPlan([t]), step=1)
    a = {"m": t.m, "v": t.v, "m_scale": t.m_scale, "v_scale": t.v_scale}
    source = np.concatenate([r.permutation(n), [-1]])
    out = carry(1, a, n, source)
    index = np.where(source >= 0, source, 0)
    nan = np.isnan(g[index]) & (source >= 0)
    for k in "mv":
        x = np.where(source >= 0, oo.values(host(a[k]), host(a[k + "_scale"]))[index], 0.0)
        assert np.array_equal(np.isnan(x), nan)
        oo.check_mxfp8(out[k], out[k + "_scale"], x, 0.0 * np.nan_to_num(x), positive=k == "v", label=k)
