"""The gradient norm past the caches and at any alignment, and the clip factor
of gradients so large that it is a denormal number."""
import math

import numpy as np
import pytest

import optim_oracle as oo
from test_gpu_optim import B1, B2, EPS, check, dtype, host, snapshot

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def normed(grads, max_norm):
    import paper_2607_01164_amd as gs
    control = gs.alloc_adam_control("cuda")
    gs.gs_grad_norm(gs.AdamPlan([gs.AdamTensor(None, g) for g in grads]), control, max_norm=max_norm)
    return gs.read_adam_control(control)


@pytest.mark.parametrize("gtype,n", [("f32", (1 << 26) + 40967), ("bf16", (1 << 27) + 40967)])
@pytest.mark.parametrize("offset", [0, 1])
def test_norm_past_the_caches(gtype, n, offset):
    """More than 256 MB of gradients in two tensors, at and off the start of
    their allocations, with pieces and vectors that end early."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(n + offset)
    whole = torch.empty(n + offset, dtype=dtype(gtype), device="cuda").normal_(generator=gen)
    if offset:
        whole[0] = 1e30  # not of the list
    a, b = whole[offset:offset + n - 7003], whole[offset + n - 7003:]
    want = math.sqrt(sum(float(x.double().square().sum()) for x in (a, b)))
    c = normed([a, b], want / 3)
    # float64 sums of 2^27 squares at most, twice: 2^-26 of the sum if every
    # rounding went one way, half of that of the root
    assert abs(c["norm"] - want) <= want * (oo.U + 2.0 ** -26) and c["step"] == 1
    assert abs(c["clip"] * 3 - 1) <= oo.U + 2.0 ** -26 + 2.0 ** -50


@pytest.mark.parametrize("gtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [1, 2, 3, 5, 7])
@pytest.mark.parametrize("n", [1, 9, 4099, 16385, 50021])
def test_norm_at_any_alignment(n, offset, gtype):
    import torch
    r = np.random.default_rng(n)
    w = torch.full((n + offset + 9,), 1e30, dtype=dtype(gtype), device="cuda")  # what is beside it is not read
    w[offset:offset + n] = torch.from_numpy(r.normal(size=n).astype(np.float32)).to(dtype(gtype))
    g = w[offset:offset + n]
    want = math.sqrt(math.fsum(float(x) for x in np.square(host(g))))
    c = normed([g], math.inf)
    assert abs(c["norm"] - want) <= want * (oo.U + 2.0 ** -37) and c["clip"] == 1.0  # 2^16 sums at most


@pytest.mark.parametrize("x", [3e38, 1e38, 1e30, 1e3, 1.0, 1e-3])
def test_clip_of_large_gradients(x):
    """max_norm / norm rounded once, also where it is a denormal number."""
    import torch
    g = torch.full((1000,), x, device="cuda")
    want = 1.0 / (float(g[0].double()) * math.sqrt(1000))
    c = normed([g], 1.0)
    want = want if want < 1.0 else 1.0
    assert c["step"] == 1 and c["clip"] > 0.0
    assert abs(c["clip"] - want) <= oo.U * want * (1 + 2.0 ** -20) + oo.TINY / 2


@pytest.mark.parametrize("form", ["f32", "mxfp8"])
def test_a_step_clipped_by_a_denormal_factor(form):
    """Gradients of 3e38 with a maximum of 1: the step is that of gradients
    clipped to a norm of 1, by the factor that is on the device."""
    import torch
    import paper_2607_01164_amd as gs
    r = np.random.default_rng(5)
    n = 1000
    g = torch.from_numpy((3e38 * r.uniform(-1, 1, n)).astype(np.float32)).cuda()
    t = gs.AdamTensor.new(torch.ones(n, device="cuda"), g, 0.01, 0.1, gs.GS_MOMENTS_F32 if form == "f32"
                          else gs.GS_MOMENTS_MXFP8)
    plan, control = gs.AdamPlan([t]), gs.alloc_adam_control("cuda")
    before = snapshot(t)
    gs.gs_grad_norm(plan, control, max_norm=1.0, beta1=B1, beta2=B2)
    gs.gs_adamw(plan, beta1=B1, beta2=B2, eps=EPS, control=control, seed=4)
    clip = gs.read_adam_control(control)["clip"]
    assert 0.0 < clip < 2.0 ** -126
    check(t, before, 0, 1, seed=4, clip=clip, label=f"{form}, clip {clip}")
