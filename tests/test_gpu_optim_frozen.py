"""Lists with tensors that have no parameter: they count for the norm, and the
step passes them by."""
import math

import numpy as np
import pytest

import optim_oracle as oo
from test_gpu_optim import B1, B2, EPS, FORMS, check, host, make, snapshot

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("frozen", [[0], [2], [0, 1, 3], [1, 2, 4]], ids=str)
def test_tensors_without_a_parameter_count_for_the_norm(frozen, form):
    """The gradients of all arrays make the norm; those with a parameter take
    the step of their place in the list, with the norm's clip factor."""
    import paper_2607_01164_amd as gs
    sizes, types = [3001, 2 * 1024, 77, 1, 5000], [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")]
    whole = [make(n, types[i % 3], form, 50 + i) for i, n in enumerate(sizes)]
    ts = [gs.AdamTensor(None, t.grad) if i in frozen else t for i, t in enumerate(whole)]
    before = [snapshot(t) for t in whole]
    plan, control = gs.AdamPlan(ts), gs.alloc_adam_control("cuda")
    gs.gs_grad_norm(plan, control, max_norm=0.25, beta1=B1, beta2=B2)
    gs.gs_adamw(plan, beta1=B1, beta2=B2, eps=EPS, control=control, seed=3)
    norm = math.sqrt(math.fsum(float(x) for b in before for x in np.square(b["g"])))
    c = gs.read_adam_control(control)
    assert abs(c["norm"] / norm - 1) <= 2 * oo.U and abs(c["clip"] * norm / 0.25 - 1) <= 4 * oo.U
    for i, (t, b) in enumerate(zip(whole, before)):
        if i in frozen:
            after = snapshot(t)
            for k in b:
                np.testing.assert_array_equal(after[k], b[k])
        else:
            check(t, b, i, 1, seed=3, clip=0.25 / norm, label=f"array {i}")


def test_a_step_of_nothing_is_refused():
    import torch
    import paper_2607_01164_amd as gs
    g, empty = torch.zeros(5, device="cuda"), torch.empty(0, device="cuda")
    for ts in ([gs.AdamTensor(None, g)], [gs.AdamTensor(None, g), gs.AdamTensor.new(empty, empty, 0.1)]):
        with pytest.raises(gs.GsError):
            gs.gs_adamw(gs.AdamPlan(ts), step=1)
    for ts in ([gs.AdamTensor(None, empty)], [gs.AdamTensor.new(empty, empty, 0.1)],
               [gs.AdamTensor.new(g.clone(), g, 0.1), gs.AdamTensor(None, g)]):
        gs.gs_adamw(gs.AdamPlan(ts), step=1)
    assert np.all(host(g) == 0)
