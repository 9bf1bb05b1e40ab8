"""Training a field from free parameters to the optimiser's step
(examples/train_field.py): the step in the loop follows the definition, the
moments follow their Gaussians through a densification, and the field is
learned as well with 8-bit moments as with 32-bit ones."""
import numpy as np
import pytest

from harness import log
from test_gpu_optim import check, host, snapshot

pytestmark = pytest.mark.gpu

FORMS = ["f32", "mxfp8"]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def trainer(form, **k):
    import paper_2607_01164_amd as gs
    from examples.train_field import Trainer
    return Trainer(moments=gs.GS_MOMENTS_F32 if form == "f32" else gs.GS_MOMENTS_MXFP8, **k)


@pytest.mark.parametrize("form", FORMS)
def test_steps_in_the_loop_follow_the_definition(form):
    import torch
    import paper_2607_01164_amd as gs
    t = trainer(form, n=1001, dims=32, max_norm=0.01, weight_decay=0.01)
    for k in range(1, 4):
        before = [snapshot(x) for x in t.adam.tensors]
        t.step()
        torch.cuda.synchronize()
        c = gs.read_adam_control(t.control)
        assert c["step"] == k and c["skipped"] == 0
        for i, (x, b) in enumerate(zip(t.adam.tensors, before)):
            b["g"] = host(x.grad)  # as this iteration's backward left it
            norm = np.sqrt(sum(np.square(host(y.grad)).sum() for y in t.adam.tensors))
            clip = min(1.0, 0.01 / norm)
            check(x, b, i, k, seed=t.seed, clip=clip, eps=1e-15, sharp=False, label=f"{form} step {k} array {i}")
        assert abs(c["norm"] / norm - 1) < 1e-6 and abs(c["clip"] / clip - 1) < 1e-6


@pytest.mark.parametrize("form", FORMS)
def test_moments_follow_their_gaussians(form):
    import torch
    from examples.train_field import ARRAYS
    t = trainer(form, n=1500, dims=32, capacity=2000)
    for _ in range(5):
        t.step()
    t.sets[t.now].weight_logit[::7] = -9.0  # below the pruning weight
    t.step()
    old_n = t.n
    before = [snapshot(x) for x in t.adam.tensors]
    t.densify(300)
    torch.cuda.synchronize()
    assert 1000 < t.n < old_n + 300
    src = host(t.source)[:t.n].astype(np.int64)
    kept = src >= 0
    assert kept.sum() <= old_n - old_n // 7 and (~kept).sum() > 0
    for (_, w, _), x, b in zip(ARRAYS, t.adam.tensors, before):
        after = snapshot(x)
        for k in ("m", "v"):
            want = np.where(kept[:, None], b[k].reshape(-1, w)[np.where(kept, src, 0)], 0.0).reshape(-1)
            if form == "f32":
                np.testing.assert_array_equal(after[k], want)
            else:  # a value's new scale may be larger: half a place of 1/8, twice that for v = s s, or of the grid's end
                top = np.repeat(np.array([np.abs(want[i:i + 32]).max() for i in range(0, len(want), 32)]), 32)[:len(want)]
                low = 2.0 ** -17 * top if k == "m" else 2.0 ** -32 * top
                assert np.all(np.abs(after[k] - want) <= (0.0626 if k == "m" else 0.13) * np.abs(want) + low)
    t.step()
    assert np.isfinite(t.loss())


def plain_updates(t, moments, k):
    """The optimiser's step of a Trainer in float64 torch operations."""
    import torch
    ts = t.adam.tensors
    norm = torch.sqrt(sum(x.grad.double().square().sum() for x in ts))
    clip = torch.where(norm > t.max_norm, t.max_norm / norm, 1.0)
    for x, s in zip(ts, moments):
        g = x.grad.double().view(-1) * clip
        s["m"] = 0.9 * s["m"] + 0.1 * g
        s["v"] = 0.999 * s["v"] + 0.001 * g * g
        u = s["m"] / (1 - 0.9 ** k) / (torch.sqrt(s["v"] / (1 - 0.999 ** k)) + 1e-15)
        x.param.view(-1).sub_((x.lr * u).float())


def learn(t, steps, every, plain):
    """Trains as examples.train_field.train does and returns the PSNR."""
    import torch
    from examples.train_field import ARRAYS
    fresh = lambda n: [{k: torch.zeros(n * w, dtype=torch.float64, device="cuda") for k in "mv"}  # noqa: E731
                       for _, w, _ in ARRAYS]
    moments = fresh(t.n)
    for k in range(1, steps + 1):
        t.gradients()
        if plain:
            plain_updates(t, moments, k)
        else:
            t.update()
        if k % every == 0 and k < steps:
            t.densify(t.sets[0].rows // 10)
            src = t.source[:t.n].long()
            old, moments = moments, fresh(t.n)
            for (_, w, _), a, b in zip(ARRAYS, old, moments):
                for q in "mv":
                    b[q].view(-1, w)[src >= 0] = a[q].view(-1, w)[src[src >= 0]]
    return t.psnr()


def test_the_field_is_learned_as_with_a_plain_optimiser():
    """200 steps with three densifications: the field's PSNR is within 1 dB
    of the one with a float64 optimiser in plain torch operations, for both
    forms of the moments."""
    want = learn(trainer("f32", n=2048, dims=32), 200, 50, plain=True)
    for form in FORMS:
        t = trainer(form, n=2048, dims=32)
        start = t.psnr()
        got = learn(t, 200, 50, plain=False)
        log(f"  {form}: {start:.2f} dB to {got:.2f} dB, with the plain optimiser to {want:.2f} dB; {t.n} Gaussians")
        assert start < want - 1.0 and abs(got - want) < 1.0 and t.n > 2048
