"""Train a Gaussian field on a synthetic volume, from free parameters to the
optimiser's step, everything on the device:

    python examples/train_field.py [--gaussians 4096] [--dims 64] [--steps 600] [--moments 8]

One iteration: activations, cell index, one jittered sample in every voxel,
losses, the sampler's and the activations' backward, then the global gradient
norm (which opens the step, or skips it when a gradient is not finite) and one
AdamW launch over the five parameter arrays, with the paper's learning rates.
Every --densify-every iterations the field is pruned and grown, and the
moments follow their Gaussians through the densification's source map. Moments
are kept in 8 bits or in 32. Prints the loss and, at the end, the PSNR of the
reconstructed volume."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_01164_amd as gs  # noqa: E402

TAU, SCALE_CAP = 0.01, 0.04
PRUNE_WEIGHT, NEW_WEIGHT = 0.005, 0.01
FN_EPS, FN_LAMBDA = 0.1, 1.0
# arrays of the free parameters: width, learning rate
ARRAYS = (("mean", 3, 1.6e-4), ("log_scale", 3, 1e-3), ("rot", 4, 1e-4), ("value_logit", 1, 2.5e-3),
          ("weight_logit", 1, 2.5e-2))


def volume(x):
    """The field to learn, in (0, 1): waves under a few smooth bumps."""
    c = x.new_tensor([[0.3, 0.35, 0.4], [0.7, 0.6, 0.3], [0.5, 0.3, 0.75], [0.25, 0.75, 0.7]])
    bumps = torch.exp(-40.0 * ((x[:, None, :] - c) ** 2).sum(2)).sum(1)
    waves = torch.sin(9.0 * x[:, 0]) * torch.sin(7.0 * x[:, 1] + 1.0) * torch.sin(8.0 * x[:, 2] + 2.0)
    return (0.45 + 0.2 * waves + 0.3 * bumps).clamp(0.02, 0.98)


class Moments:
    """The moments of all arrays, for up to `rows` Gaussians."""

    def __init__(self, rows, form, device):
        self.form, self.arrays = form, []
        for _, w, _ in ARRAYS:
            dt = torch.float32 if form == gs.GS_MOMENTS_F32 else torch.uint8
            a = {k: torch.zeros(rows * w, dtype=dt, device=device) for k in ("m", "v")}
            if form == gs.GS_MOMENTS_MXFP8:
                for k in ("m_scale", "v_scale"):
                    a[k] = torch.zeros(gs.moment_scales(rows * w), dtype=torch.uint8, device=device)
            self.arrays.append(a)

    def first(self, i, n):
        """Array i's moments of n elements."""
        a = self.arrays[i]
        return {k: x[:gs.moment_scales(n) if k.endswith("scale") else n] for k, x in a.items()}


def carry_between(a, b):
    """The moments of `a` into `b`'s arrays, for gs_adamw_carry."""
    return gs.AdamCarry([gs.AdamRows(width=w, m=x["m"], v=x["v"], m_out=y["m"], v_out=y["v"],
                                     m_scale=x.get("m_scale"), v_scale=x.get("v_scale"),
                                     m_scale_out=y.get("m_scale"), v_scale_out=y.get("v_scale"))
                         for (_, w, _), x, y in zip(ARRAYS, a.arrays, b.arrays)])


class Trainer:
    def __init__(self, n=4096, dims=64, moments=gs.GS_MOMENTS_MXFP8, capacity=None, max_norm=1.0, weight_decay=0.0,
                 seed=0, device="cuda:0"):
        self.n, self.dims, self.device, self.seed = n, (dims,) * 3, device, seed
        self.max_norm, self.weight_decay = max_norm, weight_decay
        self.gen = torch.Generator(device=device).manual_seed(seed)
        rows = capacity or 2 * n
        self.sets = [gs.ParamSet.empty(rows, device) for _ in range(2)]
        self.moments = [Moments(rows, moments, device) for _ in range(2)]
        self.carries = [carry_between(self.moments[i], self.moments[1 - i]) for i in range(2)]
        self.now = 0  # which of the two sets is trained
        self.control = gs.alloc_adam_control(device)
        cells = max(4, min(32, dims // 4))
        self.grid = gs.make_grid((cells,) * 3)
        nq = dims ** 3
        f = dict(dtype=torch.float32, device=device)
        self.offsets = torch.empty(nq, 3, **f)
        axis = torch.arange(dims, **f)
        z, y, x = torch.meshgrid(axis, axis, axis, indexing="ij")
        self.voxels = torch.stack([x, y, z], 3).view(-1, 3)  # x fastest
        self.query = gs.Query.jitter(self.dims, self.offsets)
        self.plan = gs.alloc_plan(self.query, self.grid, device)
        self.value, self.influence, self.grad_value, self.grad_influence = (torch.empty(nq, **f) for _ in range(4))
        self.terms, self.loss_work = gs.alloc_loss_terms(device), gs.alloc_loss_work(nq, device)
        self.scale = torch.empty(rows, 3, **f)
        self.act_value, self.weight = torch.empty(rows, **f), torch.empty(rows, **f)
        self.all_grads = gs.Grads.empty(rows, device)
        self.source = torch.empty(rows, dtype=torch.int32, device=device)
        p = self.sets[0]
        p.mean[:n].uniform_(0.0, 1.0, generator=self.gen)
        self.new_log_scale = math.log(0.7 / n ** (1.0 / 3.0))
        p.log_scale[:n] = self.new_log_scale
        p.rot[:n] = torch.tensor([1.0, 0.0, 0.0, 0.0], device=device)
        start = volume(p.mean[:n])
        p.value_logit[:n] = torch.log(start / (1.0 - start))
        p.weight_logit[:n] = math.log(0.1 / 0.9)
        self.index = gs.Index(self.grid, rows, 64 * rows, device)
        self.layout()

    def layout(self):
        """What depends on the number of Gaussians: views and the optimiser's list."""
        n, p, m = self.n, self.sets[self.now], self.moments[self.now]
        self.raw = p.raw(n)
        g = self.all_grads
        self.grads = gs.Grads(g.mean[:n], g.scale[:n], g.rot[:n], g.value[:n], g.weight[:n])
        self.gauss = gs.Gaussians(p.mean[:n], self.scale[:n], p.rot[:n], self.act_value[:n], self.weight[:n])
        # the activations' backward overwrites the gradients it reads
        grads = (self.grads.mean, self.grads.scale, self.grads.rot, self.grads.value, self.grads.weight)
        self.raw_grads = gs.RawParams(self.grads.scale, self.grads.value, self.grads.weight)
        self.adam = gs.AdamPlan([
            gs.AdamTensor(param=getattr(p, name)[:n], grad=grad, lr=lr, weight_decay=self.weight_decay,
                          **m.first(i, n * w))
            for i, ((name, w, lr), grad) in enumerate(zip(ARRAYS, grads))])

    def build_index(self):
        try:
            gs.gs_build_index(self.gauss, self.grid, TAU, self.index)
        except gs.GsError as e:
            if e.status != gs.GS_ERR_CAPACITY:
                raise
            self.index = gs.Index(self.grid, self.scale.shape[0], int(1.3 * self.index.n_pairs), self.device)
            gs.gs_build_index(self.gauss, self.grid, TAU, self.index)

    def step(self):
        """One iteration; nothing of it but the index's pair count is waited for."""
        self.gradients()
        self.update()

    def gradients(self):
        gs.gs_activate(self.raw, SCALE_CAP, self.gauss.scale, self.gauss.value, self.gauss.weight)
        self.build_index()
        self.offsets.uniform_(0.0, 1.0, generator=self.gen)
        self.target = volume((self.voxels + self.offsets) / self.dims[0])
        gs.gs_sample(self.gauss, self.index, self.query, self.value, self.influence, self.plan)
        gs.gs_loss(self.value, self.influence, self.target, None, TAU, FN_EPS, FN_LAMBDA, 0.0, self.grad_value,
                   self.grad_influence, self.terms, self.loss_work)
        work = gs.alloc_backward_work(self.index, self.query, self.device)
        gs.gs_sample_backward(self.gauss, self.index, self.query, self.plan, self.value, self.influence,
                              self.grad_value, self.grad_influence, self.grads, work)
        gs.gs_activate_backward(self.raw, SCALE_CAP, self.grads, self.raw_grads)

    def update(self):
        gs.gs_grad_norm(self.adam, self.control, max_norm=self.max_norm)
        gs.gs_adamw(self.adam, control=self.control, eps=1e-15, seed=self.seed)

    def densify(self, max_new):
        """Prunes and grows the field after a step; moments follow."""
        old, new = self.now, 1 - self.now
        work = gs.alloc_densify_work(self.n, self.query, self.device)
        n = gs.gs_densify(self.sets[old], self.n, self.gauss.weight, self.grid, self.query, self.value,
                          self.influence, self.target, None, PRUNE_WEIGHT, TAU, self.new_log_scale,
                          math.log(NEW_WEIGHT / (1.0 - NEW_WEIGHT)), max_new, self.sets[new], self.source, work)
        gs.gs_adamw_carry(self.carries[old], self.n, self.source, n)
        self.n, self.now = n, new
        self.layout()

    def loss(self):
        return gs.read_loss_terms(self.terms)["total"]

    def psnr(self):
        """Of the reconstruction at all voxel centres, for values in (0, 1)."""
        gs.gs_activate(self.raw, SCALE_CAP, self.gauss.scale, self.gauss.value, self.gauss.weight)
        self.build_index()
        gs.gs_sample(self.gauss, self.index, gs.Query.grid(self.dims), self.value, self.influence)
        err = (self.value - volume((self.voxels + 0.5) / self.dims[0])).double().square().mean()
        return -10.0 * math.log10(float(err))


def train(t, steps, densify_every=100, report=None):
    """`steps` iterations of a Trainer; returns [(step, Gaussians, loss)]."""
    seen = []
    for k in range(1, steps + 1):
        t.step()
        if densify_every and k % densify_every == 0 and k < steps:
            t.densify(t.sets[0].rows // 10)
        if k % 50 == 0 or k in (1, steps):
            seen.append((k, t.n, t.loss()))
            if report:
                report(*seen[-1])
    return seen


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--gaussians", type=int, default=4096)
    ap.add_argument("--dims", type=int, default=64, help="voxels per axis, a multiple of 16")
    ap.add_argument("--steps", type=int, default=600)
    ap.add_argument("--moments", type=int, choices=(8, 32), default=8, help="bits of the optimiser's moments")
    ap.add_argument("--densify-every", type=int, default=100)
    a = ap.parse_args()
    t = Trainer(a.gaussians, a.dims, gs.GS_MOMENTS_MXFP8 if a.moments == 8 else gs.GS_MOMENTS_F32)
    train(t, a.steps, a.densify_every,
          lambda k, n, x: print(f"step {k:5d}  {n:8d} Gaussians  loss {x:.5f}", flush=True))
    c = gs.read_adam_control(t.control)
    print(f"{c['step']} steps, {c['skipped']} skipped, last gradient norm {c['norm']:.3g}, PSNR {t.psnr():.2f} dB")


if __name__ == "__main__":
    main()
