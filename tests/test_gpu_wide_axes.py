"""Grids of more than 2^24 voxels, or cells, along an axis: their numbers are
past what float32 holds, and a row's last ones have to be neither left out nor
passed. Sums over the voxels at the far end against float64."""
import numpy as np
import pytest
import torch

import budget_oracle as bo
import paper_2607_01164_amd as gs
import synth
from test_gpu_budget import dev, device_gaussians, voxel_positions

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TAU = 0.01


def two_at_the_ends(size, axis, sigma):
    """A Gaussian at either end of an axis, as wide as `sigma` voxels of size 1."""
    mean = np.tile(np.asarray(size, np.float64) / 2, (2, 1))
    mean[0, axis], mean[1, axis] = size[axis] - sigma / 2, sigma / 3
    return synth.Gaussians(mean.astype(np.float32), np.full((2, 3), sigma, np.float32),
                           np.tile(np.array([1, 0, 0, 0], np.float32), (2, 1)), np.full(2, 0.5, np.float32),
                           np.array([0.5, 0.25], np.float32))


@pytest.mark.parametrize("kind", ["grid", "jitter"])
@pytest.mark.parametrize("dims,cells", [((2 ** 25 + 4, 2, 1), (1, 1, 1)), ((2 ** 24 + 2, 2, 1), (2, 1, 1)),
                                        ((1, 2 ** 25 + 4, 2), (1, 1, 1)), ((2, 1, 2 ** 24 + 2), (1, 1, 2))])
def test_voxels(kind, dims, cells):
    """gs_shares and the backward's dL/dw, whose sums over a Gaussian's voxels
    are the same but for the weight."""
    axis, nvox = int(np.argmax(dims)), int(np.prod(dims))
    size = tuple(float(d) for d in dims)  # voxels of size 1
    g = two_at_the_ends(dims, axis, 30.0)
    gauss, grid = device_gaussians(g), gs.make_grid(cells, (0.0, 0.0, 0.0), size)
    index = gs.build_index(gauss, grid, TAU)
    plan = offsets = None
    ones = torch.ones(nvox, device=DEV)
    if kind == "grid":
        query = gs.Query.grid(dims)
    else:
        offsets = torch.rand(nvox, 3, device=DEV, generator=torch.Generator(DEV).manual_seed(1))
        query = gs.Query.jitter(dims, offsets)
        plan = gs.alloc_plan(query, grid, DEV)
        gs.gs_sample(gauss, index, query, torch.empty_like(ones), torch.empty_like(ones), plan)
    # the voxels of both ends; every other one is farther than the cutoff
    reach = 200
    along = np.concatenate([np.arange(reach), np.arange(dims[axis] - reach, dims[axis])])
    xyz = [along if j == axis else np.arange(dims[j]) for j in range(3)]
    x, y, z = (a.ravel() for a in np.meshgrid(*xyz, indexing="ij"))
    ids = x + dims[0] * (y + dims[1] * z)
    u = np.float32(0.5) if offsets is None else offsets[torch.from_numpy(ids).to(DEV)].cpu().numpy()
    points = voxel_positions(dims, ids, u, (0, 0, 0), size)
    ref, tol = bo.shares(g, points, np.ones(len(ids)), tau=TAU, hi=size)
    assert ref.min() > 10 and tol.max() < 0.005  # a voxel too few or too many is more
    out = torch.empty(2, device=DEV)
    gs.gs_shares(gauss, index, query, plan, ones, out, gs.alloc_shares_work(index, query, DEV))
    assert (np.abs(out.cpu().numpy() - ref) <= tol).all(), (out, ref)
    if kind == "grid":
        grads, zero = gs.Grads.empty(2, DEV), torch.zeros(nvox, device=DEV)
        gs.gs_sample_backward(gauss, index, query, plan, zero, ones, zero, ones, grads,
                              gs.alloc_backward_work(index, query, DEV))
        # (pairs at the cutoff, 0.01 each, are decided in float32 there)
        assert (np.abs(grads.weight.cpu().numpy() - ref / g.weight) <= tol / g.weight + 0.03).all()


@pytest.mark.parametrize("cells", [(2 ** 22 + 1, 1, 1), (2 ** 22 + 2, 2, 1), (2 ** 24 + 3, 1, 1)])
def test_cells(cells):
    """Points at either end of an axis of cells, some past it: those of the
    last cell count, those outside for nothing whatever their influence."""
    size = tuple(float(c) for c in cells)  # cells of size 1
    g = two_at_the_ends(cells, 0, 30.0)
    r = np.random.default_rng(0)
    n = 3001
    points = r.uniform(0, 1, (n, 3)) * np.asarray([1.0, size[1], size[2]])
    points[:, 0] = np.where(r.random(n) < 0.5, r.uniform(-30, 150, n), size[0] + r.uniform(-150, 30, n))
    points = points.astype(np.float32)
    gauss, grid, query = device_gaussians(g), gs.make_grid(cells, (0.0, 0.0, 0.0), size), gs.Query.pts(dev(points))
    index = gs.build_index(gauss, grid, TAU)
    plan, value, influence = gs.alloc_plan(query, grid, DEV), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    gs.gs_sample(gauss, index, query, value, influence, plan)
    work, out = gs.alloc_shares_work(index, query, DEV), torch.empty(2, device=DEV)
    ones = np.ones(n, np.float32)
    inside = ((points >= 0) & (points <= np.asarray(size, np.float32))).all(1)
    assert 0.1 < (~inside).mean() < 0.3
    ref, tol = bo.shares(g, points, ones, tau=TAU, hi=size)
    beyond = bo.shares(g, points, np.where(inside, 0, ones), tau=TAU, lo=(-99, -99, -99), hi=(2.0 ** 25,) * 3)[0]
    assert beyond[0] > 50 and tol.max() < 0.02  # the points past the far end would show
    gs.gs_shares(gauss, index, query, plan, dev(ones), out, work)
    assert (np.abs(out.cpu().numpy() - ref) <= tol).all(), (out, ref)
    # dL/dw with dL/dI = 1: the sum of G over the defined points (pairs at the
    # cutoff, 0.01 each, are decided in float32 there)
    gs.gs_shares(gauss, index, query, plan, influence, out, work, gain=influence)
    grads = gs.Grads.empty(2, DEV)
    gs.gs_sample_backward(gauss, index, query, plan, value, influence, torch.zeros_like(value), dev(ones), grads,
                          gs.alloc_backward_work(index, query, DEV))
    assert (np.abs(grads.weight.cpu().numpy() * g.weight - out.cpu().numpy()) <= 2 * tol + 0.03).all()


@pytest.mark.parametrize("cells", [(2 ** 24 + 2, 1, 1), (2 ** 25 + 4, 1, 1), (1, 2, 2 ** 24 + 2)])
def test_index_boxes(cells):
    """The index lists the last cells of an axis, none past them, and points
    there are defined: I against float64."""
    axis = int(np.argmax(cells))
    size = tuple(float(c) for c in cells)
    g = two_at_the_ends(cells, axis, 30.0)
    r = np.random.default_rng(1)
    n = 501
    points = r.uniform(0, 1, (n, 3)) * np.asarray(size)
    points[:, axis] = np.where(r.random(n) < 0.4, r.uniform(0, 150, n), size[axis] - r.uniform(0, 150, n))
    points = points.astype(np.float32)
    gauss, grid, query = device_gaussians(g), gs.make_grid(cells, (0.0, 0.0, 0.0), size), gs.Query.pts(dev(points))
    index = gs.build_index(gauss, grid, TAU)
    keys = index.keys[:index.n_pairs].cpu().numpy().astype(np.uint32)
    ncells = int(np.prod(cells))
    assert keys.max() == ncells - 1 and index.cell_offsets[ncells] == index.n_pairs
    value, influence = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    gs.gs_sample(gauss, index, query, value, influence, gs.alloc_plan(query, grid, DEV))
    ref, slack = np.zeros(n), np.zeros(n)
    for i in range(2):
        q = (bo.whitened(g, i, points) ** 2).sum(1)
        ref += np.where(q <= bo.cut(TAU), g.weight[i] * np.exp(-0.5 * q), 0)
        # (pairs at the cutoff are decided in float32)
        slack += np.where(np.abs(q / bo.cut(TAU) - 1) < 1e-5, TAU * g.weight[i], 0)
    got = influence.cpu().numpy()
    sure = ref > TAU * (1 + 1e-3) + slack
    assert sure[points[:, axis] > size[axis] - 4].sum() > 2  # the last cells among them
    assert (np.abs(got - ref)[sure] <= slack[sure] + 1e-4 * ref[sure]).all()
