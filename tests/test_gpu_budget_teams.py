"""gs_shares where several Gaussians share a wave and wide ones are left to
teams of waves (16384 Gaussians and 65536 queries or more): against float64 with
the bound of sums that lanes share, and which Gaussians are left."""
import numpy as np
import pytest
import torch

import budget_oracle as bo
import paper_2607_01164_amd as gs
import synth
from test_gpu_budget import TAU, Batch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TEAM = 8


def left_to_teams(b):
    """The number of Gaussians on the lists behind the workspace's first 256
    bytes."""
    return int(b.work[256:512].view(torch.int32).sum())


def check_some(b, got, some, rows, wide):
    """Scores of Gaussians `some` against float64. rows: of a wide Gaussian, the
    most. Per pair the errors of budget_oracle.shares. A lane of a wave adds
    its share alone: for a team's an eighth of a lane for 64 queries and two
    for a row's ends, half as many again where the waves' shares differ, and 64
    for the batches' ends and the sums over lanes and waves; a Gaussian of K
    queries has no more than K."""
    g = b.g.subset(some)
    points = np.nan_to_num(b.points, nan=1e9)
    inf = b.influence.cpu().numpy()
    inside = ((points >= np.asarray(b.lo, np.float32)) & (points <= np.asarray(b.hi, np.float32))).all(1)
    f = np.zeros(len(points))
    f[inside & (inf > 0)] = 1 / inf[inside & (inf > 0)].astype(np.float64)
    shared = 1.5 * (len(points) / 64 + 2 * rows) / TEAM + 64
    top = bo.cut(TAU) / (2 * np.log(2))
    for k, i in enumerate(some):
        reach = 3.1 * float(g.scale[k].max())
        near = np.flatnonzero((np.abs(points - g.mean[k]) <= reach).all(1) & (f > 0))
        q = (bo.whitened(g, k, points[near]) ** 2).sum(1)
        t = (float(g.weight[k]) * np.exp(-0.5 * q) * f[near])[q <= bo.cut(TAU)]
        kappa = float(g.scale[k].max() / g.scale[k].min())
        adds = min(len(t), shared) if i in wide else len(t)
        rel = np.log(2) * (10 * np.sqrt(3) + 3) * kappa * bo.E32 * top + bo.EXP_ULP + (adds + 8) * bo.E32
        assert abs(float(got[i]) - t.sum()) <= rel * t.sum() + 1e-37, (i, got[i], t.sum(), rel)


SHAPES = {"points": dict(kind="points", cells=(32, 32, 32), n=300007),
          "grid": dict(kind="grid", cells=(32, 16, 16), dims=(1024, 16, 16)),
          "jitter": dict(kind="jitter", cells=(32, 16, 16), dims=(1024, 16, 16)),
          "stray": dict(kind="jitter", cells=(32, 16, 16), dims=(1024, 16, 16), spread=0.7)}
ROWS = {"points": 1024, "grid": 256, "jitter": 256, "stray": 256}


@pytest.mark.parametrize("kind", list(SHAPES))
@pytest.mark.parametrize("before", [0.02, 0.1, 0.2, 0.25, 0.3])
def test_a_wide_gaussian_behind_others(kind, before):
    """Two Gaussians a wave. The first in the order has some rows, the second,
    wherever in the wave's list its rows begin, reaches all queries and is
    left to a team, alone."""
    n = 16500
    g = synth.random_gaussians(3, n, log_mu=np.log(0.004), log_sd=0.2, lo=0.35, hi=1.0)
    g.mean[0], g.scale[0], g.rot[0] = (0.02, before / 2, before / 2), (0.002, before / 6, before / 6), (1, 0, 0, 0)
    g.mean[1], g.scale[1] = (0.45, 0.5, 0.5), (0.5, 0.6, 0.55)
    b = Batch(g, seed=5, **SHAPES[kind])
    got = b.shares(torch.empty(n, device=DEV)).cpu().numpy()
    assert left_to_teams(b) == 1
    total = int((b.influence > 0).sum())
    check_some(b, got, np.concatenate([[0, 1], np.arange(2, n, 331)]), ROWS[kind], {1})
    assert abs(got.astype(np.float64).sum() - total) <= 2e-5 * len(b.points)


@pytest.mark.parametrize("kind", list(SHAPES))
@pytest.mark.parametrize("n", [16500, 25001, 33001])
def test_shared_waves_and_teams(kind, n):
    """Two, three and four Gaussians a wave, wide ones among them."""
    g = synth.random_gaussians(n, n, log_mu=np.log(0.25 * n ** (-1 / 3)), log_sd=0.3)
    r = np.random.default_rng(n)
    wide = np.unique(r.integers(0, n, 9))
    g.scale[wide] = r.uniform(0.4, 0.6, (len(wide), 3))
    b = Batch(g, seed=n, **SHAPES[kind])
    got = b.shares(torch.empty(n, device=DEV)).cpu().numpy()
    assert left_to_teams(b) == len(wide)
    # in the order of the cells of their boxes' corners: the wide ones' neighbours
    cells = np.asarray(SHAPES[kind]["cells"])
    c = np.clip(np.floor((g.mean - 3.04 * g.scale.max(1, keepdims=True)) * cells), 0, cells - 1).astype(np.int64)
    order = np.argsort(c[:, 0] + cells[0] * (c[:, 1] + cells[1] * c[:, 2]), kind="stable")
    place = np.flatnonzero(np.isin(order, wide))
    near = order[np.unique(np.clip(place[:, None] + np.arange(-6, 7), 0, n - 1))]
    check_some(b, got, np.unique(np.concatenate([wide, near, np.arange(0, n, 401)])), ROWS[kind], set(wide.tolist()))
    total = int((b.influence > 0).sum())
    assert abs(got.astype(np.float64).sum() - total) <= 2e-5 * len(b.points)
