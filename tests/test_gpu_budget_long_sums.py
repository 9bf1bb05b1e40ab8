"""gs_shares of a Gaussian that millions of queries reach: its sum is as good as
a short one."""
import numpy as np
import pytest
import torch

import budget_oracle as bo
import synth
from test_gpu_budget import TAU, Batch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("kind,cells,n", [("points", (32, 32, 32), 1 << 21), ("points", (1, 1, 1), 1 << 21),
                                          ("points", (4, 4, 4), 65535), ("grid", (16, 16, 16), 128),
                                          ("jitter", (32, 32, 32), 128), ("jitter", (2, 128, 2), 40)])
def test_a_gaussian_over_all_queries(kind, cells, n):
    """Per pair the errors of budget_oracle.shares (10 sqrt(3) + 3) kappa in Q'.
    From 65536 queries on a team's lane adds 64 terms in float32 before they go
    to 64 bits, below them a lane adds its 64th of the queries, and one more at
    either end of each row; then come 6 sums over the lanes, 8 over the waves,
    and the weight."""
    g = synth.random_gaussians(3, 300, log_mu=np.log(0.01), log_sd=0.2)
    g.mean[1], g.scale[1] = (0.45, 0.5, 0.5), (0.5, 0.6, 0.55)
    if kind == "points":
        b = Batch(g, kind, cells, points=np.random.default_rng(1).random((n, 3), dtype=np.float32))
    else:
        b = Batch(g, kind, cells, (n, n, n))
    got = b.shares(torch.empty(300, device=DEV)).cpu().numpy()
    inf = b.influence.cpu().numpy().astype(np.float64)
    f = np.where(inf > 0, 1 / np.where(inf > 0, inf, 1), 0)
    q = (bo.whitened(g, 1, b.points) ** 2).sum(1)
    ref = float(g.weight[1]) * (np.exp(-0.5 * q) * f)[q <= bo.cut(TAU)].sum()
    rows = cells[1] * cells[2] if kind == "points" else b.query.dims[1] * b.query.dims[2]
    adds = 64 if len(b.points) >= 65536 else len(b.points) / 64 + 2 * rows
    kappa, top = 0.6 / 0.5, bo.cut(TAU) / (2 * np.log(2))
    rel = np.log(2) * (10 * np.sqrt(3) + 3) * kappa * bo.E32 * top + bo.EXP_ULP + (adds + 6 + 8 + 6) * bo.E32
    assert abs(float(got[1]) - ref) <= rel * ref, (got[1] / ref - 1, rel)
