"""gs_shares refuses an index whose arrays are not on the Gaussians' device."""
import numpy as np
import pytest
import torch

import paper_2607_01164_amd as gs
import synth
from test_gpu_budget import DEV, KINDS, Batch

pytestmark = pytest.mark.gpu


def test_index_on_another_device():
    n = 50
    b = Batch(synth.random_gaussians(1, n, log_mu=np.log(0.1)), **KINDS["points"])
    here = b.index.work
    score = torch.full((n,), 7.5, device=DEV)
    with pytest.raises(ValueError, match="index"):
        b.index.work = here.cpu()
        gs.gs_shares(b.gauss, b.index, b.query, b.plan, b.influence, score, b.work)
    assert (score == 7.5).all()
    b.index.work = here
    gs.gs_shares(b.gauss, b.index, b.query, b.plan, b.influence, score, b.work)
    assert (score != 7.5).all()
