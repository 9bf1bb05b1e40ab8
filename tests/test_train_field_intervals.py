"""examples/train_field.py where rebalancing and densification meet: which of
them train() does by default, and that a densification after a rebalance prunes
and carries the rows as they then are."""
import numpy as np
import pytest
import torch

import paper_2607_01164_amd as gs
from examples.train_field import PRUNE_WEIGHT, Trainer, train


class Calls:
    """A Trainer that only notes what is called."""

    def __init__(self):
        self.sets, self.n, self.k, self.seen = [type("Set", (), {"rows": 100})], 50, 0, []

    def step(self, attend=False):
        self.k += 1

    def rebalance(self):
        self.seen.append(("rebalance", self.k))

    def densify(self, max_new):
        self.seen.append(("densify", self.k))

    def loss(self):
        return 0.0


def test_intervals():
    t = Calls()
    train(t, 201)
    assert t.seen == [("densify", 100), ("densify", 200)]
    t = Calls()
    train(t, 250, rebalance_every=100)  # the number is held
    assert t.seen == [("rebalance", 100), ("rebalance", 200)]
    t = Calls()
    train(t, 13, 4, rebalance_every=6)
    assert t.seen == [("densify", 4), ("rebalance", 6), ("densify", 8), ("rebalance", 12), ("densify", 12)]


@pytest.mark.gpu
def test_densify_after_rebalance():
    t = Trainer(moments=gs.GS_MOMENTS_F32, n=1000, dims=32)
    t.sets[0].weight_logit[5:t.n:7] = -8.0  # below the pruning threshold
    for _ in range(3):
        t.step(attend=True)
    t.rebalance()
    n, p = t.n, t.sets[t.now]
    weight = torch.sigmoid(p.weight_logit[:n].double()).cpu().numpy()
    score, mean = t.scores[t.now][:n].cpu().numpy(), p.mean[:n].cpu().numpy()
    stay = np.flatnonzero(weight >= PRUNE_WEIGHT)
    # some go, some with a row in between (a rounding of the threshold is none)
    assert 0 < len(stay) < n and (np.abs(weight / PRUNE_WEIGHT - 1) > 1e-5).all()
    t.densify(40)
    assert t.n == len(stay) + 40
    source = t.source[:t.n].cpu().numpy()
    assert np.array_equal(source[:len(stay)], stay) and (source[len(stay):] < 0).all()
    now = t.scores[t.now][:t.n].cpu().numpy()
    assert np.array_equal(now[:len(stay)], score[stay]) and (now[len(stay):] == 0).all()
    assert np.array_equal(t.sets[t.now].mean[:len(stay)].cpu().numpy(), mean[stay])
    for _ in range(2):
        t.step(attend=True)
    t.rebalance()
    assert torch.isfinite(t.scores[t.now][:t.n]).all()
