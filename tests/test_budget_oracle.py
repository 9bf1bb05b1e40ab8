"""The oracle of the budget operators against closed forms and its own
identities (CPU)."""
import math

import numpy as np
import pytest

import budget_oracle as bo
import synth


def test_shares_add_up_to_the_defined_queries(orc):
    g = synth.random_gaussians(3, 40, log_mu=math.log(0.12), log_sd=0.4)
    p = synth.random_points(4, 500)
    ref = orc.forward(g, p)
    inf = ref.inf
    s, _ = bo.shares(g, p, inf)
    assert abs(s.sum() - (inf > 0).sum()) < 1e-9 * len(p)


def test_a_lone_gaussian_takes_all():
    g = synth.Gaussians(np.array([[0.5, 0.5, 0.5]], np.float32), np.full((1, 3), 0.1, np.float32),
                        np.array([[2, 0, 0, 0]], np.float32), np.ones(1, np.float32), np.full(1, 0.5, np.float32))
    p = np.array([[0.5, 0.5, 0.5], [0.6, 0.5, 0.5], [0.9, 0.5, 0.5], [1.5, 0.5, 0.5]], np.float32)
    inf = np.array([0.5, 0.5 * math.exp(-0.5), 0.3, 0.5], np.float32)
    s, tol = bo.shares(g, p, inf, gain=np.array([1, -3, 1, 1], np.float32), score=np.array([4.0]), decay=0.5)
    assert abs(s[0] - (2 + 1 - 3)) < 1e-6 and 0 < tol[0] < 1e-4


def test_evict_order():
    s = np.array([1, np.nan, 3, -0.0, 0.0, 3, -np.inf], np.float32)
    assert list(bo.evict(s, 2)) == [2, 5]
    assert list(bo.evict(s, 1)) == [2]
    assert list(bo.evict(s, 4)) == [0, 2, 3, 5]
    assert list(bo.evict(s, 6)) == [0, 2, 3, 4, 5, 6]
    assert list(bo.evict(s, 9)) == list(range(7))
    pin = np.array([0, 1, 0, 0, 0, 0, 1], np.uint8)
    assert list(bo.evict(s, 1, pin)) == [6]
    assert list(bo.evict(s, 3, pin)) == [1, 2, 6]


def test_draw_filters():
    x = np.array([1, 4, 2, 4, 1], np.float32)
    unit = 1 << bo.bits_of(5)
    assert bo.bits_of(5) == 52 and bo.bits_of(1 << 21) == 41 and bo.bits_of(1) == 52
    assert list(bo.kept(x, 5)) == [unit // 4, unit, unit // 2, unit, unit // 4]
    assert list(np.flatnonzero(bo.kept(x, 5, top_k=1))) == [1]
    assert list(np.flatnonzero(bo.kept(x, 5, top_k=4))) == [0, 1, 2, 3]
    # 12 quarters: before the second 4 there are 4, before the 2 there are 8
    assert list(np.flatnonzero(bo.kept(x, 5, top_p=0.3))) == [1]
    assert list(np.flatnonzero(bo.kept(x, 5, top_p=0.5))) == [1, 3]
    assert list(np.flatnonzero(bo.kept(x, 5, top_p=0.7))) == [1, 2, 3]
    assert list(np.flatnonzero(bo.kept(x, 5, top_p=0.0))) == [1]
    assert list(np.flatnonzero(bo.kept(x, 5, min_p=0.5))) == [1, 2, 3]
    assert list(np.flatnonzero(bo.kept(x, 5, temperature=0))) == [1]
    ids, p, room = bo.draw(x, np.array([0.0, 0.0833, 0.0834, 0.999999, 1.0, np.nan, -1.0]))
    assert list(ids) == [0, 0, 1, 4, 4, 0, 0] and abs(p[2] - 1 / 3) < 1e-15 and (room > 0).all()
    ids, p, _ = bo.draw(np.array([-np.inf, np.nan], np.float32), np.array([0.5]), logits=True)
    assert list(ids) == [-1] and p[0] == 0
    ids, p, _ = bo.draw(np.array([np.inf, 3, np.inf], np.float32), np.array([0.4, 0.6]), temperature=0.7)
    assert list(ids) == [0, 2] and p[0] == 0.5


def test_draw_follows_the_distribution():
    x = np.array([0.5, 2.0, 0.0, 1.0], np.float32)
    u = (np.arange(70000) + 0.5) / 70000
    ids, _, _ = bo.draw(x, u)
    assert np.array_equal(np.bincount(ids, minlength=4), [10000, 40000, 0, 20000])
    ids, _, _ = bo.draw(x, u, logits=True)
    assert np.abs(np.bincount(ids, minlength=4) / 70000 - np.exp(x) / np.exp(x).sum()).max() < 2e-5


@pytest.mark.parametrize("logit", [-800.0, -40.0, -3.0, 0.0, 2.0, 30.0, 800.0])
@pytest.mark.parametrize("c", [1, 2, 7, 1000])
def test_split_shares_the_weight(logit, c):
    got = bo.split_logit(np.array([logit]), [c])[0]
    if logit > -700:
        w = 1 / (1 + math.exp(-logit))
        assert abs(1 / (1 + math.exp(-got)) * c - w) < 1e-14 * w * c
    else:
        assert abs(got - (logit - math.log(c))) < 1e-12 * abs(logit)
    assert bo.split_logit(np.array([-np.inf]), [3])[0] == -np.inf
