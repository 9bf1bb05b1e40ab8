"""Draws from more rows than a launch has workgroups (65536 of 256 or 1024
threads, 2^20 of 64): a workgroup's second row, in memory that its first one
has used; far more draws than candidates. Against the definition."""
import numpy as np
import pytest
import torch

import budget_oracle as bo
import paper_2607_01164_amd as gs
from test_gpu_budget import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("settings", [dict(), dict(top_k=256), dict(top_k=300), dict(top_p=0.8),
                                      dict(top_k=20, top_p=0.9, min_p=0.02), dict(temperature=0.0),
                                      dict(top_k=300, top_p=0.7, temperature=0.8)])
@pytest.mark.parametrize("rows,n,launched,logits", [(65540, 513, 65536, False), ((1 << 20) + 3, 33, 1 << 20, False),
                                                    (65537, 4097, 65536, True)])
def test_a_second_row(rows, n, launched, logits, settings):
    """The rows of a second turn and those that the same workgroups had first."""
    gen = torch.Generator(DEV).manual_seed(n)
    x = torch.randn(rows, n, device=DEV, generator=gen)
    if not logits:
        x.mul_(2).exp_()
    if n == 4097:
        x = x.to(torch.bfloat16)
    draws = 3
    u = torch.rand(rows, draws, dtype=torch.float64, device=DEV, generator=gen)
    ids = torch.full((rows, draws), -77, dtype=torch.int32, device=DEV)
    prob = torch.full((rows, draws), -7.0, device=DEV)
    gs.gs_draw(x, u, ids, gs.alloc_draw_work(rows, n, draws, DEV), prob=prob, logits=logits, **settings)
    assert (ids >= 0).all() and (ids < n).all() and (prob > 0).all() and (prob <= 1).all()
    for row in (*range(rows - launched), *range(launched, rows), launched - 1):
        ref, p, _ = bo.draw(x[row].float().cpu().numpy(), u[row].cpu().numpy(), logits=logits, **settings)
        assert np.array_equal(ids[row].cpu().numpy(), ref), row
        assert (np.abs(prob[row].cpu().numpy() - p) <= bo.E32 * p + 1e-12).all(), row


@pytest.mark.parametrize("n,settings", [(300, dict()), (4096, dict(top_p=0.95)), (16384, dict(top_k=2000)),
                                        (50021, dict(top_k=128, top_p=0.9)), (50021, dict(top_p=0.9))])
def test_many_draws(n, settings):
    """Far more draws than a row has candidates, in rising order and in none."""
    gen = torch.Generator(DEV).manual_seed(n)
    x = torch.randn(n, device=DEV, generator=gen).mul_(2).exp_()
    draws = 100003
    u = torch.rand(draws, dtype=torch.float64, device=DEV, generator=gen)
    u[::7] = u[::7].sort().values
    ids = torch.full((draws + 1,), -77, dtype=torch.int32, device=DEV)
    prob = torch.empty(draws, device=DEV)
    gs.gs_draw(x, u, ids, gs.alloc_draw_work(1, n, draws, DEV), prob=prob, **settings)
    ref, p, _ = bo.draw(x.cpu().numpy(), u.cpu().numpy(), **settings)
    assert np.array_equal(ids[:draws].cpu().numpy(), ref) and ids[draws] == -77
    assert (np.abs(prob.cpu().numpy() - p) <= bo.E32 * p + 1e-12).all()
