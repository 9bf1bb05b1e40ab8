"""The operators of include/gs_budget.h against their definitions in float64
(budget_oracle), at the sizes, masks and orders where they can go wrong, and a
run of them together."""
import math

import numpy as np
import pytest
import torch

import budget_oracle as bo
import paper_2607_01164_amd as gs
import synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TAU = 0.01


def dev(a, dtype=np.float32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).to(DEV)


def device_gaussians(g):
    return gs.Gaussians(dev(g.mean), dev(g.scale), dev(g.rot), dev(g.value), dev(g.weight))


# ---- shares ---------------------------------------------------------------

def voxel_positions(dims, ids, offsets, lo, hi):
    """As gs_sample forms them, every operation rounded to float32."""
    f = np.float32
    ids = np.asarray(ids, np.int64)
    xyz = np.stack([ids % dims[0], ids // dims[0] % dims[1], ids // (dims[0] * dims[1])], 1).astype(f)
    lo, hi = np.asarray(lo, f), np.asarray(hi, f)
    size = ((hi - lo) / np.asarray(dims, f)).astype(f)
    return (lo + ((xyz + offsets).astype(f) * size).astype(f)).astype(f)


class Batch:
    """A field, an index and a batch of queries that were sampled."""

    def __init__(self, g, kind, cells, dims=(0, 0, 0), n=0, seed=0, lo=(0, 0, 0), hi=(1, 1, 1), points=None,
                 spread=0.0, tau=TAU):
        r = np.random.default_rng(seed)
        self.g, self.lo, self.hi = g, lo, hi
        self.gauss = device_gaussians(g)
        grid = gs.make_grid(cells, lo, hi)
        nvox = dims[0] * dims[1] * dims[2]
        if kind == "grid":
            self.points = voxel_positions(dims, np.arange(nvox), np.float32(0.5), lo, hi)
            self.query = gs.Query.grid(dims)
        elif kind == "voxels":
            ids = r.integers(0, nvox, n)
            self.points = voxel_positions(dims, ids, np.float32(0.5), lo, hi)
            ids[: n // 50] = nvox + 3  # no voxel: undefined
            self.points[: n // 50] = np.nan
            self.query = gs.Query.voxels(dims, dev(ids, np.int32))
        elif kind in ("jitter", "jitter_ids"):
            ids = np.arange(nvox) if kind == "jitter" else r.integers(0, nvox, n)
            u = r.random((len(ids), 3), dtype=np.float32)
            if spread:  # offsets that leave their voxels, and some the box
                u = (u + spread * r.standard_normal(u.shape)).astype(np.float32)
            self.points = voxel_positions(dims, ids, u, lo, hi)
            self.query = gs.Query.jitter(dims, dev(u), None if kind == "jitter" else dev(ids, np.int32))
        else:
            if points is None:
                lo_, hi_ = np.asarray(lo), np.asarray(hi)
                points = lo_ + (hi_ - lo_) * r.uniform(-0.05, 1.05, (n, 3))
            self.points = points.astype(np.float32)
            self.query = gs.Query.pts(dev(self.points))
        self.index = gs.build_index(self.gauss, grid, tau)
        self.tau = tau
        m = len(self.points)
        self.value, self.influence = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
        self.plan = None if kind == "grid" else gs.alloc_plan(self.query, grid, DEV)
        gs.gs_sample(self.gauss, self.index, self.query, self.value, self.influence, self.plan)
        self.work = gs.alloc_shares_work(self.index, self.query, DEV)

    def shares(self, score, gain=None, decay=0.0, influence=None, **kw):
        gs.gs_shares(self.gauss, self.index, self.query, self.plan,
                     self.influence if influence is None else influence, score, self.work, gain=gain, decay=decay, **kw)
        return score

    def check(self, gain=None, score=None, decay=0.0, influence=None):
        inf = self.influence.cpu().numpy() if influence is None else influence
        ref, tol = bo.shares(self.g, np.nan_to_num(self.points, nan=1e9), inf, gain, score, decay, self.tau, self.lo,
                             self.hi)
        n = len(self.g.mean)
        out = torch.full((n + 3,), 7.5, device=DEV)  # rows behind the last stay
        out[:n] = float("nan") if score is None else dev(score)
        self.shares(out[:n], None if gain is None else dev(gain), decay,
                    None if influence is None else dev(influence))
        got = out.cpu().numpy()
        assert (got[n:] == 7.5).all()
        assert (np.abs(got[:n] - ref) <= tol).all(), np.max(np.abs(got[:n] - ref) - tol)
        return got[:n]


KINDS = {
    "grid": dict(kind="grid", cells=(4, 4, 4), dims=(16, 12, 20)),
    "grid_coarse": dict(kind="grid", cells=(7, 5, 3), dims=(7, 5, 3)),
    "voxels": dict(kind="voxels", cells=(5, 4, 3), dims=(17, 19, 13), n=1500),
    "jitter": dict(kind="jitter", cells=(4, 5, 3), dims=(13, 11, 9)),
    "jitter_wide": dict(kind="jitter", cells=(4, 5, 3), dims=(13, 11, 9), spread=0.8),
    # from 4096 queries on jittered grids are walked by voxels, unless a
    # position leaves its voxel
    "jitter_voxels": dict(kind="jitter", cells=(4, 5, 3), dims=(21, 18, 17), lo=(-1.0, 0.5, 3.0), hi=(1.0, 1.5, 3.7)),
    "jitter_long": dict(kind="jitter", cells=(1, 64, 2), dims=(2, 30011, 3), lo=(-4.0, 10.0, 0.0), hi=(-3.9, 11.0, 0.1)),
    "jitter_stray": dict(kind="jitter", cells=(4, 5, 3), dims=(21, 18, 17), spread=0.8),
    "jitter_ids": dict(kind="jitter_ids", cells=(3, 3, 3), dims=(30, 31, 29), n=1777),
    "points": dict(kind="points", cells=(6, 6, 6), n=2003),
    "points_box": dict(kind="points", cells=(6, 3, 9), n=1201, lo=(-1.5, 2.0, -0.25), hi=(1.5, 4.0, 0.25)),
}


def scaled_to(g, lo, hi):
    lo, hi = np.asarray(lo), np.asarray(hi)
    size = float(np.prod(hi - lo)) ** (1 / 3)
    return synth.Gaussians((lo + g.mean * (hi - lo)).astype(np.float32), (g.scale * size).astype(np.float32), g.rot,
                           g.value, g.weight)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("n", [1, 2, 63, 65, 150])
def test_shares_of_every_query_kind(kind, n):
    k = KINDS[kind]
    g = synth.random_gaussians(n, n, log_mu=math.log(0.2 * n ** (-1 / 3)), log_sd=0.5, lo=-0.1, hi=1.1)
    b = Batch(scaled_to(g, k.get("lo", (0, 0, 0)), k.get("hi", (1, 1, 1))), seed=n, **k)
    r = np.random.default_rng(n)
    got = b.check()
    assert abs(got.astype(np.float64).sum() - int((b.influence > 0).sum())) <= 2e-5 * len(b.points) + 1e-3
    b.check(gain=r.standard_normal(len(b.points)).astype(np.float32),
            score=r.random(n).astype(np.float32) * 10, decay=0.75)


@pytest.mark.parametrize("kind", ["grid", "jitter", "points"])
def test_shares_many_gaussians_and_long_rows(kind):
    """More than 64 rows a Gaussian, packed waves (65536 Gaussians), tiny ones
    without a query and huge ones."""
    if kind == "points":
        g = synth.random_gaussians(1, 300, log_mu=math.log(0.06), log_sd=1.3)
        Batch(g, "points", (24, 24, 24), n=3001).check()
        return
    g = synth.random_gaussians(2, 65537, log_mu=math.log(0.002), log_sd=0.7)
    g.scale[::4099] *= 60
    k = KINDS[kind]
    b = Batch(g, kind, k["cells"], k["dims"])
    out = b.shares(torch.empty(65537, device=DEV)).cpu().numpy()
    some = np.concatenate([np.arange(0, 65537, 4099), np.arange(5, 65537, 997)])
    sub = g.subset(some)
    ref, tol = bo.shares(sub, b.points, b.influence.cpu().numpy())
    assert (np.abs(out[some] - ref) <= tol).all()
    total = int((b.influence > 0).sum())
    assert abs(out.astype(np.float64).sum() - total) <= 2e-5 * len(b.points)


@pytest.mark.parametrize("kind", ["grid", "jitter", "jitter_stray", "points", "voxels"])
def test_shares_of_gaussians_with_most_of_the_queries(kind):
    """A few Gaussians over the whole domain among small ones, whose queries or
    rows are too many for one wave; queries crowded in a few cells."""
    r = np.random.default_rng(7)
    n = 90
    g = synth.random_gaussians(13, n, log_mu=math.log(0.02), log_sd=0.5)
    g.scale[::9] *= 12
    g.scale[5] = (0.5, 0.4, 0.6)
    if kind == "points":
        crowd = 0.5 + 0.02 * r.standard_normal((60000, 3))
        b = Batch(g, "points", (9, 9, 9), points=np.concatenate([crowd, r.random((10001, 3))]))
    elif kind == "voxels":
        b = Batch(g, "voxels", (9, 9, 9), (50, 51, 52), n=70001)
    else:
        b = Batch(g, kind.split("_")[0], (8, 8, 8), (48, 48, 48), spread=0.7 if kind == "jitter_stray" else 0.0)
    b.check()
    b.check(gain=r.standard_normal(len(b.points)).astype(np.float32), score=r.random(n).astype(np.float32), decay=0.5)
    a = b.shares(torch.empty(n, device=DEV))
    assert all(torch.equal(a, b.shares(torch.empty(n, device=DEV))) for _ in range(3))


def test_shares_left_out_queries():
    """Influence set to 0 by the caller, or not a number: left out; a decay
    without queries."""
    g = synth.random_gaussians(5, 40, log_mu=math.log(0.1))
    for k in ("grid", "points"):
        b = Batch(g, seed=3, **KINDS[k])
        inf = b.influence.cpu().numpy().copy()
        inf[::3] = 0
        inf[1::7] = np.nan
        inf[2::11] = -1
        b.check(influence=inf)
        gain = np.ones(len(inf), np.float32)
        gain[::3] = np.nan  # not read where the influence is 0
        b.check(influence=np.where(np.isnan(gain), 0, b.influence.cpu().numpy()).astype(np.float32), gain=gain)
        score = np.arange(40, dtype=np.float32)
        got = b.check(influence=np.zeros_like(inf), score=score, decay=0.5)
        assert np.array_equal(got, score / 2)
    b = Batch(g, "points", (4, 4, 4), points=np.zeros((0, 3)))
    got = b.check(score=np.arange(40, dtype=np.float32), decay=2.0)
    assert np.array_equal(got, 2 * np.arange(40, dtype=np.float32))
    assert (b.check() == 0).all()


def test_shares_of_invalid_gaussians():
    g = synth.random_gaussians(6, 30, log_mu=math.log(0.15))
    g.mean[3, 1] = np.nan
    g.scale[4, 0] = 0
    g.scale[5, 2] = np.inf
    g.rot[6] = 0
    g.weight[7] = np.nan
    g.value[8] = np.inf
    g.mean[9] = 40.0
    g.weight[10] = 0
    for k in ("grid", "jitter", "voxels"):
        got = Batch(g, **KINDS[k]).check(score=np.full(30, 3, np.float32), decay=1.0)
        assert (got[[3, 4, 5, 6, 7, 8, 9, 10]] == 3).all()


def test_shares_at_the_cutoff():
    """Points around the cutoff's radius, nearer to it than float32 resolves
    Q: which are within is the float64 answer."""
    r = np.random.default_rng(0)
    n, per = 24, 400
    g = synth.random_gaussians(8, n, log_mu=math.log(0.05), log_sd=0.9, lo=0.3, hi=0.7)
    pts, own = [], []
    for i in range(n):
        d = r.standard_normal((per, 3))
        d /= np.linalg.norm(d, axis=1, keepdims=True)
        one = synth.Gaussians(*(a[i:i + 1] for a in (g.mean, g.scale, g.rot, g.value, g.weight)))
        one.mean[:] = 0
        u = bo.whitened(one, 0, d.astype(np.float32))
        d *= (math.sqrt(bo.cut(TAU)) / np.linalg.norm(u, axis=1) * (1 + 1e-7 * r.standard_normal(per)))[:, None]
        pts.append(g.mean[i] + d)
        own.append(np.full(per, i))
    points, own = np.concatenate(pts).astype(np.float32), np.concatenate(own)
    b = Batch(g, "points", (8, 8, 8), points=points)
    # each query counted for its own Gaussian alone would move the sums by
    # 0.01 w a pair, far more than the tolerance
    inf = np.ones(len(points), np.float32)
    b.check(influence=inf)
    q = np.concatenate([(bo.whitened(g, i, points[own == i]) ** 2).sum(1) for i in range(n)])
    inside = q <= bo.cut(TAU)
    assert 0.2 < inside.mean() < 0.8  # they do lie on both sides


def test_shares_repeat_bit_for_bit():
    g = synth.random_gaussians(9, 3000, log_mu=math.log(0.03))
    for k in ("grid", "jitter", "points"):
        b = Batch(g, seed=1, **KINDS[k])
        a = b.shares(torch.empty(3000, device=DEV))
        c = b.shares(torch.empty(3000, device=DEV))
        assert torch.equal(a, c)


# ---- evict ----------------------------------------------------------------

ARRAYS = ("mean", "log_scale", "rot", "value_logit", "weight_logit")


def param_set(rows, seed):
    r = np.random.default_rng(seed)
    shape = dict(mean=3, log_scale=3, rot=4)
    return gs.ParamSet(**{k: dev(r.standard_normal((rows, shape[k]) if k in shape else rows)) for k in ARRAYS})


def scores_of(kind, n, r):
    s = r.standard_normal(n).astype(np.float32)
    if kind == "ties":
        s = np.round(s).astype(np.float32)
    elif kind == "equal":
        s[:] = 0.25
    elif kind == "zeros":
        s = np.where(r.random(n) < 0.7, 0, np.exp(3 * s)).astype(np.float32)
        s[r.random(n) < 0.2] *= -1  # -0 among them
    elif kind == "odd":
        s[r.random(n) < 0.3] = np.nan
        s[r.random(n) < 0.1] = np.inf
        s[r.random(n) < 0.1] = -np.inf
        s[r.random(n) < 0.1] = 1e-42
    return s


def check_evict(n, budget, score, pinned=None, want_score=True, seed=0):
    p = param_set(n, seed)
    keep = min(n, budget)
    out = gs.ParamSet.empty(keep + 2, DEV)
    for k in ARRAYS:
        getattr(out, k).fill_(-9)
    source = torch.full((keep + 2,), -7, dtype=torch.int32, device=DEV)
    score_out = torch.full((keep + 2,), -9.0, device=DEV) if want_score else None
    got = gs.gs_evict(p, n, dev(score), budget, out, source, gs.alloc_evict_work(n, DEV),
                      pinned=None if pinned is None else dev(pinned, np.uint8), score_out=score_out)
    ref = bo.evict(score, budget, pinned)
    assert got == keep == len(ref)
    s = source.cpu().numpy()
    assert np.array_equal(s[:keep], ref) and (s[keep:] == -7).all()
    at = torch.from_numpy(ref).to(DEV)
    for k in ARRAYS:
        x, y = getattr(out, k), getattr(p, k)
        assert torch.equal(x[:keep], y[at]) and (x[keep:] == -9).all(), k
    if want_score:
        assert np.array_equal(score_out[:keep].cpu().numpy(), score[ref], equal_nan=True)
        assert (score_out[keep:] == -9).all()


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "zeros", "odd"])
@pytest.mark.parametrize("n,budget", [(1, 1), (2, 1), (63, 62), (1024, 1000), (1025, 1), (1025, 5000), (4097, 2048),
                                      (30011, 17), (30011, 30010), (150001, 99999)])
def test_evict(kind, n, budget):
    r = np.random.default_rng(n + budget)
    check_evict(n, budget, scores_of(kind, n, r))
    pinned = (r.random(n) < 0.2).astype(np.uint8) * 5
    check_evict(n, budget, scores_of(kind, n, r), pinned, want_score=False)


def test_evict_pinned_beyond_the_budget():
    r = np.random.default_rng(3)
    for n in (500, 40000):
        check_evict(n, n // 4, scores_of("ties", n, r), (r.random(n) < 0.6).astype(np.uint8))
        check_evict(n, n // 4, scores_of("odd", n, r), np.ones(n, np.uint8))
        check_evict(n, n // 4, scores_of("odd", n, r), (np.arange(n) % 4 == 0).astype(np.uint8))


def test_evict_a_large_set():
    """Stretches of more than a tile."""
    n = (1 << 21) + 3
    r = np.random.default_rng(4)
    check_evict(n, n // 2 + 1, scores_of("zeros", n, r))
    check_evict(n, n - 1, scores_of("plain", n, r), (r.random(n) < 0.5).astype(np.uint8))


def test_evict_nothing():
    p, out = param_set(5, 0), gs.ParamSet.empty(5, DEV)
    src = torch.full((5,), -7, dtype=torch.int32, device=DEV)
    assert gs.gs_evict(p, 5, torch.zeros(5, device=DEV), 0, out, src, gs.alloc_evict_work(5, DEV)) == 0
    assert gs.gs_evict(p, 0, torch.zeros(5, device=DEV), 3, out, src, gs.alloc_evict_work(0, DEV)) == 0
    assert (src == -7).all()


# ---- draw -----------------------------------------------------------------

FILTERS = [dict(), dict(top_k=1), dict(top_k=7), dict(top_p=0.8), dict(top_p=0.0), dict(min_p=0.25), dict(min_p=1.0),
           dict(top_k=40, top_p=0.9, min_p=0.05), dict(temperature=0.0), dict(temperature=0.6, top_k=300, top_p=0.5),
           dict(temperature=1.7), dict(top_k=10 ** 9, top_p=0.999), dict(temperature=1e-3, top_p=0.5)]


def scores_for(kind, rows, n, r):
    x = r.standard_normal((rows, n)).astype(np.float32)
    if kind == "weights":
        x = np.exp(2 * x)
    elif kind == "logits":
        x = 3 * x
    elif kind == "ties":  # few distinct weights, many of them 0
        x = np.clip(np.round(2 * x), 0, 3)
    elif kind == "tied_logits":
        x = np.round(x)
    elif kind == "odd":
        x[r.random(x.shape) < 0.3] = np.nan
        x[r.random(x.shape) < 0.3] = -1
        x[r.random(x.shape) < 0.1] = 1e-41
    elif kind == "odd_logits":
        x[r.random(x.shape) < 0.3] = -np.inf
        x[r.random(x.shape) < 0.1] = np.nan
        x[r.random(x.shape) < 0.1] = np.finfo(np.float32).min
        x[r.random(x.shape) < 0.1] = -0.0
    elif kind == "infinite":
        x[:, :: max(1, n // 3)] = np.inf
    return x.astype(np.float32)


def check_draw(x, draws, logits, settings, seed=0, lengths=None, bf16=False, pad=0):
    rows, n = x.shape
    r = np.random.default_rng(seed)
    u = r.random((rows, draws))
    if draws > 3:
        u[:, 0], u[:, 1], u[:, 2] = 0.0, 1.0, np.nextafter(1.0, 0)
    t = torch.full((rows, n + pad), float("nan"), device=DEV)
    t[:, :n] = dev(x)
    if bf16:
        t = t.to(torch.bfloat16)
        x = t[:, :n].float().cpu().numpy()
    ids = torch.full((rows * draws + 5,), -77, dtype=torch.int32, device=DEV)
    prob = torch.full((rows * draws + 5,), -7.0, device=DEV)
    gs.gs_draw(t[:, :n], dev(u, np.float64), ids, gs.alloc_draw_work(rows, n, draws, DEV), prob=prob, logits=logits,
               lengths=None if lengths is None else dev(lengths, np.int32), **settings)
    assert (ids[rows * draws:] == -77).all() and (prob[rows * draws:] == -7).all()
    ids = ids[:rows * draws].view(rows, draws).cpu().numpy()
    prob = prob[:rows * draws].view(rows, draws).cpu().numpy()
    for i in range(rows):
        cut = n if lengths is None else min(max(int(lengths[i]), 0), n)
        ref, p, room = bo.draw(x[i, :cut], u[i], n=n, logits=logits, **settings)
        # exp and log are good to an ulp on either side, which may move a
        # border by a few units of 2^-k a candidate: no draw is that near one
        assert np.array_equal(ids[i], ref), (i, np.flatnonzero(ids[i] != ref)[:5], room[ids[i] != ref][:5])
        assert (np.abs(prob[i] - p) <= bo.E32 * p + 1e-12).all()


@pytest.mark.parametrize("kind", ["weights", "logits", "ties", "tied_logits", "odd", "odd_logits", "infinite"])
@pytest.mark.parametrize("rows,n,draws", [(1, 1, 4), (3, 2, 5), (5, 63, 9), (4, 64, 1), (3, 511, 70), (2, 513, 300),
                                          (2, 4096, 20), (2, 5001, 33), (1, 16384, 64)])
def test_draw_rows(kind, rows, n, draws):
    logits = kind in ("logits", "tied_logits", "odd_logits", "infinite")
    r = np.random.default_rng(n + draws)
    for k, settings in enumerate(FILTERS):
        check_draw(scores_for(kind, rows, n, r), draws, logits, settings, seed=k)


@pytest.mark.parametrize("kind", ["weights", "logits", "ties", "tied_logits", "odd", "odd_logits"])
@pytest.mark.parametrize("rows,n,draws", [(1, 16385, 50), (3, 20011, 7), (1, 65536, 256), (1, 16385, 257),
                                          (2, 20011, 300), (1, 65537, 9)])
def test_draw_long_rows(kind, rows, n, draws):
    logits = kind.endswith("logits")
    r = np.random.default_rng(n + draws)
    for k, settings in enumerate(FILTERS):
        check_draw(scores_for(kind, rows, n, r), draws, logits, settings, seed=k)


@pytest.mark.parametrize("settings", [dict(), dict(top_p=0.7), dict(top_k=1000), dict(top_k=90000, top_p=0.95)])
def test_draw_very_long_rows(settings):
    """More than a stretch's least length in each of its 1024 stretches."""
    r = np.random.default_rng(11)
    x = scores_for("weights", 1, (1 << 21) + 5, r)
    x[0, 1000000:1500000] = 0
    check_draw(x, 5000, False, settings)
    check_draw(scores_for("ties", 1, (1 << 21) + 5, r), 100, False, settings)


@pytest.mark.parametrize("kind", ["weights", "tied_logits", "odd_logits", "infinite"])
@pytest.mark.parametrize("n,top_k", [(16385, 1), (16385, 1024), (16385, 8193), (50021, 200), (50021, 1024),
                                     (50021, 1025), (278529, 910), (278529, 911), (200003, 130), (999983, 17)])
def test_draw_few_of_long_rows(kind, n, top_k):
    """A stretch of 16384 candidates lists its first top_k <= 1024, and a row is
    drawn from its lists where they hold 16384 together; equals across stretches."""
    logits = kind != "weights"
    x = scores_for(kind, 2, n, np.random.default_rng(n + top_k))
    for k, settings in enumerate([dict(), dict(top_p=0.8, temperature=0.7), dict(top_p=0.5, min_p=0.1)]):
        check_draw(x, 40, logits, dict(settings, top_k=top_k), seed=k, lengths=[n, n - 16383] if k == 1 else None)
    check_draw(x, 3, logits, dict(temperature=0.0, top_k=top_k))
    check_draw(x, 5, logits, dict(top_k=top_k), bf16=True, pad=3)


@pytest.mark.parametrize("order", ["none", "rising", "falling", "late"])
@pytest.mark.parametrize("n,ks", [(500, (63, 64, 65, 499, 500)), (4000, (200, 256, 257)), (16000, (1, 1024, 1025)),
                                  (40000, (64, 1024, 1025, 5461))])
def test_draw_top_k_around_a_workgroup(order, n, ks):
    """As many candidates as a workgroup's threads, one less and one more;
    sorted rows, and rows whose candidates stand in the last threads."""
    r = np.random.default_rng(n)
    x = scores_for("logits", 2, n, r)
    if order == "late":
        x[:, : n - n // 7] = -np.inf
    elif order != "none":
        x = np.sort(x, axis=1)[:, :: 1 if order == "rising" else -1].copy()
    for k in ks:
        check_draw(x, 30, True, dict(top_k=k), seed=k)
        check_draw(x, 30, True, dict(top_k=k, top_p=0.7, min_p=0.01, temperature=1.5), seed=k)
        check_draw(np.round(x), 30, True, dict(top_k=k, top_p=0.9, temperature=2.0), seed=k)


def test_draw_best_of_a_huge_row():
    n = (1 << 28) + 7
    x = torch.zeros(n, device=DEV)
    ids = torch.empty(2, dtype=torch.int32, device=DEV)
    prob = torch.empty(2, device=DEV)
    u = torch.tensor([0.0, 0.99], dtype=torch.float64, device=DEV)
    work = gs.alloc_draw_work(1, n, 2, DEV)
    for at in (0, 16384, (1 << 28) + 2):
        x[at:at + 3] = 1.0 + at
        gs.gs_draw(x, u, ids, work, prob=prob, temperature=0.0)
        assert ids.tolist() == [at, at] and prob.tolist() == [1.0, 1.0]


@pytest.mark.parametrize("n,draws", [(70, 6), (600, 6), (5000, 6), (17000, 6), (17000, 260)])
def test_draw_types_strides_and_lengths(n, draws):
    r = np.random.default_rng(n)
    for k, settings in enumerate(FILTERS):
        check_draw(scores_for("logits", 5, n, r), draws, True, settings, seed=k, bf16=True, pad=k % 3)
        check_draw(scores_for("weights", 5, n, r), draws, False, settings, seed=k, pad=1,
                   lengths=[0, 1, n, n // 2, n + 9])
        check_draw(scores_for("tied_logits", 3, n, r), draws, True, settings, seed=k, pad=5, lengths=[-3, n - 1, 2])
    check_draw(np.zeros((2, n), np.float32), draws, False, dict(top_p=0.5))  # nothing to draw
    check_draw(np.full((2, n), -np.inf, np.float32), draws, True, dict(top_k=3))
    check_draw(np.full((2, n), 7.0, np.float32), draws, True, dict(top_k=3, top_p=0.5))


def test_draw_many_rows():
    r = np.random.default_rng(1)
    check_draw(scores_for("weights", 2000, 33, r), 3, False, dict(top_k=5, top_p=0.9))
    check_draw(scores_for("weights", 40, 16385, r), 2, False, dict(top_p=0.9))
    check_draw(scores_for("weights", 300, 16400, r), 300, False, dict(top_k=500, top_p=0.9))


def test_draw_empty_shapes():
    w = gs.alloc_draw_work(3, 0, 2, DEV)
    ids = torch.full((6,), -77, dtype=torch.int32, device=DEV)
    prob = torch.full((6,), -7.0, device=DEV)
    gs.gs_draw(torch.empty(3, 0, device=DEV), torch.rand(3, 2, dtype=torch.float64, device=DEV), ids, w, prob=prob)
    assert (ids == -1).all() and (prob == 0).all()
    gs.gs_draw(torch.ones(0, 5, device=DEV), torch.rand(0, 2, dtype=torch.float64, device=DEV), ids, w)
    gs.gs_draw(torch.ones(5, device=DEV), torch.rand(0, dtype=torch.float64, device=DEV), ids, w)
    assert (ids == -1).all()


def test_draw_odd_uniform_numbers():
    x = torch.tensor([1.0, 2.0, 0.0, 3.0], device=DEV)
    u = torch.tensor([float("nan"), -0.5, 0.0, 1.0, 7.0, float("inf"), -float("inf"), 0.5], dtype=torch.float64,
                     device=DEV)
    ids = torch.empty(8, dtype=torch.int32, device=DEV)
    gs.gs_draw(x, u, ids, gs.alloc_draw_work(1, 4, 8, DEV))
    assert ids.tolist() == [0, 0, 0, 3, 3, 3, 0, 3]


# ---- split ----------------------------------------------------------------

def check_split(n, ids, seed=0, logits=None):
    ids = np.asarray(ids, np.int32)
    count = len(ids)
    rows = n + count + 2
    p = param_set(rows, seed)
    if logits is not None:
        p.weight_logit[:n] = dev(logits)
    before = {k: getattr(p, k).cpu().numpy().copy() for k in ARRAYS}
    score = torch.rand(rows, device=DEV)
    s0 = score.cpu().numpy().copy()
    source = torch.full((rows,), 5, dtype=torch.int32, device=DEV)
    assert gs.gs_split(p, n, dev(ids, np.int32), source, gs.alloc_split_work(n, DEV), score=score) == n + count
    fine = (ids >= 0) & (ids < n)
    copies = 1 + np.bincount(ids[fine], minlength=n)[:n]
    after = {k: getattr(p, k).cpu().numpy() for k in ARRAYS}
    for k in ("mean", "log_scale", "rot", "value_logit"):
        assert np.array_equal(after[k][:n], before[k][:n])
        assert np.array_equal(after[k][n:n + count][fine], before[k][ids[fine]])
    ref = bo.split_logit(before["weight_logit"][:n], copies)
    got = after["weight_logit"]
    one = copies == 1
    assert np.array_equal(got[:n][one], before["weight_logit"][:n][one], equal_nan=True)
    # float64 of a sum whose terms may cancel near a shared weight of 1/2,
    # rounded once
    err = np.abs(got[:n] - ref)
    same = (got[:n] == ref) | (np.isnan(got[:n]) & np.isnan(ref))
    assert (same | (err <= bo.E32 * np.abs(ref) + 1e-14)).all()
    assert np.array_equal(got[n:n + count][fine], got[ids[fine]], equal_nan=True)
    s = score.cpu().numpy()
    assert (np.abs(s[:n] - s0[:n] / copies) <= bo.E32 * s0[:n]).all()
    assert np.array_equal(s[n:n + count][fine], s[ids[fine]])
    src = source.cpu().numpy()
    assert (src[:n] == 5).all() and (src[n + count:] == 5).all()
    assert np.array_equal(src[n:n + count], np.where(ids >= 0, -1 - ids.astype(np.int64), -1))
    bad = np.flatnonzero(~fine) + n
    assert np.isnan(after["mean"][bad]).all() and (after["weight_logit"][bad] == -np.inf).all()
    assert (after["log_scale"][bad] == 0).all() and (after["rot"][bad] == [1, 0, 0, 0]).all()
    assert (after["value_logit"][bad] == 0).all() and (s[bad] == 0).all()
    for k in ARRAYS:
        assert np.array_equal(after[k][n + count:], before[k][n + count:])
    assert np.array_equal(s[n + count:], s0[n + count:])


@pytest.mark.parametrize("n,count", [(1, 1), (1, 300), (5, 2), (257, 256), (1000, 5000), (70001, 14000)])
def test_split(n, count):
    r = np.random.default_rng(n)
    check_split(n, r.integers(0, n, count))
    check_split(n, np.minimum(r.geometric(0.2, count) - 1, n - 1))


def test_split_ids_out_of_range():
    check_split(10, [3, -1, 10, 3, 9, 2 ** 31 - 1, -2 ** 31, 0])
    check_split(0, [0, -1])


def test_split_extreme_weights():
    logits = [-np.inf, np.inf, np.nan, 0.0, -800.0, 800.0, -29.9, -30.1, 40.0, 3e38, -3e38]
    check_split(11, np.tile(np.arange(11), 3), logits=logits)
    check_split(11, np.arange(5), logits=logits)


def test_split_leaves_the_field():
    """Eq. 2 with c copies of weight w / c is the same sum: phi and I agree up
    to the roundings of the shared weights and of the longer sums."""
    n = 400
    g = synth.random_gaussians(21, n, log_mu=math.log(0.08))
    r = np.random.default_rng(2)
    ids = r.integers(0, n, 300)
    rows = n + len(ids)
    p = gs.ParamSet.empty(rows, DEV)
    p.mean[:n], p.log_scale[:n], p.rot[:n] = dev(g.mean), dev(np.log(g.scale)), dev(g.rot)
    logit = lambda x: dev(np.log(x.astype(np.float64) / (1 - x)))  # noqa: E731
    p.value_logit[:n], p.weight_logit[:n] = logit(g.value), logit(g.weight)
    pts = dev(synth.random_points(5, 5000))

    def field(m):
        f = gs.Gaussians(p.mean[:m], torch.empty(m, 3, device=DEV), p.rot[:m], torch.empty(m, device=DEV),
                         torch.empty(m, device=DEV))
        gs.gs_activate(p.raw(m), 0.0, f.scale, f.value, f.weight)
        grid = gs.make_grid((8, 8, 8))
        q = gs.Query.pts(pts)
        out = torch.empty(2, 5000, device=DEV)
        index = gs.build_index(f, grid, TAU)
        gs.gs_sample(f, index, q, out[0], out[1], gs.alloc_plan(q, grid, DEV))
        return out.double().cpu().numpy()

    a = field(n)
    gs.gs_split(p, n, dev(ids, np.int32), None, gs.alloc_split_work(n, DEV))
    b = field(rows)
    # a logit of size up to 8 is rounded by 2^-24 of itself and shifts its
    # weight by that; sums of at most 700 positive terms
    rel = (8 + 2 + 2 * 700) * bo.E32
    sure = a[1] > TAU * (1 + 1e-3)
    assert sure.sum() > 4000 and (b[1][sure] > 0).all()
    assert (np.abs(a[1] - b[1])[sure] <= rel * a[1][sure]).all()
    assert (np.abs(a[0] - b[0])[sure] <= 2 * rel).all()


# ---- together -------------------------------------------------------------

def test_a_budget_round():
    """A step's shares, eviction to four fifths, draws by score, copies back to
    the full number, the moments carried along, and the next step."""
    n, keep = 3000, 2400
    g = synth.random_gaussians(31, n, log_mu=math.log(0.04))
    b = Batch(g, "jitter", (8, 8, 8), (24, 24, 24))
    score = b.shares(torch.empty(n, device=DEV))
    ref, tol = bo.shares(g, b.points, b.influence.cpu().numpy())
    assert (np.abs(score.cpu().numpy() - ref) <= tol).all()
    p, q = param_set(n, 1), gs.ParamSet.empty(n, DEV)
    source = torch.empty(n, dtype=torch.int32, device=DEV)
    kept = torch.empty(n, device=DEV)
    s0 = score.cpu().numpy()
    assert gs.gs_evict(p, n, score, keep, q, source, gs.alloc_evict_work(n, DEV), score_out=kept) == keep
    at = bo.evict(s0, keep)
    assert np.array_equal(source[:keep].cpu().numpy(), at)
    u = torch.rand(n - keep, dtype=torch.float64, device=DEV)
    ids = torch.empty(n - keep, dtype=torch.int32, device=DEV)
    gs.gs_draw(kept[:keep], u, ids, gs.alloc_draw_work(1, keep, n - keep, DEV), top_p=0.9)
    want, _, _ = bo.draw(s0[at], u.cpu().numpy(), top_p=0.9)
    assert np.array_equal(ids.cpu().numpy(), want)
    assert gs.gs_split(q, keep, ids, source, gs.alloc_split_work(keep, DEV), score=kept) == n
    total = float(kept.double().sum())
    assert abs(total - s0[at].astype(np.float64).sum()) <= 4 * bo.E32 * total
    copies = 1 + np.bincount(want, minlength=keep)
    assert np.allclose(kept[:keep].cpu().numpy(), s0[at] / copies, rtol=1e-6, atol=0)
    m = torch.arange(3 * n, dtype=torch.float32, device=DEV)
    rows = gs.AdamRows(width=3, m=m, v=m.clone(), m_out=torch.empty(3 * n, device=DEV),
                       v_out=torch.empty(3 * n, device=DEV))
    gs.gs_adamw_carry(gs.AdamCarry([rows]), n, source, n)
    moved = rows.m_out.view(n, 3).cpu().numpy()
    assert np.array_equal(moved[:keep], m.view(n, 3).cpu().numpy()[at]) and (moved[keep:] == 0).all()
    logit = bo.split_logit(p.weight_logit.cpu().numpy()[at], copies)
    assert (np.abs(q.weight_logit[:keep].cpu().numpy() - logit) <= bo.E32 * np.abs(logit) + 1e-14).all()
    f = gs.Gaussians(q.mean, torch.empty(n, 3, device=DEV), q.rot, torch.empty(n, device=DEV),
                     torch.empty(n, device=DEV))
    gs.gs_activate(q.raw(n), 0.04, f.scale, f.value, f.weight)
    index = gs.build_index(f, gs.make_grid((8, 8, 8)), TAU)
    gs.gs_sample(f, index, b.query, b.value, b.influence, b.plan)
    gs.gs_shares(f, index, b.query, b.plan, b.influence, kept, gs.alloc_shares_work(index, b.query, DEV), decay=0.5)
    assert torch.isfinite(kept).all()


@pytest.mark.parametrize("form", ["f32", "mxfp8"])
def test_training_under_a_budget(form):
    """examples/train_field.py with --rebalance-every: scores follow the
    batches, the moved Gaussians the definition, and the number stays."""
    from examples.train_field import APART, MOVED, SCORE_DECAY, TAU as TRAIN_TAU, Trainer, train
    t = Trainer(moments=gs.GS_MOMENTS_F32 if form == "f32" else gs.GS_MOMENTS_MXFP8, n=1000, dims=32)
    n = t.n
    score = np.zeros(n)
    for _ in range(3):
        t.gradients()
        got = gs.Gaussians(*(getattr(t.gauss, k).clone() for k in ("mean", "scale", "rot", "value", "weight")))
        t.attend()
        t.update()
        g = synth.Gaussians(*(getattr(got, k).cpu().numpy() for k in ("mean", "scale", "rot", "value", "weight")))
        points = voxel_positions(t.dims, np.arange(32 ** 3), t.offsets.cpu().numpy(), (0, 0, 0), (1, 1, 1))
        score, tol = bo.shares(g, points, t.influence.cpu().numpy(), None, score, SCORE_DECAY)
        seen = t.scores[t.now][:n].cpu().numpy()
        assert (np.abs(seen - score) <= tol).all()
        score = seen
    before = {k: getattr(t.sets[t.now], k)[:n].cpu().numpy() for k in ARRAYS}
    score = t.scores[t.now][:n].cpu().numpy()
    keep = n - int(MOVED * n)
    t.rebalance()
    assert t.n == n
    at = bo.evict(score, keep)
    source = t.source[:n].cpu().numpy()
    assert np.array_equal(source[:keep], at)
    ids = -1 - source[keep:]
    assert (ids >= 0).all() and (ids < keep).all()
    after = {k: getattr(t.sets[t.now], k)[:n].cpu().numpy() for k in ARRAYS}
    for k in ("mean", "log_scale", "rot", "value_logit"):
        assert np.array_equal(after[k][:keep], before[k][at])
    for k in ("log_scale", "rot", "value_logit"):
        assert np.array_equal(after[k][keep:], after[k][ids])
    far = np.abs(after["mean"][keep:] - after["mean"][ids]) / np.exp(after["log_scale"][ids])
    assert far.max() < 8 * APART and far.min() < APART
    assert np.array_equal(after["weight_logit"][keep:], after["weight_logit"][ids])
    seen = train(t, 12, 0, rebalance_every=5)
    assert seen[-1][1] == n and all(np.isfinite(x) for _, _, x in seen)
    assert TRAIN_TAU == TAU


@pytest.mark.parametrize("n_long", [3000, 40000])
def test_budget_calls_in_a_graph(n_long):
    """All four calls captured on a side stream and replayed, with eager work
    and waits between the replays, on inputs that change."""
    n, keep = 2000, 1500
    g = synth.random_gaussians(41, n, log_mu=math.log(0.05))
    batches = {k: Batch(g, seed=2, **KINDS[k]) for k in ("grid", "jitter", "points")}
    p, q = param_set(n, 3), gs.ParamSet.empty(n, DEV)
    score = {k: torch.zeros(n, device=DEV) for k in batches}
    source, kept = torch.empty(n, dtype=torch.int32, device=DEV), torch.empty(n, device=DEV)
    uniform = torch.rand(n - keep, dtype=torch.float64, device=DEV)
    ids = torch.empty(n - keep, dtype=torch.int32, device=DEV)
    long = torch.rand(2, n_long, device=DEV)
    lu = torch.rand(2, 50, dtype=torch.float64, device=DEV)
    lids, lprob = torch.empty(2, 50, dtype=torch.int32, device=DEV), torch.empty(2, 50, device=DEV)
    works = (gs.alloc_evict_work(n, DEV), gs.alloc_draw_work(1, keep, n - keep, DEV), gs.alloc_split_work(keep, DEV),
             gs.alloc_draw_work(2, n_long, 50, DEV))

    def calls(stream=None):
        for k, b in batches.items():
            b.shares(score[k], decay=0.5, stream=stream)
        gs.gs_evict(p, n, score["grid"], keep, q, source, works[0], score_out=kept, stream=stream)
        gs.gs_draw(kept[:keep], uniform, ids, works[1], top_k=700, top_p=0.8, stream=stream)
        gs.gs_split(q, keep, ids, source, works[2], score=kept, stream=stream)
        gs.gs_draw(long, lu, lids, works[3], prob=lprob, top_k=n_long // 2, top_p=0.9, min_p=0.01, stream=stream)

    outs = lambda: [x.clone() for x in (*score.values(), kept, source, ids, lids, lprob, q.mean, q.weight_logit)]  # noqa: E731
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls()
    for turn in range(4):
        uniform.copy_(torch.rand_like(uniform))
        long.copy_(torch.rand_like(long))
        lu.copy_(torch.rand_like(lu))
        start = {k: torch.rand(n, device=DEV) for k in score}
        for k in score:
            score[k].copy_(start[k])
        calls()
        want = outs()
        for x in (kept, source, ids, lids, lprob, q.mean, q.weight_logit):
            x.fill_(1)
        for k in score:
            score[k].copy_(start[k])
        torch.cuda.synchronize()
        graph.replay()
        got = outs()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), turn
        if turn == 1:
            torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for k in score:
            score[k].copy_(start[k])
    calls(stream=side)  # named, not current
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs()))


def test_large_budget_calls_in_a_graph():
    """The same with sets, rows and Gaussians that take several launches."""
    n, keep = 40000, 30000
    g = synth.random_gaussians(43, n, log_mu=math.log(0.01))
    g.scale[11] = (0.5, 0.4, 0.6)
    batches = {"points": Batch(g, "points", (16, 16, 16), n=70001, seed=1),
               "jitter": Batch(g, "jitter", (16, 16, 16), (42, 43, 44), seed=2),
               "grid": Batch(g, "grid", (16, 16, 16), (48, 48, 48), seed=3)}
    p, q = param_set(n, 3), gs.ParamSet.empty(n, DEV)
    score = {k: torch.zeros(n, device=DEV) for k in batches}
    source, kept = torch.empty(n, dtype=torch.int32, device=DEV), torch.empty(n, device=DEV)
    pinned = torch.zeros(n, dtype=torch.uint8, device=DEV)
    pinned[::37] = 1
    uniform = torch.rand(n - keep, dtype=torch.float64, device=DEV)
    ids, few = (torch.empty(n - keep, dtype=torch.int32, device=DEV) for _ in range(2))
    best = torch.empty(1, dtype=torch.int32, device=DEV)
    works = (gs.alloc_evict_work(n, DEV), gs.alloc_draw_work(1, keep, n - keep, DEV), gs.alloc_split_work(keep, DEV))

    def calls():
        for k, b in batches.items():
            b.shares(score[k], decay=0.5)
        gs.gs_evict(p, n, score["points"], keep, q, source, works[0], pinned=pinned, score_out=kept)
        gs.gs_draw(kept[:keep], uniform, ids, works[1], top_k=20000, top_p=0.8)
        gs.gs_draw(kept[:keep], uniform, few, works[1], top_k=100, top_p=0.8, temperature=0.5)
        gs.gs_draw(kept[:keep], uniform[:1], best, works[1], temperature=0.0)
        gs.gs_split(q, keep, ids, source, works[2], score=kept)

    outs = lambda: [x.clone() for x in (*score.values(), kept, source, ids, few, best, q.mean, q.weight_logit)]  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for turn in range(4):
        uniform.copy_(torch.rand_like(uniform))
        start = {k: torch.rand(n, device=DEV) for k in score}
        for k in score:
            score[k].copy_(start[k])
        calls()
        want = outs()
        for x in (kept, source, ids, few, best, q.mean, q.weight_logit):
            x.fill_(1)
        for k in score:
            score[k].copy_(start[k])
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, outs())), turn
        if turn == 1:
            torch.cuda.synchronize()
