"""Holding a field to a budget of Gaussians: what is timed and checked of it,
in plain torch and through the framework's entry points.

A field is Phi(p) = sum a_i v_i / sum a_i with a_i = w_i G_i(p): attention of
the query p over the Gaussians, with weights a_i / I. A case is a dict of
plain values:

* op "shares"  the attention weight that every Gaussian gets from a batch of
               queries, gain_t a_i / I_t summed over the queries, added to a
               decaying score;
     "evict"   a set cut down to the `keep` Gaussians of the largest score,
               `pinned` of them protected, in their order, with the source
               map that the optimiser's moments follow;
     "draw"    `draws` of n candidates a row, with replacement, by given
               uniform numbers: temperature, top-k, top-p, min-p;
     "split"   copies of drawn Gaussians, the weight shared between a
               Gaussian and its copies, so that the field stays the same.

Everything is float32 but the uniform numbers (float64: a row may have more
candidates than float32 has steps) and, where a case says so, bfloat16
scores.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TAU = 0.01
CUT = 2.0 * math.log(1.0 / float(np.float32(TAU)))  # Q <= CUT: within the cutoff
DECAY = 0.9


# ---- cases ---------------------------------------------------------------

def _shares(n_gauss, query, dims, n, cells, log_sd, crowd, gain, name=None):
    c = {"op": "shares", "n_gauss": n_gauss, "query": query, "dx": dims[0], "dy": dims[1], "dz": dims[2],
         "n": n if query == "points" else dims[0] * dims[1] * dims[2], "cx": cells[0], "cy": cells[1], "cz": cells[2],
         "log_sd": log_sd, "crowd": crowd, "gain": gain}
    return dict(c, name=name) if name else c


def _evict(n, keep, pinned, zeros, name=None):
    c = {"op": "evict", "n": n, "keep": keep, "pinned": pinned, "zeros": zeros}
    return dict(c, name=name) if name else c


def _draw(rows, n, draws, scores, ragged=False, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, name=None):
    c = {"op": "draw", "rows": rows, "n": n, "draws": draws, "scores": scores, "ragged": ragged,
         "temperature": temperature, "top_k": top_k, "top_p": top_p, "min_p": min_p}
    return dict(c, name=name) if name else c


def _split(n, count, name=None):
    c = {"op": "split", "n": n, "count": count}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest field the framework is run with, on all voxels of a
        # coarse volume: launches count
        _shares(4096, "grid", (32, 32, 32), 0, (8, 8, 8), 0.3, 0, False, "shares_grid32"),
        # a ragged batch of a mildly clustered cloud of points, each with the
        # error of its sample as the gain
        _shares(50021, "points", (0, 0, 0), 100003, (37, 29, 23), 0.6, 24, True, "shares_ragged_points"),
        # the structured training step: a random position in every voxel
        _shares(131072, "jitter", (128, 128, 128), 0, (32, 32, 32), 0.4, 0, False, "shares_jitter128"),
        # a small field cut by a fifth; a trained one with its newest
        # Gaussians protected; the largest halved, three fifths of its
        # Gaussians never seen by a query (their scores are 0: ties)
        _evict(4096, 3277, 0, 0.0, "evict_4k"),
        _evict(262144, 209715, 26214, 0.05, "evict_262k_pinned"),
        _evict(2097152, 1048576, 0, 0.6, "evict_2m_ties"),
        # the Gaussians of a small field to copy, by weight
        _draw(1, 4096, 819, "weight", name="draw_4k"),
        # voxels to train on next, some in every brick of 8^3 of a 128^3
        # volume, by the error of their last samples, sharpened; border
        # bricks hold fewer
        _draw(4096, 512, 16, "error", True, 0.7, 0, 0.95, 0.0, name="draw_bricks"),
        # one candidate a row out of its best, logits in bfloat16: the
        # common form with all filters
        _draw(64, 50021, 1, "logit16", False, 0.8, 200, 0.9, 0.02, name="draw_logits"),
        # a fifth of the largest field's Gaussians, by accumulated score
        _draw(1, 2097152, 419430, "weight", False, 1.0, 0, 0.999, 0.0, name="draw_2m"),
        # copies of a fifth
        _split(4096, 819, "split_4k"),
        _split(2097152, 419430, "split_2m"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("shares", "shares", "evict", "draw", "draw", "draw", "split"))
    if op == "shares":
        n_gauss = _log(rng, 1009, 131072)
        cells = [max(2, int(n_gauss ** (1.0 / 3.0) * rng.uniform(0.5, 1.0))) for _ in range(3)]
        gain = rng.random() < 0.5
        query = rng.choice(("grid", "jitter", "points"))
        if query == "grid":  # a whole number of voxels in every cell
            dims = [c * rng.choice((1, 2, 3)) for c in cells]
            while dims[0] * dims[1] * dims[2] > 2000000:
                dims = [max(c, d - c) for c, d in zip(cells, dims)]
            return _shares(n_gauss, query, dims, 0, cells, round(rng.uniform(0.2, 0.5), 3), 0, gain)
        if query == "jitter":
            side = _log(rng, 17, 120)
            return _shares(n_gauss, query, (side, side + rng.randrange(6), max(5, side - rng.randrange(6))), 0, cells,
                           round(rng.uniform(0.2, 0.5), 3), 0, gain)
        crowd = rng.choice((0, 24, 64))
        n_gauss = min(n_gauss, 50021)
        return _shares(n_gauss, query, (0, 0, 0), _log(rng, 101, 100003 if crowd else 600011), cells,
                       round(rng.uniform(0.2, 0.6), 3), crowd, gain)
    if op == "evict":
        n = _log(rng, 1000, 2000000)
        keep = max(1, int(n * rng.uniform(0.05, 0.95)))
        return _evict(n, keep, int(keep * rng.choice((0.0, 0.1, 0.5))), round(rng.choice((0.0, rng.uniform(0, 0.7))), 3))
    if op == "split":
        n = _log(rng, 1000, 2000000)
        return _split(n, max(1, int(n * rng.uniform(0.01, 0.2))))
    n = _log(rng, 33, 2000000)
    rows = _log(rng, 1, max(1, 2000000 // n))
    draws = _log(rng, 1, max(1, min(400000 // rows, n)))
    filters = [(0, 1.0, 0.0), (_log(rng, 1, n), 1.0, 0.0), (0, round(rng.uniform(0.3, 0.999), 3), 0.0),
               (0, 1.0, round(rng.uniform(0.001, 0.3), 3)),
               (_log(rng, 1, n), round(rng.uniform(0.3, 0.999), 3), round(rng.uniform(0.0, 0.1), 3))]
    k, p, m = rng.choice(filters)
    return _draw(rows, n, draws, rng.choice(("weight", "error", "logit", "logit16")), rng.random() < 0.4,
                 rng.choice((1.0, 1.0, round(rng.uniform(0.3, 2.0), 3))), k, p, m)


def _median(case):
    """Median standard deviation of a field in the unit cube: 0.45 of the
    mean distance between Gaussians."""
    return 0.45 * case["n_gauss"] ** (-1.0 / 3.0)


def work(case):
    op = case["op"]
    if op == "shares":
        # pairs within the cutoff, for Gaussians and queries spread evenly
        volume = 4.0 / 3.0 * math.pi * CUT ** 1.5 * _median(case) ** 3 * math.exp(1.5 * case["log_sd"] ** 2)
        pairs = case["n_gauss"] * case["n"] * volume
        gather = 0 if case["query"] == "grid" else 12
        return {"bytes": case["n"] * (4 + gather + 4 * case["gain"]) + case["n_gauss"] * (44 + 4 + 4),
                "flops": 26 * pairs}
    if op == "evict":
        return {"bytes": case["n"] * (4 + (1 if case["pinned"] else 0)) + case["keep"] * (48 + 48 + 4 + 4),
                "flops": 0}
    if op == "split":
        return {"bytes": case["count"] * (4 + 48 + 4 + 48 + 4 + 4), "flops": 30 * case["count"]}
    size = 2 if case["scores"] == "logit16" else 4
    return {"bytes": case["rows"] * (case["n"] * size + case["draws"] * (8 + 4 + 4)),
            "flops": 20 * case["rows"] * case["n"]}


# ---- inputs --------------------------------------------------------------

def _gen(seed, stream):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + 7919 * stream + 29) % (1 << 62))


def _cloud(count, crowd, centre, gen):
    """Positions in the unit cube: even, or around `crowd` centres with a
    fifth of background."""
    x = torch.rand(count, 3, generator=gen, device=DEV)
    if not crowd:
        return x
    at = torch.randint(0, crowd, (count,), generator=gen, device=DEV)
    near = (centre[at] + 0.06 * torch.randn(count, 3, generator=gen, device=DEV)).clamp(0.0, 1.0)
    return torch.where(torch.rand(count, 1, generator=gen, device=DEV) < 0.2, x, near).contiguous()


def _params(rows, gen):
    """Free parameters of a trained set: mean, log-scale, quaternion, value
    logit, weight logit."""
    f = dict(generator=gen, device=DEV)
    return {"mean": torch.rand(rows, 3, **f), "log_scale": -4.0 + 0.5 * torch.randn(rows, 3, **f),
            "rot": torch.randn(rows, 4, **f), "value_logit": torch.randn(rows, **f),
            "weight_logit": -2.0 + 2.0 * torch.randn(rows, **f)}


def _cells(case):
    return case["cx"], case["cy"], case["cz"]


def prepare(case, seed):
    gen = _gen(seed, 1)
    if case["op"] == "shares":
        return _prepare_shares(case, seed, gen)
    st = {"case": dict(case)}
    if case["op"] == "evict":
        n = case["n"]
        st["params"] = _params(n, gen)
        # accumulated scores spread over many powers of ten; what no query
        # reached has none
        score = torch.exp(2.5 * torch.randn(n, generator=gen, device=DEV))
        st["score"] = torch.where(torch.rand(n, generator=gen, device=DEV) < case["zeros"], 0.0, score)
        st["pinned"] = None
        if case["pinned"]:  # the last added stand at the end
            st["pinned"] = torch.zeros(n, dtype=torch.uint8, device=DEV)
            st["pinned"][n - case["pinned"]:] = 1
        if own:
            import paper_2607_01164_amd as gs
            st["in"] = gs.ParamSet(**st["params"])
            st["out"] = gs.ParamSet.empty(case["keep"], DEV)
            st["source"] = torch.empty(case["keep"], dtype=torch.int32, device=DEV)
            st["score_out"] = torch.empty(case["keep"], dtype=torch.float32, device=DEV)
            st["work"] = gs.alloc_evict_work(n, DEV)
    elif case["op"] == "split":
        n, count = case["n"], case["count"]
        st["params"] = _params(n + count, gen)
        weight = torch.sigmoid(st["params"]["weight_logit"][:n].double())
        share = weight.cumsum(0)
        u = torch.rand(count, dtype=torch.float64, generator=gen, device=DEV) * share[-1]
        st["ids"] = torch.searchsorted(share, u).clamp_max(n - 1).to(torch.int32)
        st["score"] = torch.exp(torch.randn(n + count, generator=gen, device=DEV))
        st["source"] = torch.zeros(n + count, dtype=torch.int32, device=DEV)
        if own:
            import paper_2607_01164_amd as gs
            st["set"] = gs.ParamSet(**st["params"])
            st["work"] = gs.alloc_split_work(n, DEV)
    else:
        rows, n = case["rows"], case["n"]
        noise = torch.randn(rows, n, generator=gen, device=DEV)
        st["scores"] = {"weight": lambda: torch.sigmoid(2.0 * noise - 2.0), "error": lambda: 0.1 * noise.abs() ** 3,
                        "logit": lambda: 2.5 * noise,
                        "logit16": lambda: (2.5 * noise).to(torch.bfloat16)}[case["scores"]]()
        del noise
        st["lengths"] = None
        if case["ragged"]:
            st["lengths"] = torch.randint(n // 2, n + 1, (rows,), generator=gen, device=DEV, dtype=torch.int32)
        st["uniform"] = torch.rand(rows, case["draws"], dtype=torch.float64, generator=gen, device=DEV)
        if own:
            import paper_2607_01164_amd as gs
            st["ids"] = torch.empty(rows, case["draws"], dtype=torch.int32, device=DEV)
            st["prob"] = torch.empty(rows, case["draws"], dtype=torch.float32, device=DEV)
            st["work"] = gs.alloc_draw_work(rows, n, case["draws"], DEV)
    return st


def _prepare_shares(case, seed, gen):
    n_gauss, n = case["n_gauss"], case["n"]
    f = dict(generator=gen, device=DEV)
    centre = 0.1 + 0.8 * torch.rand(max(1, case["crowd"]), 3, **f)
    rot = torch.randn(n_gauss, 4, **f)
    st = {"case": dict(case), "mean": _cloud(n_gauss, case["crowd"], centre, gen),
          "scale": torch.exp(math.log(_median(case)) + case["log_sd"] * torch.randn(n_gauss, 3, **f)),
          "rot": rot / rot.norm(dim=1, keepdim=True),
          "value": torch.rand(n_gauss, **f), "weight": torch.sigmoid(torch.randn(n_gauss, **f) - 1.0)}
    if case["query"] == "points":
        st["points"] = _cloud(n, case["crowd"], centre, gen)
    elif case["query"] == "jitter":
        st["points"] = torch.rand(n, 3, **f)
    st["gain"] = 0.1 * torch.randn(n, **f).abs() if case["gain"] else None
    st["score"] = 5.0 * torch.rand(n_gauss, **f)
    # what the sampler's forward hands on: I, and 0 where the field is undefined
    total = torch.zeros(n, dtype=torch.float64, device=DEV)
    g, t, a = _pairs(st)
    total.index_add_(0, t, a.double())
    del g, t, a
    st["influence"] = torch.where(total > TAU, total, 0.0).float()
    if own:
        import paper_2607_01164_amd as gs
        st["gauss"] = gs.Gaussians(st["mean"], st["scale"], st["rot"], st["value"], st["weight"])
        grid = gs.make_grid(_cells(case))
        st["index"] = gs.build_index(st["gauss"], grid, TAU)
        dims = (case["dx"], case["dy"], case["dz"])
        st["queries"] = {"grid": lambda: gs.Query.grid(dims), "points": lambda: gs.Query.pts(st["points"]),
                         "jitter": lambda: gs.Query.jitter(dims, st["points"])}[case["query"]]()
        st["plan"] = None
        if case["query"] != "grid":  # the plan that the forward filled
            out = [torch.empty(n, dtype=torch.float32, device=DEV) for _ in range(2)]
            st["plan"] = gs.alloc_plan(st["queries"], grid, DEV)
            gs.gs_sample(st["gauss"], st["index"], st["queries"], out[0], out[1], st["plan"])
        st["work"] = gs.alloc_shares_work(st["index"], st["queries"], DEV)
    return st


# ---- the operators -------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return _own(state, op)
    return {"shares": _plain_shares, "evict": _plain_evict, "draw": _plain_draw, "split": _plain_split}[op](state)


def _own(state, op):
    import paper_2607_01164_amd as gs
    case = state["case"]
    if op == "shares":
        gs.gs_shares(state["gauss"], state["index"], state["queries"], state["plan"], state["influence"],
                     state["score"], state["work"], gain=state["gain"], decay=DECAY)
        return state["score"]
    if op == "evict":
        gs.gs_evict(state["in"], case["n"], state["score"], case["keep"], state["out"], state["source"],
                    state["work"], pinned=state["pinned"], score_out=state["score_out"])
        out = state["out"]
        return {"mean": out.mean, "log_scale": out.log_scale, "rot": out.rot, "value_logit": out.value_logit,
                "weight_logit": out.weight_logit, "source": state["source"], "score": state["score_out"]}
    if op == "split":
        gs.gs_split(state["set"], case["n"], state["ids"], state["source"], state["work"], score=state["score"])
        return {**state["params"], "source": state["source"], "score": state["score"]}
    gs.gs_draw(state["scores"], state["uniform"], state["ids"], state["work"], prob=state["prob"],
               logits=case["scores"].startswith("logit"), lengths=state["lengths"], temperature=case["temperature"],
               top_k=case["top_k"], top_p=case["top_p"], min_p=case["min_p"])
    return {"ids": state["ids"], "prob": state["prob"]}


# ---- the plain form ------------------------------------------------------

def _voxels(case):
    """x, y, z of every voxel, x fastest."""
    dx, dy, dz = case["dx"], case["dy"], case["dz"]
    i = torch.arange(case["n"], device=DEV)
    return torch.stack([i % dx, i // dx % dy, i // (dx * dy)], 1).float(), torch.tensor([dx, dy, dz], device=DEV)


def _positions(st):
    case = st["case"]
    if case["query"] == "points":
        return st["points"]
    voxel, dims = _voxels(case)
    at = voxel + (0.5 if case["query"] == "grid" else st["points"])
    return at * (1.0 / dims.float())


def _factors(st):
    """S^-1 R^T of every Gaussian, as rows, and the half-extents of its
    cutoff ellipsoid along the axes, in 64 bits."""
    q = st["rot"].double()
    w, x, y, z = (q / q.norm(dim=1, keepdim=True)).unbind(1)
    rt = torch.stack([1 - 2 * (y * y + z * z), 2 * (x * y + w * z), 2 * (x * z - w * y),
                      2 * (x * y - w * z), 1 - 2 * (x * x + z * z), 2 * (y * z + w * x),
                      2 * (x * z + w * y), 2 * (y * z - w * x), 1 - 2 * (x * x + y * y)], 1).view(-1, 3, 3)
    s = st["scale"].double()
    half = math.sqrt(CUT) * (rt * s[:, :, None]).square().sum(1).sqrt()
    return rt / s[:, :, None], half


def _spread(count):
    """The places of `count` elements each laid end to end: owner and rank."""
    owner = torch.repeat_interleave(torch.arange(len(count), device=DEV), count)
    first = count.cumsum(0) - count
    return owner, torch.arange(len(owner), device=DEV) - first[owner]


def _pairs(st):
    """Gaussian, query and a = w G of every pair within the cutoff. The
    queries are put in order by cell, and every row of cells that a
    Gaussian's box meets is a run of them. Which pairs are within the cutoff
    is decided in 64 bits."""
    cx, cy, cz = _cells(st["case"])
    cells = torch.tensor([cx, cy, cz], device=DEV)
    p = _positions(st)
    c = (p.double() * cells).long().clamp_min(0).minimum(cells - 1)
    order = torch.argsort(c[:, 0] + cx * (c[:, 1] + cy * c[:, 2]))
    start = torch.zeros(cx * cy * cz + 1, dtype=torch.long, device=DEV)
    start[1:] = torch.bincount(c[:, 0] + cx * (c[:, 1] + cy * c[:, 2]), minlength=cx * cy * cz).cumsum(0)
    m, half = _factors(st)
    mean = st["mean"].double()
    low = ((mean - half * 1.000001) * cells).floor().long().clamp_min(0).minimum(cells - 1)
    high = ((mean + half * 1.000001) * cells).floor().long().clamp_min(0).minimum(cells - 1)
    span = high - low + 1
    g, rank = _spread(span[:, 1] * span[:, 2])
    row = cx * (low[g, 1] + rank % span[g, 1] + cy * (low[g, 2] + rank // span[g, 1]))
    begin = start[row + low[g, 0]]
    r, rank = _spread(start[row + high[g, 0] + 1] - begin)
    g, t = g[r], order[begin[r] + rank]
    del r, rank, begin, row
    d = p[t].double() - mean[g]
    u = torch.stack([m[g, k, 0] * d[:, 0] + m[g, k, 1] * d[:, 1] + m[g, k, 2] * d[:, 2] for k in range(3)], 1)
    del d
    q = u.square().sum(1)
    within = q <= CUT
    g, t = g[within], t[within]
    return g, t, st["weight"][g] * torch.exp(-0.5 * q[within]).float()


def _plain_shares(st):
    g, t, a = _pairs(st)
    f = torch.where(st["influence"] > 0, 1.0 / st["influence"], 0.0)
    if st["gain"] is not None:
        f = f * st["gain"]
    new = torch.zeros(st["case"]["n_gauss"], dtype=torch.float64, device=DEV)
    new.index_add_(0, g, (a * f[t]).double())
    st["score"].copy_(DECAY * st["score"].double() + new)
    return st["score"]


def _plain_evict(st):
    score = st["score"]
    if st["pinned"] is not None:  # protected ones go before all others
        by = torch.argsort(score, descending=True, stable=True)
        by = by[torch.argsort(st["pinned"][by], descending=True, stable=True)]
    else:
        by = torch.argsort(score, descending=True, stable=True)
    source = by[:st["case"]["keep"]].sort().values
    out = {k: x[source] for k, x in st["params"].items()}
    return {**out, "source": source.to(torch.int32), "score": score[source]}


def _bits(n):
    """2^_bits: the mass of a row's best candidate."""
    return min(52, 62 - (n - 1).bit_length())


def _scaled(m, total):
    """floor(m total / 2^53) for m <= 2^53, total < 2^62, without leaving 64 bits."""
    mh, ml, th, tl = m >> 22, m & 0x3FFFFF, total >> 31, total & 0x7FFFFFFF
    return mh * th + ((mh * tl + ((ml * th) << 9) + ((ml * tl) >> 22)) >> 31)


def _plain_draw(st):
    case = st["case"]
    n, t = case["n"], case["temperature"]
    x = st["scores"].double()
    if st["lengths"] is not None:
        out = torch.arange(n, device=DEV) >= st["lengths"][:, None]
        x = torch.where(out, -math.inf if case["scores"].startswith("logit") else 0.0, x)
    top = x.amax(1, keepdim=True)
    if case["scores"].startswith("logit"):
        e = torch.exp((x - top) / t)
    else:
        e = x / top if t == 1.0 else torch.exp(torch.log(x / top) / t)
    mass = torch.round(e * 2.0 ** _bits(n)).long()
    del e
    if case["top_k"] or case["top_p"] < 1.0:
        by = torch.argsort(x, dim=1, descending=True, stable=True)
        ranked = mass.gather(1, by)
        if case["top_k"]:
            ranked[:, case["top_k"]:] = 0
        if case["top_p"] < 1.0:
            sums = ranked.cumsum(1)
            share = torch.tensor(int(case["top_p"] * 2.0 ** 53), device=DEV)
            # kept while those before it have at most top_p of the mass
            ranked = torch.where(sums - ranked <= _scaled(share, sums[:, -1:]), ranked, 0)
        mass = torch.zeros_like(mass).scatter_(1, by, ranked)
        del by, ranked
    if case["min_p"]:
        mass = torch.where(mass.double() >= case["min_p"] * 2.0 ** _bits(n), mass, 0)
    sums = mass.cumsum(1)
    total = sums[:, -1:]
    u = (st["uniform"].clamp(0.0, 1.0 - 2.0 ** -53) * 2.0 ** 53).long()
    ids = torch.searchsorted(sums, _scaled(u, total), right=True)
    prob = mass.gather(1, ids).double() / total.double()
    return {"ids": ids.to(torch.int32), "prob": prob.float()}


def _plain_split(st):
    n, ids = st["case"]["n"], st["ids"].long()
    copies = 1 + torch.bincount(ids, minlength=n)
    p = st["params"]
    for k in ("mean", "log_scale", "rot", "value_logit"):
        p[k][n:] = p[k][ids]
    logit, c = p["weight_logit"][:n].double(), copies.double()
    shared = torch.where(copies == 1, logit, -torch.log((c - 1) + c * torch.exp(-logit)))
    shared = torch.where(logit < -30.0, logit - torch.log(c), shared).float()
    p["weight_logit"][:n] = shared
    p["weight_logit"][n:] = shared[ids]
    score = st["score"][:n] / copies
    st["score"][:n] = score
    st["score"][n:] = score[ids]
    st["source"][n:] = (-1 - ids).to(torch.int32)
    return {**p, "source": st["source"], "score": st["score"]}


# ---- the definitions in 64 bits ------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"shares": _exact_shares, "evict": _exact_evict, "draw": _exact_draw, "split": _exact_split}[case["op"]](st)


def _exact_shares(st):
    """Blocks of the unit cube one after the other: all queries of a block
    with all Gaussians whose box meets it, through the inverse covariance's
    square root."""
    case = st["case"]
    p, mean = _positions(st).double(), st["mean"].double()
    q = st["rot"].double()
    q = q / q.square().sum(1, keepdim=True).sqrt()
    r, v = q[:, :1], q[:, 1:]
    scale = st["scale"].double()

    def unturned(d, i):  # R^T d: the inverse rotation of the vector d
        c = torch.linalg.cross(v[i][None].expand_as(d), d, dim=2)
        return d - 2 * r[i] * c + 2 * torch.linalg.cross(v[i][None].expand_as(d), c, dim=2)

    reach = math.sqrt(CUT) * scale.amax(1, keepdim=True)
    share = torch.where(st["influence"] > 0, 1.0 / st["influence"].double(), 0.0)
    if st["gain"] is not None:
        share = share * st["gain"].double()
    side = 8 if case["n"] > 4096 else 2
    block = (p * side).long().clamp(0, side - 1)
    block = block[:, 0] + side * (block[:, 1] + side * block[:, 2])
    score = DECAY * st["score"].double()
    for b in torch.unique(block).tolist():
        t = torch.nonzero(block == b).view(-1)
        lo, hi = p[t].amin(0), p[t].amax(0)
        i = torch.nonzero(((mean + reach >= lo) & (mean - reach <= hi)).all(1)).view(-1)
        for part in torch.split(t, max(1, 20000000 // max(1, len(i)))):
            u = unturned(p[part][:, None, :] - mean[i], i) / scale[i]
            square = (u * u).sum(2)
            g = torch.where(square <= CUT, torch.exp(-square / 2), 0.0)
            score[i] += st["weight"][i].double() * (g * share[part][:, None]).sum(0)
    return score


def _exact_evict(st):
    score = st["score"].cpu().numpy()
    pinned = np.zeros(len(score)) if st["pinned"] is None else st["pinned"].cpu().numpy()
    by = np.lexsort((np.arange(len(score)), -score, -pinned.astype(np.int64)))
    source = np.sort(by[:st["case"]["keep"]])
    at = torch.from_numpy(source).to(DEV)
    return {**{k: x.double()[at] for k, x in st["params"].items()}, "source": at.to(torch.int32),
            "score": st["score"].double()[at]}


def _exact_draw(st):
    """Row by row on the host, with integers of any size."""
    case = st["case"]
    x = st["scores"].double().cpu().numpy()
    u = st["uniform"].cpu().numpy()
    lengths = None if st["lengths"] is None else st["lengths"].cpu().numpy()
    if x.size > 6000000 or case["rows"] > 6000:
        return None
    ids, prob = np.zeros(u.shape, np.int32), np.zeros(u.shape)
    unit = 1 << _bits(case["n"])
    for r in range(case["rows"]):
        w = x[r] if lengths is None else x[r][:lengths[r]]
        if case["scores"].startswith("logit"):
            e = np.exp((w - w.max()) / case["temperature"])
        elif case["temperature"] == 1.0:
            e = w / w.max()
        else:
            with np.errstate(divide="ignore"):
                e = np.exp(np.log(w / w.max()) / case["temperature"])
        mass = np.rint(e * unit).astype(np.int64)
        by = np.argsort(-w, kind="stable")
        kept = mass[by]
        if case["top_k"]:
            kept = kept[:case["top_k"]]
        if case["top_p"] < 1.0:
            sums = np.cumsum(kept)
            most = int(case["top_p"] * 2.0 ** 53) * int(sums[-1]) >> 53
            kept = kept[:int(np.searchsorted(sums - kept, most, side="right"))]
        kept = kept * (kept >= case["min_p"] * unit)
        final = np.zeros_like(mass)
        final[by[:len(kept)]] = kept
        sums = np.cumsum(final)
        total = int(sums[-1])
        at = np.array([int(float(y) * 2.0 ** 53) * total >> 53 for y in u[r]], dtype=np.int64)
        ids[r] = np.searchsorted(sums, at, side="right")
        prob[r] = final[ids[r]] / total
    return {"ids": torch.from_numpy(ids), "prob": torch.from_numpy(prob)}


def _exact_split(st):
    n, ids = st["case"]["n"], st["ids"].long()
    p = {k: x.double() for k, x in st["params"].items()}
    times = torch.zeros(n, dtype=torch.float64, device=DEV)
    times.index_add_(0, ids, torch.ones(len(ids), dtype=torch.float64, device=DEV))
    # w / c through the odds: logit(w / c) = ln w - ln(c - w), w = 1 / (1 + e^-l)
    l, c = p["weight_logit"][:n], times + 1
    ln_w = -torch.nn.functional.softplus(-l)
    rest = times + torch.exp(-torch.nn.functional.softplus(l))  # c - w = (c - 1) + (1 - w)
    l = torch.where(times > 0, ln_w - torch.log(rest), l)
    s = st["score"][:n].double() / c
    out = {k: torch.cat([p[k][:n], p[k][ids]]) for k in ("mean", "log_scale", "rot", "value_logit")}
    source = torch.cat([st["source"][:n].long(), -1 - ids]).to(torch.int32)
    return {**out, "weight_logit": torch.cat([l, l[ids]]), "source": source, "score": torch.cat([s, s[ids]])}
