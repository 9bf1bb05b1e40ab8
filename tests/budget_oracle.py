"""The operators of include/gs_budget.h in float64 and whole numbers of any
size (numpy), written from their definitions, with the bounds that float32
allows."""
import math

import numpy as np

E32 = 2.0 ** -24  # half a step of float32, relative
EXP_ULP = 2.0 ** -23  # v_exp_f32: one unit in the last place


def cut(tau):
    return 2.0 * math.log(1.0 / float(np.float32(tau)))


def whitened(g, i, points):
    """S^-1 R^T (p - mu) of Gaussian i at float32 positions, in float64."""
    q = g.rot[i].astype(np.float64)
    w, x, y, z = q / np.sqrt((q * q).sum())
    r = np.array([[1 - 2 * (y * y + z * z), 2 * (x * y - w * z), 2 * (x * z + w * y)],
                  [2 * (x * y + w * z), 1 - 2 * (x * x + z * z), 2 * (y * z - w * x)],
                  [2 * (x * z - w * y), 2 * (y * z + w * x), 1 - 2 * (x * x + y * y)]])
    return (points.astype(np.float64) - g.mean[i].astype(np.float64)) @ r / g.scale[i].astype(np.float64)


def valid(g, i):
    fine = all(np.isfinite(a[i]).all() for a in (g.mean, g.scale, g.rot, g.value, g.weight))
    n2 = float((g.rot[i].astype(np.float32) ** 2).sum())
    return fine and (g.scale[i] > 0).all() and n2 > 0


def shares(g, points, influence, gain=None, score=None, decay=0.0, tau=0.01, lo=(0, 0, 0), hi=(1, 1, 1)):
    """(scores, how far float32 may be off). Per pair: f is rounded once, Q' is
    off by at most (5 sqrt(3) 2 + 3) kappa 2^-24 of itself (the entries of U and
    d are rounded once, u's sums three times) and shifts G by ln 2 times that,
    the exponential by a unit, a product by half a step; K terms are added with
    at most K roundings; the weight and the decay take three more."""
    inside = ((points >= np.array(lo, np.float32)) & (points <= np.array(hi, np.float32))).all(1)
    f = np.zeros(len(points))
    on = inside & (influence > 0)
    f[on] = (1.0 if gain is None else gain.astype(np.float64)[on]) / influence.astype(np.float64)[on]
    out, tol = np.zeros(len(g.mean)), np.zeros(len(g.mean))
    top = cut(tau) / (2 * math.log(2))  # the largest Q'
    for i in range(len(g.mean)):
        a = size = 0.0
        if valid(g, i):
            q = (whitened(g, i, points) ** 2).sum(1)
            near = q <= cut(tau)
            t = float(g.weight[i]) * np.exp(-0.5 * q[near]) * f[near]
            a, size = t.sum(), np.abs(t).sum()
            kappa = float(g.scale[i].max() / g.scale[i].min())
            rel = math.log(2) * (10 * math.sqrt(3) + 3) * kappa * E32 * top + EXP_ULP + (near.sum() + 6) * E32
            tol[i] = size * rel
        before = decay * float(score[i]) if decay else 0.0
        out[i] = before + a
        tol[i] += 2 * E32 * (abs(before) + size) + 1e-37
    return out, tol


def evict(score, budget, pinned=None):
    """Indices kept."""
    n = len(score)
    pin = np.zeros(n, np.int64) if pinned is None else (pinned != 0).astype(np.int64)
    s = score.astype(np.float64)
    nan = np.isnan(s)
    s = np.where(nan, -np.inf, s)
    by = np.lexsort((np.arange(n), nan, -s, -pin))
    return np.sort(by[:min(budget, n)])


def bits_of(n):
    return min(52, 62 - (n - 1).bit_length() if n > 0 else 52)


def masses(x, n, temperature, logits):
    """q of a row's candidates; n: the candidates that a row has room for."""
    x = x.astype(np.float64)
    live = x > (-np.inf if logits else 0)
    q = np.zeros(len(x), np.int64)
    if not live.any():
        return q
    unit = 1 << bits_of(n)
    top = x[live].max()
    if temperature == 0:
        q[np.flatnonzero(live & (x == top))[0]] = unit
        return q
    if np.isinf(top):
        q[live & (x == top)] = unit
        return q
    v = x[live]
    with np.errstate(over="ignore"):
        if logits:
            e = np.exp((v - top) / temperature)
        else:
            e = v / top if temperature == 1 else np.exp(np.log(v / top) / temperature)
    q[live] = np.rint(e * unit).astype(np.int64)
    return q


def kept(x, n, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, logits=False):
    """The masses that the filters leave of a row."""
    q = masses(x, n, temperature, logits)
    order = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    if not logits:
        order = np.where(order > 0, order, 0)
    by = np.lexsort((np.arange(len(x)), -order))
    stay = by
    if temperature > 0:
        if top_k:
            stay = stay[:top_k]
        if top_p < 1:
            most = int(top_p * 2.0 ** 53) * sum(int(v) for v in q[stay]) >> 53
            before, n_stay = 0, 0
            for j in stay:
                if before > most:
                    break
                before += int(q[j])
                n_stay += 1
            stay = stay[:n_stay]
    out = np.zeros_like(q)
    out[stay] = q[stay]
    out[out.astype(np.float64) < min_p * float(1 << bits_of(n))] = 0
    return out


def draw(x, u, n=None, **settings):
    """(ids, probabilities, room): room, the share of the mass between each
    draw and the nearest border between two candidates."""
    n = len(x) if n is None else n
    q = kept(x, n, **settings)
    run = np.cumsum(q)
    total = int(run[-1]) if len(run) else 0
    if total == 0:
        return np.full(len(u), -1, np.int32), np.zeros(len(u)), np.ones(len(u))
    u = np.where(np.isnan(u), 0, u)
    m = [min(max(int(min(max(v, 0.0), 1.0) * 2.0 ** 53), 0), (1 << 53) - 1) for v in u]
    r = np.array([v * total >> 53 for v in m], dtype=np.int64)
    ids = np.searchsorted(run, r, side="right")
    low = np.where(ids > 0, run[np.maximum(ids - 1, 0)], 0)
    room = np.minimum(r - low + 1, run[ids] - r)
    return ids.astype(np.int32), q[ids] / total, room / total


def split_logit(logit, copies):
    """Logit of sigmoid(logit) / copies, from ln w - ln(copies - w)."""
    out = np.empty(len(logit))
    for i, (l, c) in enumerate(zip(logit.astype(np.float64), copies)):
        if c == 1 or np.isnan(l) or l == -np.inf:
            out[i] = l
            continue
        ln_w = -math.log1p(math.exp(-l)) if l > 0 else l - math.log1p(math.exp(l))
        rest = 1 / (1 + math.exp(l)) if l < 700 else 0.0  # 1 - w
        out[i] = ln_w - math.log((c - 1) + rest)
    return out
