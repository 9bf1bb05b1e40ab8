"""The operators of include/gs_budget.h refuse outputs and workspaces that
overlap each other or any input, the index's and the query's arrays and the
plan among them (no GPU needed: nothing here launches a kernel)."""
import ctypes

import pytest

import paper_2607_01164_amd as gs
from paper_2607_01164_amd import gsq

BIG = 1 << 60
SCORE, WORK, STEP = 1 << 40, 1 << 42, 1 << 32  # no array here reaches the next


def refused(status, name):
    msg = gs.load_library().gs_last_error().decode()
    assert status == 1 and msg.startswith(name) and "overlap" in msg, (status, msg)


def places(first, count):
    return [first + k * STEP for k in range(count)]


CELLS = (4, 4, 4)
QUERIES = {"points": (gs.GS_QUERY_POINTS, (0, 0, 0), 1000), "voxels": (gs.GS_QUERY_VOXELS, (9, 9, 9), 1000),
           "jitter": (gs.GS_QUERY_JITTER, (10, 10, 10), 1000), "jitter_ids": (gs.GS_QUERY_JITTER, (9, 9, 9), 1000),
           "grid": (gs.GS_QUERY_GRID, (12, 12, 12), 0)}


def call_shares(kind, score=SCORE, work=WORK):
    """Every input apart from the others; returns the spans of the inputs."""
    n, cap = 100, 500
    g = gsq.GsGaussians(n, *places(1 << 34, 5))
    grid = gs.make_grid(CELLS)
    keys, gids, offsets, iwork = places(1 << 36, 4)
    L, byref = gs.load_library(), ctypes.byref
    need = L.gs_index_work_bytes(n, byref(grid), cap)
    ix = gsq.GsIndex(keys, gids, offsets, cap, iwork, need, 50, n, grid, 0.01)
    ids, points, influence, gain, plan = places(1 << 38, 5)
    k, dims, count = QUERIES[kind]
    listed = kind in ("voxels", "jitter_ids")
    q = gsq.GsQuery(k, (ctypes.c_int32 * 3)(*dims), count, ids if listed else None,
                    points if kind != "grid" and kind != "voxels" else None)
    nq = L.gs_query_size(byref(q))
    spans = {"mean": (g.mean, 12 * n), "scale": (g.scale, 12 * n), "rot": (g.rot, 16 * n), "value": (g.value, 4 * n),
             "weight": (g.weight, 4 * n), "keys": (keys, 4 * cap), "gids": (gids, 4 * cap),
             "offsets": (offsets, 4 * 65), "index": (iwork, need), "influence": (influence, 4 * nq),
             "gain": (gain, 4 * nq)}
    if listed:
        spans["ids"] = (ids, 4 * nq)
    if q.points:
        spans["points"] = (points, 12 * nq)
    if kind != "grid":
        spans["plan"] = (plan, L.gs_plan_bytes(byref(q), byref(grid)))
    if score is None:
        return spans
    st = L.gs_shares(byref(g), byref(ix), byref(q), None if kind == "grid" else plan, BIG, influence, gain, 0.0,
                     score, work, BIG, None)
    refused(st, "gs_shares")


@pytest.mark.parametrize("kind", list(QUERIES))
def test_shares(kind):
    for name, (at, size) in call_shares(kind, score=None).items():
        # the first and the last word of an input; work is 256-byte aligned
        call_shares(kind, score=at - 396)
        call_shares(kind, score=at + size - 4)
        call_shares(kind, work=at)
        call_shares(kind, work=at + (size - 1) // 256 * 256)
    call_shares(kind, score=WORK)
    call_shares(kind, score=WORK - 396)


def evict(**moved):
    a = dict(zip(("mean", "log_scale", "rot", "value", "weight", "source", "score_out", "work"), places(1 << 36, 8)))
    a.update(moved)
    i = gsq.GsParams(*places(1 << 34, 5))
    o = gsq.GsParams(a["mean"], a["log_scale"], a["rot"], a["value"], a["weight"])
    L = gs.load_library()
    refused(L.gs_evict(ctypes.byref(i), 100, 1 << 40, 1 << 41, 50, ctypes.byref(o), a["source"], a["score_out"],
                       a["work"], BIG, None), "gs_evict")


def test_evict():
    at = dict(zip(("mean", "log_scale", "rot", "value", "weight", "source", "score_out", "work"), places(1 << 36, 8)))
    need = gs.load_library().gs_evict_work_bytes(100)
    evict(source=at["score_out"] + 196)
    evict(source=at["rot"] + 796)
    evict(score_out=at["mean"] - 196)
    evict(score_out=at["work"] + need - 4)
    evict(weight=at["value"] + 196)
    evict(work=at["mean"] + 512)
    evict(work=(1 << 40) + 256)  # the scores
    evict(work=1 << 41)  # pinned
    evict(work=1 << 34)


def draw(rows=3, n=100, ids=1 << 36, prob=1 << 37, work=1 << 38):
    p = gsq.GsDrawParams(1.0, 1.0, 0.0, 0, 0, gs.GS_SCORE_F32)
    refused(gs.load_library().gs_draw(rows, n, 1 << 32, n + 28, 1 << 33, ctypes.byref(p), 40, 1 << 34, ids, prob, work,
                                      BIG, None), "gs_draw")


def test_draw():
    draw(prob=(1 << 36) + 476)
    draw(prob=(1 << 36) - 476)
    draw(ids=(1 << 38) + 252)
    draw(work=(1 << 37) + 256)
    draw(work=(1 << 32) + 1024)
    draw(work=1 << 33)
    draw(work=(1 << 34) + 768)
    need = gs.load_library().gs_draw_work_bytes(1, 100000, 40)
    draw(rows=1, n=100000, ids=(1 << 38) + need - 4)


def split(**moved):
    a = dict(zip(("mean", "log_scale", "rot", "value", "weight", "ids", "source", "score", "work"), places(1 << 36, 9)))
    a.update(moved)
    p = gsq.GsParams(a["mean"], a["log_scale"], a["rot"], a["value"], a["weight"])
    refused(gs.load_library().gs_split(ctypes.byref(p), 100, a["ids"], 40, a["source"], a["score"], a["work"], BIG,
                                       None), "gs_split")


def test_split():
    at = dict(zip(("mean", "log_scale", "rot", "value", "weight", "ids", "source", "score", "work"), places(1 << 36, 9)))
    split(work=at["ids"])
    split(work=at["mean"] + 1536)
    split(work=at["source"] + 512)
    split(score=at["work"] + 396)
    split(value=at["weight"] - 556)
    split(log_scale=at["mean"] + 1676)
