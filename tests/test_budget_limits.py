"""What the operators of include/gs_budget.h refuse, before any device work
(no GPU needed: nothing here launches a kernel), and their sizes."""
import ctypes

import pytest
import torch

import paper_2607_01164_amd as gs
from paper_2607_01164_amd import gsq

SIZE_ERR = ctypes.c_size_t(-1).value
FAKE = 4096  # never followed
BIG = 1 << 60


def err(status):
    return status, gs.load_library().gs_last_error().decode()


def params(p=FAKE):
    return gsq.GsParams(p, p, p, p, p)


def index(n=10, pairs=5):
    g = gs.make_grid((4, 4, 4))
    return gsq.GsIndex(FAKE, FAKE, FAKE, 100, FAKE, BIG, pairs, n, g, 0.01)


def gauss(n=10):
    return gsq.GsGaussians(n, FAKE, FAKE, FAKE, FAKE, FAKE)


def query(kind=gs.GS_QUERY_POINTS, n=100, dims=(0, 0, 0)):
    return gsq.GsQuery(kind, (ctypes.c_int32 * 3)(*dims), n, None, FAKE)


def shares(g=None, i=None, q=None, plan=FAKE, plan_bytes=BIG, influence=FAKE, decay=0.0, score=FAKE, work=FAKE,
           work_bytes=BIG):
    g, i, q = g or gauss(), i or index(), q or query()
    return err(gs.load_library().gs_shares(ctypes.byref(g), ctypes.byref(i), ctypes.byref(q), plan, plan_bytes,
                                           influence, None, decay, score, work, work_bytes, None))


@pytest.mark.parametrize("args,code,word", [
    (dict(influence=None), 1, "influence"), (dict(score=None), 1, "score"), (dict(decay=-0.5), 1, "decay"),
    (dict(decay=float("nan")), 1, "decay"), (dict(decay=float("inf")), 1, "decay"),
    (dict(i=index(pairs=-1)), 1, "built"), (dict(i=index(n=11)), 1, "built for"),
    (dict(q=query(kind=9)), 1, ""), (dict(q=query(gs.GS_QUERY_GRID, 0, (5, 4, 4))), 1, "multiple"),
    (dict(work=None), 3, "workspace"), (dict(work=FAKE + 1), 3, "workspace"), (dict(work_bytes=100), 3, "workspace"),
    (dict(plan=None), 3, "plan"), (dict(plan=FAKE + 4), 3, "plan"), (dict(plan_bytes=64), 3, "plan")])
def test_shares_refuses(args, code, word):
    st, msg = shares(**args)
    assert st == code and word in msg, msg


def test_shares_work():
    L = gs.load_library()
    size = lambda i, q: L.gs_shares_work_bytes(ctypes.byref(i), ctypes.byref(q))  # noqa: E731
    assert size(index(), query()) >= 1600
    assert size(index(), query(gs.GS_QUERY_GRID, 0, (8, 8, 8))) >= 2048
    assert size(index(pairs=-1), query()) == SIZE_ERR
    assert size(index(), query(kind=7)) == SIZE_ERR
    assert L.gs_shares_work_bytes(None, None) == SIZE_ERR


def evict(p=None, n=10, score=FAKE, budget=5, out=None, source=FAKE, work=FAKE, work_bytes=BIG):
    p, out = p or params(), out or params()
    return err(gs.load_library().gs_evict(ctypes.byref(p), n, score, None, budget, ctypes.byref(out), source, None,
                                          work, work_bytes, None))


@pytest.mark.parametrize("args,code,word", [
    (dict(n=-1), 1, "range"), (dict(n=1 << 31), 1, "range"), (dict(budget=-1), 1, "range"),
    (dict(budget=1 << 31), 1, "range"), (dict(score=None), 1, "input"), (dict(p=params(None)), 1, "input"),
    (dict(out=params(None)), 1, "output"), (dict(source=None), 1, "output"), (dict(work=None), 3, "workspace"),
    (dict(work=FAKE + 8), 3, "workspace"), (dict(work_bytes=16), 3, "workspace")])
def test_evict_refuses(args, code, word):
    st, msg = evict(**args)
    assert st == code and word in msg, msg


def test_evict_of_nothing():
    assert evict(budget=0, p=params(None), out=params(None), score=None, source=None, work=None)[0] == 0
    assert evict(n=0, p=params(None), out=params(None), score=None, source=None, work=None)[0] == 0
    L = gs.load_library()
    assert L.gs_evict_work_bytes(-1) == SIZE_ERR and L.gs_evict_work_bytes(1 << 31) == SIZE_ERR
    assert L.gs_evict_work_bytes(0) > 0


def draw(rows=3, n=100, scores=FAKE, stride=100, temperature=1.0, top_p=1.0, min_p=0.0, top_k=0, kind=0, draws=4,
         uniform=FAKE, ids=FAKE, work=FAKE, work_bytes=BIG, settings=True):
    p = gsq.GsDrawParams(temperature, top_p, min_p, top_k, 0, kind)
    return err(gs.load_library().gs_draw(rows, n, scores, stride, None, ctypes.byref(p) if settings else None, draws,
                                         uniform, ids, None, work, work_bytes, None))


NAN = float("nan")


@pytest.mark.parametrize("args,code,word", [
    (dict(rows=-1), 1, "range"), (dict(n=-1), 1, "range"), (dict(draws=-1), 1, "range"),
    (dict(rows=1 << 31), 1, "range"), (dict(n=1 << 31, stride=1 << 31), 1, "range"),
    (dict(draws=1 << 31), 1, "range"), (dict(rows=1 << 20, n=1 << 20, stride=1 << 20), 1, "range"),
    (dict(rows=1 << 20, draws=1 << 20), 1, "range"), (dict(settings=False), 1, "params"),
    (dict(temperature=-1.0), 1, "temperature"), (dict(temperature=NAN), 1, "temperature"),
    (dict(temperature=float("inf")), 1, "temperature"), (dict(top_p=-0.1), 1, "top_p"),
    (dict(top_p=1.1), 1, "top_p"), (dict(top_p=NAN), 1, "top_p"), (dict(min_p=-0.1), 1, "min_p"),
    (dict(min_p=1.5), 1, "min_p"), (dict(min_p=NAN), 1, "min_p"), (dict(top_k=-1), 1, "top_k"),
    (dict(kind=2), 1, "type"), (dict(stride=99), 1, "stride"), (dict(scores=None), 1, "null"),
    (dict(uniform=None), 1, "null"), (dict(ids=None), 1, "null"), (dict(work=None), 3, "workspace"),
    (dict(work=FAKE + 16), 3, "workspace"), (dict(n=20000, stride=20000, work_bytes=1000), 3, "workspace")])
def test_draw_refuses(args, code, word):
    st, msg = draw(**args)
    assert st == code and word in msg, msg


def test_draw_of_nothing():
    assert draw(rows=0, scores=None, uniform=None, ids=None, work=None)[0] == 0
    assert draw(draws=0, scores=None, uniform=None, ids=None, work=None)[0] == 0
    L = gs.load_library()
    assert L.gs_draw_work_bytes(-1, 5, 5) == SIZE_ERR and L.gs_draw_work_bytes(1 << 30, 1 << 30, 1) == SIZE_ERR
    assert L.gs_draw_work_bytes(1, 100000, 5) >= 200000


def split(p=None, n=10, ids=FAKE, count=5, work=FAKE, work_bytes=BIG):
    p = p or params()
    return err(gs.load_library().gs_split(ctypes.byref(p), n, ids, count, None, None, work, work_bytes, None))


@pytest.mark.parametrize("args,code,word", [
    (dict(n=-1), 1, "range"), (dict(count=-1), 1, "range"), (dict(n=(1 << 31) - 1, count=1), 1, "range"),
    (dict(n=1 << 31), 1, "range"), (dict(p=params(None)), 1, "null"), (dict(ids=None), 1, "null"),
    (dict(work=None), 3, "workspace"), (dict(work=FAKE + 2), 3, "workspace"), (dict(work_bytes=39), 3, "workspace")])
def test_split_refuses(args, code, word):
    st, msg = split(**args)
    assert st == code and word in msg, msg


def test_split_of_nothing():
    assert split(count=0, p=params(None), ids=None, work=None)[0] == 0
    L = gs.load_library()
    assert L.gs_split_work_bytes(-1) == SIZE_ERR and L.gs_split_work_bytes(1000) >= 4000


def test_binding_refuses_host_tensors():
    """Before the library is reached: types, devices, sizes."""
    h = torch.zeros(8)
    u = torch.zeros(4, dtype=torch.float64)
    i = torch.zeros(4, dtype=torch.int32)
    w = torch.zeros(256, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device"):
        gs.gs_draw(h, u, i, w)
    with pytest.raises(ValueError, match=r"\[rows"):
        gs.gs_draw(h.view(2, 4), u, i, w)
    with pytest.raises(ValueError, match="device"):
        gs.gs_draw(h.double(), u, i, w)
    p = gs.ParamSet.empty(8, "cpu")
    with pytest.raises(ValueError, match="fewer rows"):
        gs.gs_evict(p, 8, h, 5, gs.ParamSet.empty(4, "cpu"), i, w)
    with pytest.raises(ValueError, match="input rows"):
        gs.gs_evict(p, 9, h, 5, p, i, w)
    with pytest.raises(ValueError, match="score"):
        gs.gs_evict(p, 8, h, 4, gs.ParamSet.empty(4, "cpu"), i, w)
    with pytest.raises(ValueError, match="room"):
        gs.gs_split(p, 5, i, None, w)
    with pytest.raises(ValueError, match="ids"):
        gs.gs_split(p, 4, i, None, w)


def apart(first, step=1 << 16):
    """Addresses that no array here reaches from one to the next."""
    return [first + k * step for k in range(5)]


def test_overlapping_arrays_are_refused():
    """Outputs on inputs, at their ends too: the kernels read rows after others
    have written."""
    L, byref = gs.load_library(), ctypes.byref
    i, o = gsq.GsParams(*apart(1 << 20)), gsq.GsParams(*apart(1 << 24))
    far = [1 << 26, (1 << 26) + 4096, (1 << 26) + 8192]  # score, source, score_out

    def evict_at(out=o, score=far[0], pinned=None, source=far[1], score_out=far[2]):
        return err(L.gs_evict(byref(i), 10, score, pinned, 5, byref(out), source, score_out, FAKE, BIG, None))

    for args in (dict(out=i), dict(source=far[0]), dict(score_out=far[0] + 36), dict(score_out=far[0] - 16),
                 dict(pinned=far[1] + 19), dict(source=i.rot + 156), dict(source=i.weight_logit - 16)):
        st, msg = evict_at(**args)
        assert st == 1 and "overlaps" in msg, args

    p = gsq.GsDrawParams(1.0, 1.0, 0.0, 0, 0, gs.GS_SCORE_BF16)

    def draw_at(scores=1 << 20, lengths=None, uniform=1 << 22, ids=1 << 24, prob=1 << 26):
        return err(L.gs_draw(3, 100, scores, 120, lengths, byref(p), 4, uniform, ids, prob, FAKE, BIG, None))

    for args in (dict(ids=(1 << 20) + 676), dict(ids=(1 << 20) - 44), dict(prob=(1 << 22) + 92), dict(uniform=1 << 24),
                 dict(lengths=(1 << 26) + 44)):
        st, msg = draw_at(**args)
        assert st == 1 and "overlaps" in msg, args

    def split_at(ids=far[0], source=far[1], score=far[2]):
        return err(L.gs_split(byref(o), 10, ids, 6, source, score, FAKE, BIG, None))

    for args in (dict(ids=far[1] + 40), dict(ids=far[1] + 60), dict(ids=far[2]), dict(source=far[2] + 60),
                 dict(ids=o.mean + 188), dict(source=o.value_logit), dict(score=o.weight_logit + 60)):
        st, msg = split_at(**args)
        assert st == 1 and "overlap" in msg, args

    g = gsq.GsGaussians(10, *apart(1 << 20))
    ix, q = index(), query()

    def shares_at(influence=1 << 24, gain=1 << 25, score=1 << 26):
        return err(L.gs_shares(byref(g), byref(ix), byref(q), FAKE, BIG, influence, gain, 0.0, score, FAKE, BIG, None))

    for args in (dict(score=(1 << 24) + 396), dict(score=(1 << 25) - 36), dict(score=g.mean + 116), dict(score=g.rot)):
        st, msg = shares_at(**args)
        assert st == 1 and "overlaps" in msg, args
