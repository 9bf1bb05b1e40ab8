"""Plans of the optimiser's step on streams other than the current one: their
workspace is that stream's, and neither it nor the tensors' memory goes to
another allocation while calls still run. The first two need no GPU."""
import numpy as np
import pytest
import torch

import paper_2607_01164_amd as gs
from paper_2607_01164_amd import gsq


class Memory:
    """Stands for a tensor: which streams it was kept for."""

    def __init__(self):
        self.kept, self.device = [], "device"

    def record_stream(self, s):
        self.kept.append(s)

    def data_ptr(self):
        return 1 << 20

    def get_device(self):
        return 0

    def numel(self):
        return 1 << 20


class Library:
    def __getattr__(self, name):
        return lambda *a: 4096 if name.endswith("bytes") else gs.GS_OK


class Entered:
    now = 1

    def __init__(self, s):
        self.s = s

    def __enter__(self):
        self.was, Entered.now = Entered.now, self.s

    def __exit__(self, *a):
        Entered.now = self.was


@pytest.fixture
def streams(monkeypatch):
    """Streams are numbers, 1 the current one; returns [(stream, memory)] of
    the workspaces allocated."""
    made = []

    def alloc(nbytes, device):
        made.append((Entered.now, Memory()))
        return made[-1][1]

    monkeypatch.setattr(gsq, "load_library", Library)
    monkeypatch.setattr(gsq, "_alloc_bytes", alloc)
    monkeypatch.setattr(gsq, "_stream", lambda s=None: 1 if s is None else s)
    monkeypatch.setattr(gsq, "_torch_stream", lambda s, device: 1 if s is None else s, raising=False)
    monkeypatch.setattr(gsq, "_control_ptr", lambda *a: 8)
    monkeypatch.setattr(torch.cuda, "stream", Entered)
    return made


def test_a_plans_memory_is_kept_for_its_streams(streams):
    here = gs.AdamPlan([], device="device")
    gs.gs_adamw(here, step=1)
    gs.gs_grad_norm(here, None)
    assert streams[0][0] == 1 and streams[0][1].kept == []
    gs.gs_adamw(here, step=2, stream=5)
    gs.gs_grad_norm(here, None, stream=6)
    gs.gs_adamw(here, step=3, stream=5)
    assert sorted(streams[0][1].kept) == [5, 6]
    there = gs.AdamPlan([], device="device", stream=7)
    gs.gs_adamw(there, step=1, stream=7)
    gs.gs_adamw(there, step=2)
    gs.gs_adamw(there, step=3, stream=8)
    assert streams[1][0] == 7 and sorted(streams[1][1].kept) == [1, 8]


def test_a_plans_tensors_are_kept_for_its_streams(streams, monkeypatch):
    monkeypatch.setattr(gsq.AdamTensor, "c", lambda self: gsq.GsAdamwTensor())
    for kept, use in (([5], lambda p: gs.gs_adamw(p, step=1, stream=5)), ([], lambda p: gs.gs_adamw(p, step=1))):
        t = gs.AdamTensor(Memory(), Memory(), Memory(), Memory(), Memory(), Memory())
        use(gs.AdamPlan([t]))
        assert all(x.kept == kept for x in (t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale))
    t = gs.AdamTensor(None, Memory())
    gs.AdamPlan([t], stream=9)
    assert t.grad.kept == [9]


# ---- on the device ----------------------------------------------------------

def busy(x):
    """Some ten milliseconds of work on the current stream."""
    for _ in range(40):
        x.add_(1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["f32", "mxfp8"])
@pytest.mark.parametrize("kind", ["stream", "number"])
@pytest.mark.parametrize("made", ["here", "there"])
def test_a_plan_dropped_while_its_step_runs(made, kind, form):
    """The step waits behind other work of its stream while the plan and its
    moments are dropped and memory of the same sizes is taken and written on
    the current stream: none of it is theirs, and the step's result is right."""
    from test_gpu_optim import host, make
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    n = 300_007
    a, b = make(n, ("f32", "f32"), form, 3), make(n, ("f32", "f32"), form, 3)
    gs.gs_adamw(gs.AdamPlan([a]), step=5, seed=2)
    load = torch.zeros(1 << 28, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    arg = s if kind == "stream" else s.cuda_stream
    plan = gs.AdamPlan([b]) if made == "here" else gs.AdamPlan([b], stream=arg)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        busy(load)
    gs.gs_adamw(plan, step=5, seed=2, stream=arg)
    param = b.param
    theirs = [plan.work] + [x for x in (b.grad, b.m, b.v, b.m_scale, b.v_scale) if x is not None]
    sizes, places = [x.numel() * x.element_size() for x in theirs], {x.data_ptr() for x in theirs}
    del plan, b, theirs
    taken = [torch.full((k,), 255, dtype=torch.uint8, device="cuda") for k in sizes * 3]
    running = not s.query()
    assert not running or not places & {x.data_ptr() for x in taken}
    s.synchronize()
    np.testing.assert_array_equal(host(param), host(a.param))
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_a_plans_workspace_is_its_streams():
    """A plan made on a stream while the current one is busy with memory of the
    same size that was given back."""
    from test_gpu_optim import host, make
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    a, b = make(70_001, ("f32", "f32"), "f32", 8), make(70_001, ("f32", "f32"), "f32", 8)
    first = gs.AdamPlan([a])
    gs.gs_adamw(first, step=2)
    size = first.work.numel()
    load = torch.zeros(1 << 28, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    busy(load)
    given = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(4)]
    places = {x.data_ptr() for x in given}
    for x in given:
        x.fill_(255)
    del x, given
    plan = gs.AdamPlan([b], stream=s)
    assert plan.work.data_ptr() not in places
    gs.gs_adamw(plan, step=2, stream=s)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(host(b.param), host(a.param))
