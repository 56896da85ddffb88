"""What the calls of the binding make for themselves when their kernels run on another stream than the current one: where it is taken
from, and what that stream waits for.  No GPU: the library and the streams are stand-ins that note what they are asked."""
import contextlib

import pytest
import torch

from paper_2207_12000_b200 import build as libbuild


class Stream:
    def __init__(self, name, log):
        self.name, self.cuda_stream, self.log = name, id(self), log

    def wait_stream(self, other):
        self.log.append(("wait", self.name, other.name))


class Library:
    """The real sizes of workspaces, and a note instead of every launch."""

    def __init__(self, real, log):
        self.real, self.log = real, log

    def __getattr__(self, name):
        if name.endswith("_workspace"):
            return getattr(self.real, name)
        return lambda *args: self.log.append(("launch", name)) or 0


@pytest.fixture
def world(monkeypatch):
    libbuild.build()
    from paper_2207_12000_b200 import binding as B
    log, on = [], ["current"]
    current, side = Stream("current", log), Stream("side", log)
    empty, zeros, clamp = torch.empty, torch.zeros, torch.Tensor.clamp

    @contextlib.contextmanager
    def stream(s):
        on.append(s.name)
        yield
        on.pop()

    def noted(make, what):
        def f(*args, **kwargs):
            log.append((what, on[-1]))
            return make(*args, **kwargs)
        return f

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: {current.cuda_stream: current, side.cuda_stream: side}[handle])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: current)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)  # (what get_device says of a host tensor)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: log.append(("record", s.name)))
    monkeypatch.setattr(torch.Tensor, "clamp", noted(clamp, "convert"))
    monkeypatch.setattr(torch, "empty", noted(empty, "empty"))
    monkeypatch.setattr(torch, "zeros", noted(zeros, "zeros"))
    monkeypatch.setattr(B, "_lib", Library(B._lib, log))
    monkeypatch.setattr(B, "_raw_stream", lambda device: 0)
    return B, side, log


def check_log(log, workspace):
    launch = [i for i, e in enumerate(log) if e[0] == "launch"]
    assert len(launch) == 1
    before, wait = log[:launch[0]], ("wait", "side", "current")
    # a block of the current stream's memory: the side stream waits for its last users and the allocator hears of the side stream
    for i, e in enumerate(before):
        if e == ("empty", "current"):
            assert wait in before[i:] and ("record", "side") in log[i:]
        if e[0] in ("zeros", "convert"):
            assert e[1] == "side" and wait in before[:i]
    assert ("empty", "side") in before or not workspace


CALLS = {
    "lookup": (False, lambda B, **k: B.gnnpre_embedding_lookup(torch.ones((5, 8)), torch.arange(3), **k), (3, 8)),
    "table_grad": (True, lambda B, **k: B.gnnpre_embedding_grad(torch.ones((3, 8)), torch.arange(3), 5, **k), (5, 8)),
    "lc_grad": (True, lambda B, **k: B.gnnpre_lc_first_layer_grad([torch.ones((9, 8))], torch.arange(3), torch.ones((1, 3, 16)), **k), (16, 8)),
    "lc": (False, lambda B, **k: B.gnnpre_lc_first_layer([torch.ones((9, 8))], torch.arange(3), torch.ones((16, 8)), **k), (1, 3, 16)),
    "orth": (True, lambda B, **k: B.gnnpre_orthogonalize(torch.ones((16, 8)), **k), (16, 8)),
}


@pytest.mark.parametrize("result", ("made", "given"))
@pytest.mark.parametrize("name", CALLS)
def test_what_a_call_makes_for_itself_is_ordered_with_its_stream(world, name, result):
    B, side, log = world
    workspace, call, shape = CALLS[name]
    out = None if result == "made" else torch.ones(shape)
    for check in (False, True) if name in ("lc", "lc_grad", "orth") else (None,):
        del log[:]
        call(B, out=out, stream=side, **({} if check is None else {"check": check}))
        check_log(log, workspace)
        if result == "given" and not check and name not in ("lc", "lc_grad"):  # nothing of the current stream's: nothing to wait for
            assert not any(e[0] == "wait" for e in log)


@pytest.mark.parametrize("name", CALLS)
def test_on_the_current_stream_nothing_waits(world, name):
    B, side, log = world
    workspace, call, shape = CALLS[name]
    call(B)
    assert not any(e[0] in ("wait", "record") or e[-1] == "side" for e in log)


def test_hops_that_a_call_makes_are_ordered_with_its_stream(world):
    B, side, log = world
    plan = B.Plan(0, nnz_tilde=7)
    X = torch.ones((5, 8))
    for call in (lambda: B.gnnpre_propagate(plan, X, 3, stream=side), lambda: B.gnnpre_propagate_weighted(plan, X, (0.5, 0.5), stream=side),
                 lambda: B.gnnpre_degrees(torch.zeros(6, dtype=torch.int64), torch.zeros(0, dtype=torch.int32), stream=side)):
        del log[:]
        call()
        log[:] = [e for e in log if e[0] != "zeros"]
        check_log(log, False)
        assert ("empty", "current") in log
