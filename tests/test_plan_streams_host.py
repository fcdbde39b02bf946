"""PlanExecutor's plans on streams of the caller's (no GPU). It makes a plan's id lists on the plan's
stream: their memory is then handed out again in that stream's order only, behind the
kernels that read them. And a plan waits for the one before it: they share the staging."""

import contextlib
import types

import numpy as np
import pytest
import torch

pytest.importorskip("paper_2504_09590_amd.bros", reason="libbros_attn.so not built")

from paper_2504_09590_amd import swap  # noqa: E402


class Stream:
    def __init__(self, name, log):
        self.name, self.log = name, log

    def synchronize(self):
        pass

    def record_event(self):
        self.log.append(("end", self.name))
        return f"end of {self.name}'s plan"

    def wait_event(self, e):
        self.log.append(("wait", self.name, e))


def executor(monkeypatch, log):
    """An executor without a device; what it does goes to `log`."""
    current = ["the current stream"]

    @contextlib.contextmanager
    def stream(s):
        current.append(s)
        yield
        current.pop()

    monkeypatch.setattr(swap.torch.cuda, "stream", stream)
    monkeypatch.setattr(swap.bros, "bros_copy_dma", lambda *a, **kw: None)

    class Watched(swap.PlanExecutor):
        def __init__(self):
            self.pools = (torch.zeros(1), torch.zeros(1))
            self._gather = self._scatter = lambda *a, **kw: None
            self.max_rows, self.store = 2, {(3, 0): (torch.zeros(2),) * 2, (3, 1): (torch.zeros(2),) * 2}
            self.staging = self.host = [torch.zeros((2, 2))] * 2
            self._done = None

        def _ids(self, ids):
            log.append(("ids", current[-1]))
            return super()._ids(ids)

    return Watched()


def test_ids_are_made_on_the_given_stream(monkeypatch):
    log = []
    ex, at = executor(monkeypatch, log), Stream("side", log)
    plan = types.SimpleNamespace(victims=np.array([[4, 0, 1, 2]]), move_src=np.array([1, 2, 3]), move_dst=np.array([5, 6, 7]),
                                 restore_pos=np.array([0, 1]), restore_dst=np.array([8, 9]))
    ex.execute(3, plan, stream=at)
    assert [x[1] for x in log if x[0] == "ids"] == [at] * 6


def test_a_plan_waits_for_the_one_before(monkeypatch):
    log = []
    ex = executor(monkeypatch, log)
    plan = types.SimpleNamespace(victims=np.zeros((0, 4), dtype=int), move_src=np.array([1]), move_dst=np.array([5]),
                                 restore_pos=np.array([]), restore_dst=np.array([]))
    a, b = Stream("a", log), Stream("b", log)
    ex.execute(3, plan, stream=a)
    ex.execute(3, plan, stream=b)
    assert log == [("ids", a), ("ids", a), ("end", "a"), ("wait", "b", "end of a's plan"), ("ids", b), ("ids", b), ("end", "b")]


def test_a_plan_waits_for_one_that_failed(monkeypatch):
    log = []
    ex = executor(monkeypatch, log)
    nothing = np.zeros((0, 4), dtype=int)
    lost = types.SimpleNamespace(victims=nothing, move_src=np.array([1]), move_dst=np.array([5]), restore_pos=np.array([77]),
                                 restore_dst=np.array([8]))
    with pytest.raises(KeyError):      # (a row that was never saved; its moves are on the way)
        ex.execute(3, lost, stream=Stream("a", log))
    ex.execute(3, types.SimpleNamespace(victims=nothing, move_src=np.array([1]), move_dst=np.array([5]), restore_pos=np.array([]),
                                        restore_dst=np.array([])), stream=Stream("b", log))
    assert [x for x in log if x[0] != "ids"] == [("end", "a"), ("wait", "b", "end of a's plan"), ("end", "b")]
