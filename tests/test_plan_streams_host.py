"""PlanExecutor makes its id lists on the stream that it is given (no GPU): their memory is then
handed out again in that stream's order only, behind the kernels that read them."""

import contextlib
import types

import numpy as np
import pytest
import torch

pytest.importorskip("paper_2504_09590_amd.bros", reason="libbros_attn.so not built")

from paper_2504_09590_amd import swap  # noqa: E402


def test_ids_are_made_on_the_given_stream(monkeypatch):
    current, seen = ["the current stream"], []

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
            self.at = types.SimpleNamespace(synchronize=lambda: None)

        def _ids(self, ids):
            seen.append(current[-1])
            return super()._ids(ids)

    ex = Watched()
    plan = types.SimpleNamespace(victims=np.array([[4, 0, 1, 2]]), move_src=np.array([1, 2, 3]), move_dst=np.array([5, 6, 7]),
                                 restore_pos=np.array([0, 1]), restore_dst=np.array([8, 9]))
    ex.execute(3, plan, stream=ex.at)
    assert len(seen) == 6 and all(s is ex.at for s in seen)
