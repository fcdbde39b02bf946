"""The bounds of a step over a latent cache (no GPU)."""

import pytest
import torch

pytest.importorskip("paper_2504_09590_amd.bros", reason="libbros_attn.so not built")

from paper_2504_09590_amd import bros  # noqa: E402
from paper_2504_09590_amd.step import LatentStep  # noqa: E402
from tests.test_draft_steps_host import given  # noqa: E402


def test_bounds_of_chunks():
    pool, w = torch.zeros((5, 16, 576), dtype=torch.bfloat16), torch.zeros((4, 256, 512), dtype=torch.bfloat16)
    batch = given([40, 30, 1], prefill=2)                    # contexts of 49 and 39
    step = LatentStep(*batch, pool, w)
    assert step.max_ctx_pre == 49 and step.total_ctx == 88
    step = LatentStep(*batch, pool, w, max_ctx_chunks=64, total_ctx=120)
    assert step.max_ctx_pre == 64 and step.total_ctx == 120
    assert step.workspace.numel() >= bros.bros_latent_prefill_workspace_size(2, 120, 4)
    for kw in (dict(max_ctx_chunks=48), dict(total_ctx=87), dict(max_ctx_chunks=64, total_ctx=10)):
        with pytest.raises(ValueError, match="beyond"):
            LatentStep(*batch, pool, w, **kw)
    assert LatentStep(*given([1, 1]), pool, max_ctx_chunks=0).total_ctx == 0
