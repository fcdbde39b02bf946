"""What the steps of drafts and of a latent cache turn down when they are made, and their lengths (no GPU)."""

import types

import numpy as np
import pytest
import torch

pytest.importorskip("paper_2504_09590_amd.bros", reason="libbros_attn.so not built")

from paper_2504_09590_amd.step import DraftStep, LatentStep, _advance  # noqa: E402


def given(n, prefill=0, dtype="bf16"):
    cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    batch = types.SimpleNamespace(num_prefill=prefill, num_seqs=len(n), cu_new=cu, ctx_lens=np.asarray(n) + 9, num_q_heads=4,
                                  head_dim=128, dtype=dtype)
    dev = types.SimpleNamespace(block_tables=torch.zeros((len(n), 4), dtype=torch.int32), k_pool=torch.zeros((5, 2, 16, 128)))
    return batch, dev


def test_drafts():
    step = DraftStep(*given([3, 0, 5]))
    assert step.max_drafts == 5 and step.q.shape == (8, 4, 128) and step.max_ctx == 64 and step.drafts.tolist() == [3, 0, 5]
    for kw, words in [(dict(n=[3], prefill=1), "prefill"), (dict(n=[3], dtype="f32"), "bf16"), (dict(n=[257]), "at most 256")]:
        with pytest.raises(ValueError, match=words):
            DraftStep(*given(**kw))


def test_latent():
    pool = torch.zeros((5, 16, 576), dtype=torch.bfloat16)
    step = LatentStep(*given([40, 30, 1, 4], prefill=2), pool, torch.zeros((4, 256, 512), dtype=torch.bfloat16))
    assert step.out_chunks.shape == (70, 4, 128) and step.out_rows.shape == (5, 4, 512) and step.cu_rows.tolist() == [0, 1, 5]
    assert step.total_ctx == 88 and step.max_chunk == 40 and step.max_rows == 4
    few = LatentStep(*given([40, 30, 1, 4], prefill=2), pool, torch.zeros((4, 256, 512), dtype=torch.bfloat16), pass_heads=1)
    assert few.workspace.numel() <= step.workspace.numel()
    assert LatentStep(*given([1, 1]), pool).out_chunks.shape[0] == 0
    with pytest.raises(ValueError, match="weights"):
        LatentStep(*given([40], prefill=1), pool)


def test_lengths_behind_a_commit():
    pos0, drafts = torch.tensor([5, 7, 0, 9], dtype=torch.int32), torch.tensor([3, 0, 4, 9], dtype=torch.int32)
    ctx = torch.zeros(4, dtype=torch.int32)
    _advance(pos0, ctx, drafts, torch.tensor([2, 1, -3, 9], dtype=torch.int32), 6)
    assert pos0.tolist() == [7, 7, 0, 15] and ctx.tolist() == [10, 7, 4, 24]
