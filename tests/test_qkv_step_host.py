"""What QkvStep turns down when it is made (no GPU)."""

import types

import pytest
import torch

from paper_2504_09590_amd import workload as W

pytest.importorskip("paper_2504_09590_amd.bros", reason="libbros_attn.so not built")

from paper_2504_09590_amd.step import QkvStep  # noqa: E402


def made(dtype, eight):
    b = W.custom([40, 50], [W.RT, W.BE], 8, 2, dtype=dtype, num_prefill=1, new_counts=[40, 1], spare_blocks=1)
    shape = (b.num_blocks, 2, 16, 128)
    kind = torch.uint8 if eight else torch.float32 if dtype == "f32" else torch.bfloat16
    dev = types.SimpleNamespace(k_pool=torch.zeros(shape, dtype=kind), v_pool=torch.zeros(shape, dtype=kind))
    return QkvStep(b, dev, kv_scales=torch.zeros((b.num_blocks, 2, 2, 16), dtype=torch.uint8) if eight else None)


def test_an_eight_bit_cache_takes_no_32_bit_rows():
    # (refused before the first run writes the cache, not by its attention)
    with pytest.raises(ValueError, match="bf16"):
        made("f32", True)


@pytest.mark.parametrize("dtype,eight", [("bf16", False), ("bf16", True), ("f32", False)])
def test_the_others_are_made(dtype, eight):
    step = made(dtype, eight)
    assert step.q.shape == (41, 8, 128) and step.rows_prefill == 40
