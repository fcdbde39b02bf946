"""What the binding of the append takes and turns down (no GPU: what passes its checks of
shapes fails the device check, never a launch)."""

import pytest
import torch

from tests.test_q8_host import bros, py_call, rows


@pytest.mark.parametrize("sections", [(63,), (65,), (128,), (0,), (16, 24, 23), (70, -6), (16, 24, 24, 1)])
def test_sections_that_do_not_fit_the_table(sections):
    with pytest.raises(ValueError, match="sections"):
        bros.Rope(torch.zeros((9, 128)), sections=sections)


def test_sections_that_fit():
    assert bros.Rope(torch.zeros((9, 128)), sections=(64,)).axes == 1
    assert bros.Rope(torch.zeros((9, 96)), sections=(0, 24, 24)).axes == 3
    assert bros.Rope(torch.zeros((9, 96))).axes == 1


@pytest.mark.parametrize("kw", [dict(q=None), dict(q_out=None)])
def test_q_and_q_out_come_together(kw):
    with pytest.raises(ValueError, match="both q and q_out"):
        py_call(**kw)
    with pytest.raises(ValueError, match="current device"):
        py_call(q=None, q_out=None)


def test_one_head_of_many():
    # one KV head as every fourth of a wider tensor: contiguous within a token, whatever the heads' stride says
    pool = torch.zeros((4, 1, 16, 128), dtype=torch.bfloat16)
    k = rows(5, 4)[:, ::4]
    assert k.shape == (5, 1, 128) and k.stride(1) != 128
    with pytest.raises(ValueError, match="current device"):
        py_call(k=k, v=k, k_pool=pool, v_pool=pool)
