"""bros_tree_commit at the ends of its sizes."""

import pytest

from tests.gpu_helpers import announce, require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,dtype", [(16384, "float32"), (16383, "float32"), (16384, "bfloat16"), (1, "float32")])
def test_most_heads(heads, dtype):
    """Every head's row of both pools moves, whatever their number and size."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    announce(f"commit of {heads} heads, {dtype}")
    dt = getattr(torch, dtype)
    k = torch.arange(2 * 16, device="cuda", dtype=torch.float32).view(2, 1, 16, 1).expand(2, heads, 16, 128).to(dt).contiguous()
    v = k + 64
    k_was, v_was = k.clone(), v.clone()
    tables = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    dirs = torch.ones(1, dtype=torch.int8, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    bros.bros_tree_commit(k, v, tables, dirs, None, i32(20), i32(0, 6), i32(5, 3).view(1, 2), i32(2))   # drafts at positions 14 .. 19
    torch.cuda.synchronize()
    for got, was in ((k, k_was), (v, v_was)):
        assert torch.equal(got[1, :, 14], was[0, :, 3]) and torch.equal(got[1, :, 15], was[0, :, 1])
        got[1, :, 14:], was[1, :, 14:] = 0, 0
        assert torch.equal(got, was)


def test_offsets_and_lengths_that_are_inconsistent():
    """Lengths below the drafts there are or below zero, and offsets out of order, near the ends of 32 bits too: nothing moves."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    announce("commit, inconsistent lengths")
    k = torch.randn((6, 2, 16, 128), device="cuda")
    v = torch.randn_like(k)
    k_was, v_was = k.clone(), v.clone()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    tables = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    dirs = torch.ones(3, dtype=torch.int8, device="cuda")
    path = i32(3, 1, 2, 0, 3, 2).view(3, 2)
    for ctx in ((-2 ** 31, -2 ** 31 + 1, -1), (3, 0, 2)):
        bros.bros_tree_commit(k, v, tables, dirs, None, i32(*ctx), i32(0, 4, 8, 12), path, i32(2, 2, 2))
    for cu in ((12, 8, 4, 0), (2 ** 31 - 1, 0, -2 ** 31, -2 ** 31), (0, -2 ** 31, 2 ** 31 - 1, 0), (5, 5, 5, 5)):
        bros.bros_tree_commit(k, v, tables, dirs, None, i32(20, 20, 20), i32(*cu), path, i32(2, 2, 2))
    torch.cuda.synchronize()
    assert torch.equal(k, k_was) and torch.equal(v, v_was)
