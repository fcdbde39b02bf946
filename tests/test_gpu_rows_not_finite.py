"""Values that are not finite among keys that only some rows see: each wave of a unit leaves its own out of its products and
notes it, and they are added to the rows that see them, whichever wave met them."""

import numpy as np
import pytest

from tests.gpu_helpers import announce, require_gpu
from tests.rows_helpers import check
from tests.test_gpu_latent import Chunks
from tests.test_gpu_tree import D, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shift", [0, 16, 32, 48])
@pytest.mark.parametrize("n,c0,hq,hkv", [(4, [300], 8, 2), (6, [480, 17, 300], 8, 2), (2, [240] * 150, 8, 2), (20, [2000], 8, 2),
                                         (16, [4000] * 8, 16, 4), (30, [8000] * 16, 16, 4)])
def test_in_any_key_group(n, c0, hq, hkv, shift):
    """Drafts whose keys lie in the first or the second group of a step's keys, one wave's or another's, of whole units and cut
    ones, in many workgroups at once."""
    torch = require_gpu()
    c0 = [c // 64 * 64 + shift for c in c0]
    S = len(c0)
    rows = [(1 << j) | (2 if j % 2 else 0) for _ in range(S) for j in range(n)]   # every other draft sees draft 1
    c = Case([n] * S, c0, hq, hkv, rows, seed=n + shift)
    want, tol = c.want()
    for s in range(S):
        blk, slot = c.b.places(s, [c0[s] + 1])
        c.v[blk, :, slot, 7] = float("inf")
    announce(f"tree, not finite in any key group {n} {c0[:3]}")
    got = c.run()
    assert torch.equal(got.isnan(), c.run().isnan())
    got = got.double().cpu().view(S, n, hq, D)
    want, tol = want.view_as(got).clone(), tol.view_as(got)
    assert not torch.isfinite(got[:, 1::2, :, 7]).any()
    got[:, 1::2, :, 7] = want[:, 1::2, :, 7] = 0.0
    check(got, want, tol, "all others")


@pytest.mark.parametrize("n,c0", [([70, 33], [200, 0]), ([70, 33], [1200, 90]), ([512, 512], [1000, 1300])])
def test_in_expanded_chunks(n, c0):
    """A row's values of one head's dim, by a weight of which only that dim has any: rows before it are as without it."""
    torch = require_gpu()
    c = Chunks(n, c0, 2, seed=3)
    # (dim 9 of head 1 is made of latent dim 3 alone, of which no other weight takes anything)
    c.w[:, :, 3] = 0
    c.w[1, 128 + 9] = 0
    c.w[1, 128 + 9, 3] = 1.0
    want, tol = c.want()
    at = [30, 5]
    for s in range(2):
        blk, slot = c.b.places(s, [c0[s] + at[s]])
        c.pool[blk, slot, 3] = 3.0e38
    c.w[1, 128 + 9, 3] = 16.0                  # beyond what 32 bits hold
    announce(f"latent prefill, not finite in one dim {n}")
    got = c.run().double().cpu()
    c.w[1, 128 + 9, 3] = 1.0
    want2, tol2 = want.clone(), tol.clone()
    want2[:, 1, 9], tol2[:, 1, 9] = 16 * want[:, 1, 9], 16 * tol[:, 1, 9]
    for s in range(2):
        lo, hi = int(c.b.cu[s]) + at[s], int(c.b.cu[s + 1])
        assert not torch.isfinite(got[lo:hi, 1, 9]).any()
        got[lo:hi, 1, 9] = want2[lo:hi, 1, 9]
    check(got, want2, tol2, "all others")
