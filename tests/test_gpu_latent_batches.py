"""Batches of the expanded form as a serving loop makes them: sequences without rows beside others, padded to a
fixed number, and ranges and lengths that make a sequence one without rows, in units that are cut."""

import numpy as np
import pytest

from tests.gpu_helpers import announce, require_gpu
from tests.rows_helpers import check
from tests.test_gpu_latent import Chunks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,c0,hq", [
    ([0, 1400, 601], [0, 300, 900], 2), ([140, 0, 61], [1300, 0, 2000], 4), ([140, 61, 0, 0, 0], [1300, 2000, 0, 0, 0], 3),
    ([0, 0, 512, 0, 512, 0], [0, 40, 1000, 0, 1300, 1500], 2), ([700, 0, 600, 0, 1], [900, 0, 1100, 7, 1024], 2), ([0, 0, 1024], [2000, 0, 1100], 3)])
def test_sequences_without_rows(n, c0, hq):
    """Before, between and behind the others, with and without context; one, two and four workgroups side by side."""
    torch = require_gpu()
    c = Chunks(n, c0, hq, seed=len(n), directions="table")
    got = c.check(f"latent prefill without rows {n} {c0}")
    assert torch.equal(got, c.run())


def test_nothing_but_sequences_without_rows():
    """Rows that belong to no sequence stay as they were."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    c = Chunks([5, 40], [1500, 3], 2, seed=3)
    announce("latent prefill, rows of no sequence")
    tables, dirs, ctx, _ = c.b.cuda()
    out = torch.full((45, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((bros.bros_latent_prefill_workspace_size(2, 1548, 2),), 255, dtype=torch.uint8, device="cuda")
    args = c.q.cuda(), c.w.cuda(), c.pool.cuda()
    for cu in ([0, 0, 0], [45, 45, 45], [-1, 44, 46], [7, 3, 3]):
        bros.bros_attn_latent_prefill(out, args[0], torch.tensor(cu, dtype=torch.int32).cuda(), 45, args[1], args[2], tables, dirs, None, ctx,
                                      1505, 1548, workspace=ws)
        torch.cuda.synchronize()
        assert (out == 7.0).all(), cu


@pytest.mark.parametrize("place", [0, 1, 2])
def test_a_sequence_that_is_made_one_without_rows(place):
    """Its range lies outside the rows; its context above the bound. The others are as they are without it."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    n, c0 = [150, 70], [1300, 1100]
    n.insert(place, 0)
    c0.insert(place, 1700)
    c = Chunks(n, c0, 3, seed=4)
    want, tol = c.want()
    announce(f"latent prefill, a range outside the rows at {place}")
    tables, dirs, ctx, cu = c.b.cuda()
    q, w, pool = c.q.cuda(), c.w.cuda(), c.pool.cuda()
    ws = torch.full((bros.bros_latent_prefill_workspace_size(3, 1450 * 3, 3),), 255, dtype=torch.uint8, device="cuda")

    def run():
        out = torch.full((220, 3, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        bros.bros_attn_latent_prefill(out, q, cu, 150, w, pool, tables, dirs, None, ctx, 1450, 1450 * 3, workspace=ws)
        torch.cuda.synchronize()
        return out

    check(run(), want, tol, "a context above the bound, no rows")
    ctx[place] = -9
    check(run(), want, tol, "a length below zero, no rows")
    if place == 2:
        cu[3] = 500
        check(run(), want, tol, "a range that ends behind the rows")
    if place == 0:
        cu[0] = -4
        check(run(), want, tol, "a range that begins before the rows")


def test_a_padded_batch_in_a_graph():
    """A batch of a fixed number of sequences, whose offsets and lengths change between replays."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    c = Chunks([130, 40, 33, 1, 60], [1300, 0, 700, 1500, 20], 2, seed=5)
    announce("latent prefill, a padded batch in a graph")
    tables, dirs, _, _ = c.b.cuda()
    q, w, pool = c.q.cuda(), c.w.cuda(), c.pool.cuda()
    total = int(c.b.ctx.sum())
    ctx, cu = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")
    out = torch.empty((264, 2, 128), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(bros.bros_latent_prefill_workspace_size(5, total, 2), dtype=torch.uint8, device="cuda")
    call = lambda: bros.bros_attn_latent_prefill(out, q, cu, 130, w, pool, tables, dirs, None, ctx, 1501, total, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    full = c.b.n.copy()
    for there in ([1, 1, 1, 1, 1], [1, 0, 1, 0, 0], [0, 0, 0, 0, 0], [0, 1, 0, 0, 1], [1, 1, 0, 0, 0]):
        c.b.n = full * there
        c.b.ctx = c.b.n + c.b.c0 * there
        c.b.cu = np.concatenate([[0], np.cumsum(c.b.n)]).astype(np.int32)
        ctx.copy_(torch.from_numpy(c.b.ctx.astype(np.int32)))
        cu.copy_(torch.from_numpy(c.b.cu))
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        rows = int(c.b.cu[-1])
        c0 = c.b.c0
        c.b.c0 = c0 * np.asarray(there)
        want, tol = c.want()
        c.b.c0 = c0
        check(out[:rows], want[:rows], tol[:rows], f"sequences {there}")
        assert (out[rows:] == 7.0).all()
