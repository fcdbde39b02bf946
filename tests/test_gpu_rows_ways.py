"""Every way of running the attention of few rows (units' widths, whole units and cut ones) where it can go
wrong: long contexts with blocks missing across the windows of table entries, masks' later words, values far from one, offsets."""

import numpy as np
import pytest

from tests.gpu_helpers import announce, require_gpu
from tests.rows_helpers import TEAMS_CHUNKS, TEAMS_TREE, WAYS_LATENT, WAYS_TREE, bf16, check
from tests.test_gpu_latent import LATENT, ROW, Absorbed, Chunks
from tests.test_gpu_tree import D, Case

pytestmark = pytest.mark.gpu


def lose_blocks(b, seed):
    """Takes entries out of every table: some alone, some side by side, each way that an entry is invalid."""
    rng = np.random.default_rng(seed)
    for s in range(b.S):
        last = int(b.c0[s]) // 16            # (the drafts' own blocks stay)
        if last < 8:
            continue
        at = rng.integers(0, last - 4, max(1, last // 24))
        b.tables[s, at] = rng.choice([-1, b.num_blocks, -2 ** 31, 2 ** 31 - 1], at.size)
        i = int(rng.integers(0, last - 6))
        b.tables[s, i:i + 5] = -1


@pytest.mark.parametrize("bits", ["tree", None])
@pytest.mark.parametrize("way", WAYS_TREE, ids=lambda w: f"way{w[0]}-{len(w[1])}")
def test_drafts_take_every_way(way, bits):
    torch = require_gpu()
    w, n, c0, hq, hkv = way
    c = Case(n, c0, hq, hkv, bits, seed=40 + w, directions="table")
    lose_blocks(c.b, w)
    got = c.check(f"tree way {w} {bits}")
    assert torch.equal(got, c.run())


@pytest.mark.parametrize("bits", ["tree", None])
@pytest.mark.parametrize("way", WAYS_LATENT, ids=lambda w: f"way{w[0]}-{len(w[1])}")
def test_latent_rows_take_every_way(way, bits):
    torch = require_gpu()
    w, n, c0, hq = way
    c = Absorbed(n, c0, hq, bits, seed=50 + w, directions="table")
    lose_blocks(c.b, w)
    got = c.check(f"latent way {w} {bits}")
    assert torch.equal(got, c.run())


@pytest.mark.parametrize("bits", ["tree", None])
@pytest.mark.parametrize("case", TEAMS_TREE, ids=lambda c: f"team{c[0]}-{len(c[1])}")
def test_drafts_in_teams(case, bits):
    """Units that share their keys side by side: all there, the last missing, sequences without rows; cut and whole."""
    torch = require_gpu()
    team, n, c0, hq, hkv = case
    c = Case(n, c0, hq, hkv, bits, seed=60 + team, directions="table")
    lose_blocks(c.b, team)
    got = c.check(f"tree teams of {team} {n[:4]} {bits}")
    assert torch.equal(got, c.run())


@pytest.mark.parametrize("case", TEAMS_CHUNKS, ids=lambda c: f"team{c[0]}-{c[1][0]}")
def test_chunks_in_teams(case):
    """Likewise for chunks, of which one unit ends some steps before its neighbour."""
    torch = require_gpu()
    team, n, c0, hq = case
    c = Chunks(n, c0, hq, seed=70 + team)
    got = c.check(f"latent prefill teams of {team} {n} {c0}")
    assert torch.equal(got, c.run())


@pytest.mark.parametrize("hq", [8, 64, 128])
def test_one_long_sequence_beside_short_ones(hq):
    """Shares that lie in one unit, and shares that hold many; a context without any valid block."""
    require_gpu()
    n = [1] * 40
    c0 = [int(x) for x in np.random.default_rng(hq).integers(0, 200, 40)]
    c0[7], c0[23] = 20000, 1000
    c = Absorbed(n, c0, hq, None, seed=hq)
    c.b.tables[23] = -1
    got = c.check(f"latent, one long sequence, {hq} heads")
    assert (got[23] == 0).all()
    c = Case([3] * 40, c0, 8, 1, seed=hq)
    c.b.tables[23] = -1
    got = c.check("tree, one long sequence")
    assert (got[69:72] == 0).all()


def test_last_words_of_masks_over_long_contexts():
    """Drafts of every word behind contexts that end inside a step of keys."""
    require_gpu()
    rng = np.random.default_rng(3)
    n, c0 = [256, 200], [1999, 345]
    rows = [sum(1 << int(x) for x in rng.integers(0, m, 3)) for m in n for _ in range(m)]
    Case(n, c0, 8, 4, rows, seed=4, words=4).check("tree, masks of four words")
    Absorbed(n, c0, 4, rows, seed=5, words=4).check("latent, masks of four words")


def test_a_chunk_without_mask_of_many_rows():
    require_gpu()
    Case([700], [130], 8, 2, None, seed=7).check("tree, 700 rows without a mask")
    Absorbed([333], [50], 6, None, seed=8).check("latent, 333 rows without a mask")


def test_bounds_far_above_the_rows_there_are():
    """max_q_len is a bound: whatever it says, the rows are those of the offsets."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    c = Case([5, 1, 8], [700, 20, 2000], 8, 2, seed=41)
    a = Absorbed([5, 1, 8], [700, 20, 2000], 16, seed=41)
    e = Chunks([40, 3], [700, 20], 2, seed=42)
    announce("bounds far above")
    for k, most in ((c, 256), (a, 64), (e, 2 ** 31 - 1)):
        k.b.max_n = most
        if k is not e:
            k.bits = np.concatenate([k.bits, np.zeros((k.b.rows, 3), dtype=np.int64)], 1)
        check(k.run(), *k.want(), f"bound {most}")
    # one sequence with all of the rows, among many with one
    Case([1] * 30 + [120], [90] * 31, 32, 8, None, seed=43).check("tree, one of many rows")
    Absorbed([1] * 30 + [60], [90] * 31, 16, None, seed=44).check("latent, one of many rows")
    Chunks([1] * 10 + [700], [1200] * 11, 2, seed=45).check("latent prefill, one of many rows")


def test_scale_and_scores_far_from_zero():
    """A scale of the caller's; scores of hundreds, where one weight is all there is."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    c = Case([5, 20], [300, 700], 8, 2, seed=9)
    c.q = (c.q.float() * 16).bfloat16()
    c.check("tree, large scores")
    a = Absorbed([2, 2], [300, 700], 20, "tree", seed=9)
    a.q = (a.q.float() * 16).bfloat16()
    a.check("latent, large scores")
    announce("latent, a scale of the caller's")
    tables, dirs, ctx, cu = a.b.cuda()
    got = torch.empty((a.b.rows, a.hq, LATENT), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(bros.bros_attn_workspace_size(3, 1, 1, 1, ROW, 0), dtype=torch.uint8, device="cuda")
    a.q = (a.q.float() / 16).bfloat16()       # (a power of two: the same scores from the scale)
    bros.bros_attn_latent(got, a.q.cuda(), cu, 2, a.pool.cuda(), tables, dirs, None, ctx, a.b.max_ctx,
                          mask=torch.from_numpy(a.bits).cuda(), scale=16 * 192 ** -0.5, workspace=ws)
    torch.cuda.synchronize()
    a.q = (a.q.float() * 16).bfloat16()
    check(got, *a.want(), "latent, scale")


@pytest.mark.parametrize("c0", [[200, 0], [1200, 90]])
@pytest.mark.parametrize("gain", [2.0 ** -40, 2.0 ** -9, 2.0 ** 12, 2.0 ** 60])
def test_expanded_values_far_from_one(gain, c0):
    """The values' weights: all small or large. (The result grows with them, so the bounds do.) Contexts of narrow
    units of rows and of wide ones."""
    require_gpu()
    c = Chunks([70, 33], c0, 2, seed=31)
    c.w[:, 128:] = (c.w[:, 128:].float() * gain).bfloat16()
    c.check(f"latent prefill, values of {gain}")


@pytest.mark.parametrize("n,c0,hq", [([301], [0], 3), ([20] * 90, [40] * 90, 6), ([64, 1, 65, 128, 129], [0, 900, 33, 64, 0], 2),
                                     ([65, 64], [1000, 7], 2), ([100] * 3, [950] * 3, 2)])
def test_expanded_units(n, c0, hq):
    """Narrow units and wide ones, whole and cut; contexts that end inside a step, and in the last tile of the dense rows."""
    torch = require_gpu()
    c = Chunks(n, c0, hq, seed=len(n), directions="table")
    got = c.check(f"latent prefill units {n[:5]} {c0[:5]}")
    assert torch.equal(got, c.run())


def test_expanded_sequences_without_context_behind_a_full_buffer():
    """The dense rows end where the second sequence would begin, which has more rows than tokens: zeros."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    for n0, c0 in ((64, 0), (64, 1216)):
        c = Chunks([n0, 5], [c0, 0], 2, seed=36)
        announce(f"latent prefill, nothing behind a full buffer, {c0}")
        tables, dirs, ctx, cu = c.b.cuda()
        ctx[1] = 3
        total = n0 + c0 - 62                      # dense rows for two sequences: rounded up, n0 + c0 of them
        q, pool, w = c.q.cuda(), c.pool.cuda(), c.w.cuda()
        out = torch.full((n0 + 5, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        ws = torch.full((bros.bros_latent_prefill_workspace_size(2, total, 2),), 255, dtype=torch.uint8, device="cuda")
        bros.bros_attn_latent_prefill(out, q, cu, n0, w, pool, tables, dirs, None, ctx, n0 + c0, total, workspace=ws)
        torch.cuda.synchronize()
        want, tol = c.want()
        check(out[:n0], want[:n0], tol[:n0], "the first sequence")
        assert (out[n0:] == 0).all()


def test_expanded_rows_of_different_sizes():
    """A row of 2^20 times the others': the rows before it share its tile of 32 values. Values are halves behind a
    power of two that brings the tile's largest magnitude m to 2^13 or more; halves below their
    normal range are off by at most 2^-25, which is 2^-38 of m. (From that row on, scores are in the millions,
    and which row takes all of the weight is a matter of roundings: those are only to be finite.)"""
    require_gpu()
    b = Chunks([96], [0], 2, seed=32)
    big = 70
    blk, slot = b.b.places(0, [big])
    b.pool[blk, slot, :LATENT] = (b.pool[blk, slot, :LATENT].float() * 2.0 ** 20).bfloat16()
    announce("latent prefill, rows of different sizes")
    got = b.run().double().cpu()
    assert got.isfinite().all()
    want, tol = b.want()
    m = (b.pool[b.b.places(0, [big])].double()[:, :LATENT] @ b.w[:, 128:].double().transpose(1, 2)).abs().amax((1, 2))   # [heads]
    tol[64:] += m[None, :, None] * 2.0 ** -38
    check(got[:big], want[:big], tol[:big], "rows of different sizes")


def test_expanded_slots_behind_the_context_hold_anything():
    """What lies behind the contexts in their last blocks, finite and huge, counts nowhere (the poisoned
    pool of the other tests holds NaN there)."""
    torch = require_gpu()
    c = Chunks([37, 5], [0, 90], 2, seed=33)
    announce("latent prefill, huge values behind the contexts")
    first = c.run()
    blk, slot = np.nonzero(~c.b.owned())
    c.pool[blk, slot] = 3.0e38
    assert torch.equal(first, c.run())
    c.pool[blk, slot] = 0.0
    assert torch.equal(first, c.run())


def test_latent_offsets_beyond_32_bits():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    nb = 300000                               # 5.5e9 bytes
    a = Absorbed([3], [900], 16, "tree", seed=34)
    e = Chunks([40], [500], 2, seed=35)
    announce("latent offsets")
    pool = torch.empty((nb, 16, ROW), dtype=torch.bfloat16, device="cuda")
    for c, call in ((a, "absorbed"), (e, "expanded")):
        tables, dirs, ctx, cu = c.b.cuda()
        pool[nb - c.b.num_blocks:] = c.pool.cuda()
        tables = torch.where(tables >= 0, tables + (nb - c.b.num_blocks), tables)
        q = c.q.cuda()
        if call == "absorbed":
            out = torch.empty((c.b.rows, c.hq, LATENT), dtype=torch.bfloat16, device="cuda")
            ws = torch.empty(bros.bros_attn_workspace_size(3, 1, 1, 1, ROW, 0), dtype=torch.uint8, device="cuda")
            bros.bros_attn_latent(out, q, cu, 3, pool, tables, dirs, None, ctx, c.b.max_ctx, mask=torch.from_numpy(c.bits).cuda(), workspace=ws)
        else:
            out = torch.empty((c.b.rows, c.hq, 128), dtype=torch.bfloat16, device="cuda")
            ws = torch.empty(bros.bros_latent_prefill_workspace_size(1, 540, 2), dtype=torch.uint8, device="cuda")
            bros.bros_attn_latent_prefill(out, q, cu, 40, c.w.cuda(), pool, tables, dirs, None, ctx, 540, 540, workspace=ws)
        torch.cuda.synchronize()
        check(out, *c.want(), f"latent offsets, {call}")
    # the append to the last block, and a commit there
    kv = bf16(np.random.default_rng(1), (3, ROW)).cuda()
    tables = torch.tensor([[nb - 1]], dtype=torch.int32).cuda()
    dirs, at, cu = torch.ones(1, dtype=torch.int8).cuda(), torch.tensor([5], dtype=torch.int32).cuda(), torch.tensor([0, 3], dtype=torch.int32).cuda()
    bros.bros_latent_append(None, None, kv, pool, tables, dirs, None, at, cu)
    torch.cuda.synchronize()
    assert torch.equal(pool[nb - 1, 5:8], kv)
    path = torch.tensor([[2]], dtype=torch.int32).cuda()
    bros.bros_tree_commit(pool, None, tables, dirs, None, at + 3, cu, path, torch.tensor([1], dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    assert torch.equal(pool[nb - 1, 5], kv[2]) and torch.equal(pool[nb - 1, 6:8], kv[1:])


def test_dirty_workspaces_and_two_streams():
    """Two calls at once, each with a workspace of its own that held anything before."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    c = Case([20] * 3, [3000] * 3, 8, 2, seed=36)
    a = Absorbed([2] * 3, [3000] * 3, 32, "tree", seed=37)
    announce("two calls at once")
    first_c, first_a = c.run(), a.run()
    tc, ta = c.b.cuda(), a.b.cuda()
    mc, ma = torch.from_numpy(c.bits).cuda(), torch.from_numpy(a.bits).cuda()
    wc = torch.full((bros.bros_attn_workspace_size(2, 1, 1, 1, D, 0),), 127, dtype=torch.uint8, device="cuda")
    wa = torch.full((bros.bros_attn_workspace_size(3, 1, 1, 1, ROW, 0),), 127, dtype=torch.uint8, device="cuda")
    oc, oa = torch.empty_like(first_c), torch.empty_like(first_a)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        q, k, v = c.dev
        bros.bros_attn_tree(oc, q, tc[3], 20, k, v, tc[0], tc[1], None, tc[2], c.b.max_ctx, mask=mc, workspace=wc, stream=s1)
        q, pool = a.dev
        bros.bros_attn_latent(oa, q, ta[3], 2, pool, ta[0], ta[1], None, ta[2], a.b.max_ctx, mask=ma, workspace=wa, stream=s2)
    torch.cuda.synchronize()
    assert torch.equal(oc, first_c) and torch.equal(oa, first_a)


@pytest.mark.parametrize("units", [32, 96])
def test_on_a_share_of_the_compute_units(units):
    """Fewer workgroups, other widths and cuts: within the same bounds."""
    require_gpu()
    from paper_2504_09590_amd import bros
    stream = bros.bros_stream_create_cu_share(0, units)
    try:
        for c in (Case([20, 3, 64], [3000, 500, 900], 16, 4, seed=51), Case([64] * 3, [5000, 400, 3000], 64, 8, seed=52),
                  Absorbed([2] * 3, [3000, 50, 700], 32, "tree", seed=53), Absorbed([1] * 20, [1500] * 20, 128, None, seed=54),
                  Chunks([256, 250], [1500, 40], 3, seed=55), Chunks([300], [0], 4, seed=56)):
            c.check(f"a share of {units} compute units, {type(c).__name__}", stream=stream)
    finally:
        bros.bros_stream_destroy(stream)


def test_directions_by_class():
    """Without directions a sequence's class gives them: 0 from the left, 1 from the right."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    for c in (Case([20, 3, 9], [300, 500, 0], 16, 4, seed=61), Absorbed([2, 3, 1], [300, 50, 700], 16, "tree", seed=62),
              Chunks([70, 33, 5], [1500, 40, 3], 2, seed=63)):
        announce(f"directions by class, {type(c).__name__}")
        first = c.run()
        tables, dirs, ctx, cu = c.b.cuda()
        cls = (dirs < 0).to(torch.uint8)
        out = torch.full_like(first, 7.0)
        if isinstance(c, Chunks):
            q, pool, w = c.dev
            total = int(c.b.ctx.sum())
            ws = torch.empty(bros.bros_latent_prefill_workspace_size(3, total, 2), dtype=torch.uint8, device="cuda")
            bros.bros_attn_latent_prefill(out, q, cu, c.b.max_n, w, pool, tables, None, cls, ctx, c.b.max_ctx, total, workspace=ws)
        else:
            mask = torch.from_numpy(c.bits).cuda()
            latent = isinstance(c, Absorbed)
            ws = torch.empty(bros.bros_attn_workspace_size(3 if latent else 2, 1, 1, 1, ROW if latent else D, 0), dtype=torch.uint8, device="cuda")
            call = bros.bros_attn_latent if latent else bros.bros_attn_tree
            q, *pools = c.dev
            call(out, q, cu, c.b.max_n, *pools, tables, None, cls, ctx, c.b.max_ctx, mask=mask, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(out, first)
    # the append and the commit, into a pool of zeros: the same slots either way
    rng = np.random.default_rng(64)
    b = Absorbed([6, 3, 8], [30, 5, 100], 4, None, seed=64).b
    tables, dirs, ctx, cu = b.cuda()
    cls, kv = (dirs < 0).to(torch.uint8), bf16(rng, (17, ROW)).cuda()
    at = torch.from_numpy(b.c0.astype(np.int32)).cuda()
    path, lens = torch.tensor([[4, 2], [2, 0], [7, 3]], dtype=torch.int32).cuda(), torch.tensor([2, 2, 1], dtype=torch.int32).cuda()
    pools = []
    for way in ((dirs, None), (None, cls)):
        pool = torch.zeros((b.num_blocks, 16, ROW), dtype=torch.bfloat16, device="cuda")
        bros.bros_latent_append(None, None, kv, pool, tables, *way, at, cu)
        bros.bros_tree_commit(pool, None, tables, *way, ctx, cu, path, lens)
        pools.append(pool)
    torch.cuda.synchronize()
    assert torch.equal(*pools) and int((pools[0] != 0).any(-1).sum()) == 17
