"""bros_attn_prefill_chunk_q8 against the fp64 oracle over the values the 8-bit pool
stands for."""

import dataclasses

import numpy as np
import pytest

import oracle
from paper_2504_09590_amd import workload as W
from tests import q8_helpers as Q
from tests.gpu_helpers import announce, owned_mask, require_gpu, with_direction_table

pytestmark = pytest.mark.gpu

WEIGHTS = 2.0 ** -7


def chunks(c0s, ns, group=4, hkv=2, seed=0, dirs=None, cls=None):
    cls = [W.RT if i % 3 else W.BE for i in range(len(ns))] if cls is None else cls
    return W.custom([c + n for c, n in zip(c0s, ns)], cls, hkv * group, hkv, seed=seed, num_prefill=len(ns), new_counts=ns,
                    spare_blocks=5, dirs=dirs, share_tails=dirs is None)


def run(q8, with_ws=True, ws_bytes=None, stream=None, max_ctx=None, max_q=None, pad=0):
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    b = q8.batch
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    q = bros._tensor(b.q_prefill, "bf16", "cuda")
    if pad:
        q = torch.cat([q, torch.full((pad,) + tuple(q.shape[1:]), float("nan"), dtype=q.dtype, device="cuda")])
    out = torch.full_like(q, 7.0)
    max_ctx = int(b.ctx_lens.max()) if max_ctx is None else max_ctx
    max_q = int(np.diff(b.cu_q).max()) if max_q is None else max_q
    size = bros.bros_attn_workspace_size(bros.BROS_WS_PREFILL, bros.BROS_BF16, q.shape[0], b.num_q_heads, 128, max_ctx)
    ws = torch.full((size if ws_bytes is None else ws_bytes,), 255, dtype=torch.uint8, device="cuda") if with_ws else None
    bros.bros_attn_prefill_chunk_q8(out, q, up(b.cu_q), max_q, up(q8.k), up(q8.v), up(q8.scales), up(b.block_tables), up(b.dir),
                                    up(b.cls), up(b.ctx_lens), max_ctx, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    return bros.to_host_bits(out)


def check(q8, got, what):
    b = q8.batch
    want = oracle.prefill_chunk(b.q_prefill, b.cu_q, b.k_pool, b.v_pool, b.block_tables, b.dir, b.ctx_lens, "bf16")
    seq = np.repeat(np.arange(b.num_prefill), np.diff(b.cu_q))
    Q.check(got, want, b.q_prefill, b, seq, WEIGHTS, what)


# A bound of 30000 tokens takes the call to units of 128 rows, the exact one to groups of 16 columns.
UNITS = 30000
BOUNDS = [None, UNITS]


@pytest.mark.parametrize("bound", BOUNDS)
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_edge_lengths_and_groups(group, bound):
    c0s = [0, 0, 0, 0, 5, 16, 31, 100, 3, 64, 0, 250]
    ns = [1, 16, 17, 130, 40, 1, 33, 64, 1, 16, 300, 7]
    b = chunks(c0s, ns, group, 2, seed=group)
    q8 = Q.poison(Q.held(b, group), owned_mask(b))
    announce(f"prefill_q8 edges G={group} bound={bound}")
    check(q8, run(q8, max_ctx=bound), f"edges G={group}")


@pytest.mark.parametrize("group,hkv", [(4, 2), (1, 8), (8, 1)])
def test_long_chunk_in_pieces_and_whole(group, hkv):
    b = chunks([9000, 0, 7], [200, 64, 1], group, hkv, seed=34 + group, cls=[W.RT] * 3)
    q8 = Q.poison(Q.held(b, group), owned_mask(b))
    announce(f"prefill_q8 200 rows on 9000 tokens, G={group} Hkv={hkv}")
    split, whole = run(q8), run(q8, with_ws=False)
    check(q8, split, "pieces")
    check(q8, whole, "whole")
    assert not np.array_equal(split, whole)
    assert np.array_equal(run(q8, ws_bytes=4096), whole)


def test_beyond_the_whole_table():
    # contexts whose table does not fit LDS: the ring variant
    b = chunks([40000, 100], [70, 30], 4, 2, seed=3, cls=[W.RT, W.BE])
    q8 = Q.held(b, 3)
    announce("prefill_q8 70 rows on 40000 tokens")
    check(q8, run(q8), "40000 tokens")


@pytest.mark.parametrize("group,hkv", [(1, 1), (2, 3), (4, 8), (8, 2)])
def test_groups_of_columns(group, hkv):
    # many sequences (more than a wave looks at at once), empty ones among them, deep contexts
    rng = np.random.default_rng(group)
    ns = rng.integers(0, 4, 90)
    ns[[3, 70, 88]] = 33, 17, 5
    c0s = rng.integers(0, 60, 90)
    c0s[[3, 70]] = 1300, 700
    m = 90 if hkv < 8 else 50
    b = chunks(c0s[:m].tolist(), ns[:m].tolist(), group, hkv, seed=50 + group)
    q8 = Q.poison(Q.held(b, group), owned_mask(b))
    announce(f"prefill_q8 groups of columns, G={group} Hkv={hkv}")
    n = int(b.cu_q[-1])
    got = run(q8, pad=5)
    assert (oracle.widen(got[n:], "bf16") == 7.0).all()
    check(q8, got[:n], "groups of columns")


@pytest.mark.parametrize("group,hkv,c0s,ns", [(4, 2, [4000, 30, 900], [20, 3, 9]), (8, 1, [9000], [9]), (1, 8, [1500, 0], [16, 7]),
                                               (2, 3, [20000, 5], [4, 33])])
def test_groups_of_columns_in_pieces(group, hkv, c0s, ns):
    b = chunks(c0s, ns, group, hkv, seed=70 + group, cls=[W.RT, W.BE, W.RT][:len(ns)])
    q8 = Q.poison(Q.held(b, group), owned_mask(b))
    announce(f"prefill_q8 groups of columns in pieces, {ns} rows on {c0s}, G={group} Hkv={hkv}")
    n = int(b.cu_q[-1])
    got = run(q8, pad=3)
    assert (oracle.widen(got[n:], "bf16") == 7.0).all()
    check(q8, got[:n], "pieces")
    assert np.array_equal(got, run(q8, pad=3))
    # a NaN in a row of V that the first new row does not see, and one that all see
    for at, first in ((c0s[0] + 2, 2), (1, 0)):
        blk, slot = oracle.physical_location(b.block_tables, b.dir, 0, np.array([at]))
        q8.v[blk, hkv - 1, slot, 3] = 0x7F
        nan = np.isnan(oracle.widen(run(q8), "bf16"))
        want = np.zeros_like(nan)
        want[first:ns[0], (hkv - 1) * group:, 3] = True
        assert np.array_equal(nan, want)


def test_nans_in_groups_of_columns():
    # every value of a row of V, one of V, an unset scale: each reaches the rows from its position on
    b = chunks([90], [40], 2, 3, seed=61, cls=[W.RT])
    q8 = Q.held(b, 61)
    for p, h, what in ((95, 0, "row"), (128, 1, "one"), (100, 2, "scale"), (3, 1, "one")):
        blk, slot = oracle.physical_location(b.block_tables, b.dir, 0, np.array([p]))
        if what == "row":
            q8.v[blk, h, slot] = 0xFF
        elif what == "one":
            q8.v[blk, h, slot, 77 + p % 5] = 0x7F
        else:
            q8.scales[blk, h, 1, slot] = 255
    announce("prefill_q8 NaNs in groups of columns")
    nan = ~np.isfinite(oracle.widen(run(q8), "bf16"))
    want = np.zeros_like(nan)
    want[5:, :2] = True
    want[38:, 2:4, 77 + 128 % 5] = True
    want[:, 2:4, 77 + 3] = True
    want[10:, 4:] = True
    assert np.array_equal(nan, want)


def test_many_units():
    rng = np.random.default_rng(4)
    b = chunks(rng.integers(0, 40, 300).tolist(), rng.integers(1, 40, 300).tolist(), 4, 2, seed=4)
    q8 = Q.poison(Q.held(b, 4), owned_mask(b))
    announce("prefill_q8 300 chunks")
    check(q8, run(q8), "300 chunks")


def test_directions_and_loose_bounds():
    b = chunks([20, 0, 77, 300], [50, 90, 16, 33], 4, 4, seed=5, dirs=[-1, 1, -1, 1])
    q8 = Q.poison(Q.held(b, 5), owned_mask(b))
    announce("prefill_q8 explicit directions")
    got = run(q8)
    check(q8, got, "explicit directions")
    assert np.array_equal(got, run(q8, with_ws=False))                  # groups of columns: no workspace
    loose = run(q8, max_ctx=UNITS, max_q=4000, with_ws=False)
    check(q8, loose, "loose bounds")
    assert np.array_equal(loose, run(q8, max_ctx=20000, with_ws=False))  # units, whatever the bounds
    t = with_direction_table(chunks([20, 0, 77, 300], [50, 90, 16, 33], 4, 4, seed=6))
    q8 = Q.poison(Q.held(t, 6), owned_mask(t))
    announce("prefill_q8 direction table")
    for bound in BOUNDS:
        check(q8, run(q8, max_ctx=bound), "direction table")


@pytest.mark.parametrize("bound", BOUNDS)
def test_empty_chunks_and_rows_behind_the_last(bound):
    b = chunks([20, 40, 77, 0], [50, 0, 16, 33], 4, 2, seed=7, cls=[W.RT] * 4)
    q8 = Q.held(b, 7)
    announce("prefill_q8 an empty chunk, rows behind the last")
    got = run(q8, pad=29, max_ctx=bound)
    n = int(b.cu_q[-1])
    assert (oracle.widen(got[n:], "bf16") == 7.0).all()
    check(q8, got[:n], "empty chunk")


@pytest.mark.parametrize("bound", BOUNDS)
def test_invalid_entries(bound):
    b = chunks([200, 0], [60, 90], 4, 2, seed=8, cls=[W.RT] * 2)
    tables = b.block_tables.copy()
    tables[0, [1, 9, 14]] = [-1, b.num_blocks, 2 ** 31 - 1]
    tables[1, 0] = -3
    b = dataclasses.replace(b, block_tables=tables)
    q8 = Q.held(b, 8)
    announce("prefill_q8 invalid entries")
    got = run(q8, max_ctx=bound)
    want = np.zeros(b.q_prefill.shape)
    for s in range(2):
        lo, hi = int(b.cu_q[s]), int(b.cu_q[s + 1])
        pos = np.arange(int(b.ctx_lens[s]))
        e = tables[s][pos // 16]
        pos = pos[(e >= 0) & (e < b.num_blocks)]
        blk, slot = oracle.physical_location(tables, b.dir, s, pos)
        k, v = (oracle.widen(p[blk, :, slot], "bf16") for p in (q8.batch.k_pool, q8.batch.v_pool))
        for r in range(lo, hi):
            seen = int((pos <= b.ctx_lens[s] - (hi - lo) + r - lo).sum())
            if seen:
                want[r] = oracle.softmax_attention(oracle.widen(b.q_prefill[r:r + 1], "bf16"), k, v, np.array([seen]),
                                                   oracle.default_scale(128))[0]
    # (rows of the second chunk below position 16 see nothing: zeros)
    assert (want[60:76] == 0).all() and (oracle.widen(got[60:76], "bf16") == 0).all()
    Q.check(got, want, b.q_prefill, q8.batch, np.repeat([0, 1], [60, 90]), WEIGHTS, "invalid entries")


def test_a_nan_reaches_only_rows_that_see_it():
    # a NaN in the cache of position p belongs to the rows from p on, also where they
    # share a tile of keys with earlier rows
    b = chunks([20, 0], [70, 40], 4, 2, seed=9, cls=[W.RT] * 2)
    q8 = Q.held(b, 9)
    blk, slot = oracle.physical_location(b.block_tables, b.dir, 0, np.array([57]))
    q8.v[blk, 1, slot, 5] = 0x7F
    blk, slot = oracle.physical_location(b.block_tables, b.dir, 1, np.array([30]))
    q8.k[blk, 0, slot, 9] = 0xFF
    announce("prefill_q8 NaN codes")
    for ws, bound in ((True, None), (True, UNITS), (False, UNITS)):
        got = oracle.widen(run(q8, with_ws=ws, max_ctx=bound), "bf16")
        nan = np.isnan(got)
        want = np.zeros_like(nan)
        want[57 - 20:70, 4:, 5] = True          # heads of KV head 1, dim 5, rows at positions 57 and later
        want[70 + 30:, :4] = True               # heads of KV head 0, rows at positions 30 and later
        assert np.array_equal(nan, want)


def test_a_query_that_is_not_finite_stays_alone():
    # infinite scores have no softmax (inf - inf), NaNs neither: NaN in their own rows, nothing elsewhere
    b = chunks([20, 0], [70, 40], 4, 2, seed=19, cls=[W.RT] * 2)
    q8 = Q.held(b, 19)
    odd = dataclasses.replace(q8, batch=dataclasses.replace(q8.batch, q_prefill=q8.batch.q_prefill.copy()))
    rows = [(3, 2, 0x7F80), (69, 7, 0x7FC0), (70 + 39, 0, 0xFF80)]        # +inf, NaN, -inf
    for r, h, bits in rows:
        odd.batch.q_prefill[r, h, 17] = bits
    announce("prefill_q8 queries that are not finite")
    for ws, bound in ((True, None), (True, UNITS), (False, UNITS)):
        got, plain = run(odd, with_ws=ws, max_ctx=bound), run(q8, with_ws=ws, max_ctx=bound)
        for r, h, _ in rows:
            assert np.isnan(oracle.widen(got[r, h], "bf16")).all()
            got[r, h] = plain[r, h]
        check(q8, got, "the other rows")


def test_on_a_share_and_captured():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    b = chunks([5000, 0, 7], [300, 64, 1], 4, 2, seed=10, cls=[W.RT] * 3)
    q8 = Q.held(b, 10)
    announce("prefill_q8 on 96 compute units")
    share = bros.bros_stream_create_cu_share(0, 96)
    try:
        got = run(q8, stream=share)
    finally:
        torch.cuda.synchronize()
        bros.bros_stream_destroy(share)
    check(q8, got, "96 compute units")

    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    q = bros._tensor(b.q_prefill, "bf16", "cuda")
    out = torch.empty_like(q)
    size = bros.bros_attn_workspace_size(bros.BROS_WS_PREFILL, bros.BROS_BF16, q.shape[0], 8, 128, 5300)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    args = (out, q, up(b.cu_q), 300, up(q8.k), up(q8.v), up(q8.scales), up(b.block_tables), up(b.dir), None, up(b.ctx_lens), 5300)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    announce("prefill_q8 captured")
    with torch.cuda.stream(side):
        bros.bros_attn_prefill_chunk_q8(*args, workspace=ws)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            bros.bros_attn_prefill_chunk_q8(*args, workspace=ws)
    for _ in range(3):
        out.zero_()
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(q8, bros.to_host_bits(out), "replay")


def test_far_blocks():
    # rows beyond 32-bit byte offsets: the variant with 64-bit ones
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    nb, hkv = 300000, 8
    b = chunks([150, 0], [70, 200], 2, hkv, seed=17, cls=[W.RT] * 2)
    q8 = Q.held(b, 17)
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    far = [torch.full((nb,) + x.shape[1:], 0x7F, dtype=torch.uint8, device="cuda") for x in (q8.k, q8.v, q8.scales)]
    for x, y in zip(far, (q8.k, q8.v, q8.scales)):
        x[nb - b.num_blocks:] = up(y)
    tables = np.where(b.block_tables >= 0, b.block_tables + (nb - b.num_blocks), b.block_tables).astype(np.int32)
    q = bros._tensor(b.q_prefill, "bf16", "cuda")
    out = torch.empty_like(q)
    announce("prefill_q8 in blocks beyond 4 GiB")
    for bound in (220, UNITS):
        out.fill_(7.0)
        bros.bros_attn_prefill_chunk_q8(out, q, up(b.cu_q), 200, *far, up(tables), up(b.dir), None, up(b.ctx_lens), bound)
        torch.cuda.synchronize()
        check(q8, bros.to_host_bits(out), f"far blocks, bound {bound}")
