"""bros_attn_prefill_chunk_q8 in units of 128 rows, at the lengths, masks and tables that
the rule would give to groups of 16 columns: wide tables with a loose bound take them
to the units (test_gpu_prefill_q8_edges.arranged)."""

import dataclasses

import numpy as np
import pytest

import oracle
from paper_2504_09590_amd import workload as W
from tests import q8_helpers as Q
from tests.gpu_helpers import announce, owned_mask, require_gpu, with_direction_table
from tests.test_gpu_prefill_q8 import WEIGHTS, check, chunks, run
from tests.test_gpu_prefill_q8_edges import arranged, check_spoilt, place, spoilt, wide

pytestmark = pytest.mark.gpu


def units(q8, **kw):
    return arranged(q8, "units", **kw)


@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_edge_lengths_and_groups(group):
    c0s = [0, 0, 0, 0, 5, 16, 31, 100, 3, 64, 0, 250]
    ns = [1, 16, 17, 130, 40, 1, 33, 64, 1, 16, 300, 7]
    b = chunks(c0s, ns, group, 2, seed=group)
    q8 = Q.poison(Q.held(b, group), owned_mask(b))
    announce(f"prefill_q8 units, edges G={group}")
    check(q8, units(q8), f"edges G={group}")


@pytest.mark.parametrize("group,hkv", [(1, 3), (8, 1)])
def test_one_row(group, hkv):
    for c0 in (0, 15, 16, 31, 32, 33):
        b = chunks([c0], [1], group, hkv, seed=c0, cls=[W.BE])
        q8 = Q.poison(Q.held(b, c0), owned_mask(b))
        announce(f"prefill_q8 units, one row on {c0}, G={group}")
        check(q8, units(q8), f"one row on {c0}")


def test_directions():
    b = chunks([20, 0, 77, 300], [50, 90, 16, 33], 4, 4, seed=5, dirs=[-1, 1, -1, 1])
    t = with_direction_table(chunks([20, 0, 77, 300], [50, 90, 16, 33], 4, 4, seed=6))
    for x, what in ((b, "explicit directions"), (t, "direction table")):
        q8 = Q.poison(Q.held(x, 5), owned_mask(x))
        announce(f"prefill_q8 units, {what}")
        check(q8, units(q8), what)


def test_empty_chunks_and_rows_behind_the_last():
    b = chunks([20, 40, 77, 0], [50, 0, 16, 33], 4, 2, seed=7, cls=[W.RT] * 4)
    q8 = Q.held(b, 7)
    announce("prefill_q8 units, an empty chunk, rows behind the last")
    n = int(b.cu_q[-1])
    got = units(q8, pad=29)
    assert (oracle.widen(got[n:], "bf16") == 7.0).all()
    check(q8, got[:n], "empty chunk")


def test_invalid_entries():
    b = chunks([200, 0], [60, 90], 4, 2, seed=8, cls=[W.RT] * 2)
    tables = b.block_tables.copy()
    tables[0, [1, 9, 14]] = [-1, b.num_blocks, 2 ** 31 - 1]
    tables[1, 0] = -3
    b = dataclasses.replace(b, block_tables=tables)
    q8 = Q.held(b, 8)
    announce("prefill_q8 units, invalid entries")
    got = units(q8)
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


@pytest.mark.parametrize("dirs", ["sequence", "table"])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_nans_reach_only_rows_that_see_them(group, dirs):
    # whole rows of V, single values and unset scales, in new keys and in the first and last cached ones
    c0, n = 90, 150
    b = chunks([c0], [n], group, 3, seed=61 + group, cls=[W.BE])
    if dirs == "table":
        b = with_direction_table(b)
    q8 = Q.held(b, 61)
    odd = spoilt(q8)
    want = np.zeros((n, 3 * group, 128), dtype=bool)
    for p, h, what in ((95, 0, "row"), (128, 1, "one"), (100, 2, "scale"), (3, 1, "one"), (89, 1, "one"), (91, 1, "one"),
                       (c0 + n - 1, 1, "one"), (160, 1, "key")):
        blk, slot = place(b, 0, p)
        dims = slice(None)
        if what == "row":
            odd.v[blk, h, slot] = 0xFF
        elif what == "one":
            dims = 10 + p % 100
            odd.v[blk, h, slot, dims] = 0x7F
        elif what == "scale":
            odd.scales[blk, h, 1, slot] = 255
        else:
            odd.k[blk, h, slot, 5] = 0xFF
        want[max(0, p - c0):, h * group:(h + 1) * group, dims] = True
    announce(f"prefill_q8 units, NaNs, G={group}, a direction per {dirs}")
    check_spoilt(units(odd), units(q8), want, f"G={group}")


@pytest.mark.parametrize("group", [1, 4])
def test_nans_in_units_in_pieces(group):
    # units of a long context, split into pieces whose partials are folded
    c0, n = 9000, 100
    b = chunks([c0], [n], group, 3, seed=group, cls=[W.RT])
    q8 = Q.held(b, 62)
    whole = units(q8)
    q8 = dataclasses.replace(q8, batch=wide(q8.batch))
    odd = spoilt(q8)
    want = np.zeros((n, 3 * group, 128), dtype=bool)
    for p, h in ((4, 0), (4000, 1), (c0 - 1, 2), (c0, 0), (c0 + 31, 1), (c0 + 77, 2)):
        blk, slot = place(b, 0, p)
        odd.v[blk, h, slot, p % 128] = 0x7F
        want[max(0, p - c0):, h * group:(h + 1) * group, p % 128] = True
    announce(f"prefill_q8 units in pieces, NaNs, G={group}")
    clean = run(q8, max_ctx=30000)
    assert not np.array_equal(clean, whole)      # (pieces: sums in another order)
    check(q8, clean, "pieces")
    check_spoilt(run(odd, max_ctx=30000), clean, want, f"G={group}")


def test_a_query_that_is_not_finite_stays_alone():
    b = chunks([20, 0], [70, 40], 4, 2, seed=19, cls=[W.RT] * 2)
    q8 = Q.held(b, 19)
    odd = dataclasses.replace(q8, batch=dataclasses.replace(q8.batch, q_prefill=q8.batch.q_prefill.copy()))
    rows = [(3, 2, 0x7F80), (69, 7, 0x7FC0), (70 + 39, 0, 0xFF80)]        # +inf, NaN, -inf
    for r, h, bits in rows:
        odd.batch.q_prefill[r, h, 17] = bits
    announce("prefill_q8 units, queries that are not finite")
    got, plain = units(odd), units(q8)
    for r, h, _ in rows:
        assert np.isnan(oracle.widen(got[r, h], "bf16")).all()
        got[r, h] = plain[r, h]
    assert np.array_equal(got, plain)
    check(q8, got, "the other rows")


@pytest.mark.parametrize("group,hkv,ring", [(1, 8, False), (2, 8, False), (4, 8, False), (8, 8, False), (1, 8, True), (2, 8, True), (4, 8, True),
                                            (8, 8, True)])
def test_far_blocks(group, hkv, ring):
    # rows beyond 32-bit byte offsets: the variants with 64-bit ones, tables whole in LDS and through its ring
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    nb = 300000
    b = chunks([150, 0], [70, 200], group, hkv, seed=17, cls=[W.RT] * 2)
    q8 = Q.held(b, 17)
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    far = [torch.full((nb,) + x.shape[1:], 0x7F, dtype=torch.uint8, device="cuda") for x in (q8.k, q8.v, q8.scales)]
    for x, y in zip(far, (q8.k, q8.v, q8.scales)):
        x[nb - b.num_blocks:] = up(y)
    tables = wide(b, 2600 if ring else 1900).block_tables
    tables = np.where(tables >= 0, tables + (nb - b.num_blocks), tables).astype(np.int32)
    q = bros._tensor(b.q_prefill, "bf16", "cuda")
    out = torch.full_like(q, 7.0)
    bound = 41000 if ring else 30000
    ws = None
    if ring:
        size = bros.bros_attn_workspace_size(bros.BROS_WS_PREFILL, bros.BROS_BF16, q.shape[0], hkv * group, 128, bound)
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    announce(f"prefill_q8 units in blocks beyond 4 GiB, G={group}, ring={ring}")
    bros.bros_attn_prefill_chunk_q8(out, q, up(b.cu_q), 200, *far, up(tables), up(b.dir), None, up(b.ctx_lens), bound, workspace=ws)
    torch.cuda.synchronize()
    check(q8, bros.to_host_bits(out), f"far blocks, G={group}")


def test_eight_heads_through_the_ring():
    b = chunks([150, 0], [70, 200], 8, 2, seed=18, cls=[W.BE] * 2)
    q8 = Q.poison(Q.held(b, 18), owned_mask(b))
    announce("prefill_q8 units, a ring of table entries, G=8")
    check(q8, run(dataclasses.replace(q8, batch=wide(q8.batch, 2600)), max_ctx=41000), "G=8")
