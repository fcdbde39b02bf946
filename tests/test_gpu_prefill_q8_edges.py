"""bros_attn_prefill_chunk_q8 where values that are not finite meet invalid table
entries, long tables and keys of the future: they reach the rows that see them and no
others, in every arrangement of the work."""

import dataclasses

import numpy as np
import pytest

import oracle
from paper_2504_09590_amd import workload as W
from tests import q8_helpers as Q
from tests.gpu_helpers import announce
from tests.test_gpu_prefill_q8 import chunks, run

pytestmark = pytest.mark.gpu

# Groups of 16 columns, which the rule takes for the calls here, and units of 128 rows, which it takes
# where the longest context may have many blocks: by the table's width and the bound, and no workspace for pieces.
ARRANGEMENTS = ["groups", "units"]


def wide(b, width=1900):
    """The batch with tables of `width` entries, what is behind the contexts' invalid."""
    more = width - b.block_tables.shape[1]
    tables = np.pad(b.block_tables, ((0, 0), (0, more)), constant_values=-1)
    dirs = np.pad(b.dir, ((0, 0), (0, more)), constant_values=-1) if b.dir.ndim == 2 else b.dir
    return dataclasses.replace(b, block_tables=np.ascontiguousarray(tables), dir=np.ascontiguousarray(dirs))


def arranged(q8, how, **kw):
    if how == "groups":
        return run(q8, **kw)
    return run(dataclasses.replace(q8, batch=wide(q8.batch)), with_ws=False, max_ctx=30000, **kw)


def place(b, s, pos):
    """Block and slot of a position of sequence s."""
    blk, slot = oracle.physical_location(b.block_tables, b.dir, s, np.array([pos]))
    return int(blk[0]), int(slot[0])


def spoilt(q8):
    """A copy that values may be planted in."""
    return dataclasses.replace(q8, k=q8.k.copy(), v=q8.v.copy(), scales=q8.scales.copy())


def check_spoilt(got_bits, clean_bits, want, what):
    """Not finite exactly where `want` says, every other output as without the planted values, bit for bit."""
    odd = ~np.isfinite(oracle.widen(got_bits, "bf16"))
    assert (odd == want).all(), f"{what}: {(odd & ~want).sum()} outputs too many, {(want & ~odd).sum()} missing"
    same = want | (got_bits == clean_bits)
    assert same.all(), f"{what}: {(~same).sum()} other outputs changed"


@pytest.mark.parametrize("how", ARRANGEMENTS)
@pytest.mark.parametrize("c0", [200, 4000])
def test_a_nan_beside_an_invalid_entry(c0, how):
    # pairs of blocks whose other block is invalid: far below every row's position, and around it
    n = 60
    b = chunks([c0], [n], 4, 2, seed=c0, cls=[W.RT])
    first = c0 // 16                     # block of the first new row
    tables = b.block_tables.copy()
    tables[0, [1, 8, first + 2]] = [-1, b.num_blocks, -7]
    b = dataclasses.replace(b, block_tables=tables)
    q8 = Q.held(b, 18)
    odd = spoilt(q8)
    want = np.zeros((n, 8, 128), dtype=bool)
    for pos, head, dim in ((5, 1, 7), (9 * 16 + 3, 0, 120), ((first + 3) * 16 + 2, 1, 64)):
        blk, slot = place(b, 0, pos)
        odd.v[blk, head, slot, dim] = 0x7F
        want[max(0, pos - c0):, 4 * head:4 * head + 4, dim] = True
    blk, slot = place(b, 0, 9 * 16 + 7)
    odd.scales[blk, 1, 1, slot] = 255    # a scale that is none: every dim
    odd.v[blk, 1, slot] = 0x38
    want[:, 4:] = True
    announce(f"prefill_q8 NaNs beside invalid entries, {n} rows on {c0}, {how}")
    check_spoilt(arranged(odd, how), arranged(q8, how), want, how)


@pytest.mark.parametrize("group,c0,n", [(1, 16320, 128), (2, 16370, 64)])
def test_a_nan_where_the_table_ring_has_gone_on(group, c0, n):
    # contexts beyond the table's copy in LDS: 514 tiles of 32 keys, of which the last but one step
    # takes in entries for those behind tile 512, in the places of tiles up to 511. With 600
    # empty chunks more there are units enough for the chip, and none is split.
    b = chunks([c0] + [1] * 600, [n] + [0] * 600, group, 1, seed=group, cls=[W.RT] * 601)
    q8 = Q.held(dataclasses.replace(b, block_tables=wide(b, 2600).block_tables), 5)
    odd = spoilt(q8)
    want = np.zeros((n, group, 128), dtype=bool)
    for j, dim in ((3, 9), (13, 70), (40, 101), (n - 2, 33)):
        blk, slot = place(q8.batch, 0, c0 + j)
        odd.v[blk, 0, slot, dim] = 0xFF
        want[j:, :, dim] = True
    announce(f"prefill_q8 NaNs in the new rows, {n} rows on {c0}, G={group}")
    check_spoilt(run(odd, max_ctx=41000), run(q8, max_ctx=41000), want, f"G={group}")


@pytest.mark.parametrize("how", ARRANGEMENTS)
def test_infinite_values_reach_only_rows_that_see_them(how):
    # codes and scales of 2^128 and more, as the append writes them for finite values above 1.9375 * 2^127
    # (scale byte 247, code 256) and as larger scale bytes have them, in keys that some rows do not see
    c0, n = 90, 75
    b = chunks([c0], [n], 4, 2, seed=44, cls=[W.BE])
    q8 = Q.held(b, 44)
    odd = spoilt(q8)
    row = np.zeros(128)
    row[7], row[30] = 3.38e38, -3.38e38
    codes, byte = oracle.encode(row[None])
    assert byte[0] == 247 and codes[0, 7] == 0x78 and codes[0, 30] == 0xF8
    want = np.zeros((n, 8, 128), dtype=bool)
    blk, slot = place(b, 0, c0 + 6)
    odd.v[blk, 0, slot], odd.scales[blk, 0, 1, slot] = codes[0], 247
    want[6:, :4, [7, 30]] = True
    for j, code, by in ((18, 0x70, 248), (41, 0xC0, 254), (70, 0x7E, 250)):
        blk, slot = place(b, 0, c0 + j)
        odd.v[blk, 1, slot] = 0
        odd.v[blk, 1, slot, j] = code
        odd.scales[blk, 1, 1, slot] = by
        want[j:, 4:, j] = True
    announce(f"prefill_q8 infinite values, {how}")
    got, clean = arranged(odd, how), arranged(q8, how)
    # (rows that see a planted key have other values too: only those that see none are compared bit for bit)
    odd_at = ~np.isfinite(oracle.widen(got, "bf16"))
    assert (odd_at == want).all(), f"{(odd_at & ~want).sum()} outputs too many, {(want & ~odd_at).sum()} missing"
    assert (got[:6, :4] == clean[:6, :4]).all() and (got[:18, 4:] == clean[:18, 4:]).all()


@pytest.mark.parametrize("how", ARRANGEMENTS)
def test_equal_weights_sum_to_one(how):
    # Four keys ahead of all others, one in each of the first four pairs of blocks (where a wave's
    # reference maximum comes from), the others equally far behind them, and V one constant: whatever the
    # common weight is rounded to, the output is the constant. The others' weight is 2^-3 (1 + 0.0038),
    # which bf16 rounds down to 2^-3: with some 200 of them, 25 beside 4 in all, numerators of rounded
    # weights over the sum of those that are not are 0.0032 short, 0.0061 at 1.875, more than half a
    # bf16 step there (2^-8).
    # Tolerance: sums in fp32 of at most 209 terms are off by 2 * 209 * 2^-24 = 2.5e-5 of the quotient, far below
    # half a step, so the constant comes out exactly.
    c0, n = 200, 9
    b = chunks([c0], [n], 4, 2, seed=3, cls=[W.RT])
    k, v = np.zeros(b.k_pool.shape), np.full(b.v_pool.shape, 1.875)
    for pos in (2, 34, 66, 98):
        blk, slot = place(b, 0, pos)
        k[blk, :, slot, :2] = 1.0
    (kc, ks), (vc, vs) = oracle.encode(k), oracle.encode(v)
    q = np.zeros(b.q_prefill.shape)
    q[..., 0], q[..., 1] = 23.5, -0.0166
    ahead = (23.5 - 0.0166) / np.sqrt(128) / np.log(2)             # in powers of two
    assert 0.0036 < 2.0 ** (3 - ahead) - 1 < 2.0 ** -8             # the others' weight: a little above 2^-3, less than half a step
    b = dataclasses.replace(b, q_prefill=W._to_bf16_bits(q.astype(np.float32)))
    q8 = Q.Q8Batch(b, kc, vc, np.ascontiguousarray(np.stack([ks, vs], axis=2)))
    announce(f"prefill_q8 equal weights, {how}")
    got = oracle.widen(arranged(q8, how), "bf16")
    assert (got == 1.875).all(), f"off by up to {np.abs(got - 1.875).max()}"


@pytest.mark.parametrize("how", ARRANGEMENTS)
def test_rows_without_a_scale(how):
    # scale byte 255, K's and V's, in a key that all rows see and in keys that some do; codes of one sign, of zero
    c0, n = 100, 50
    b = chunks([c0], [n], 4, 6, seed=45, cls=[W.RT])
    q8 = Q.held(b, 45)
    odd = spoilt(q8)
    want = np.zeros((n, 24, 128), dtype=bool)
    for h, (pos, codes, which) in enumerate(((20, odd.k, 0), (120, odd.k, 0), (21, odd.v, 1), (123, odd.v, 1), (22, odd.v, 1), (130, odd.v, 1))):
        blk, slot = place(b, 0, pos)
        codes[blk, h, slot] = 0x30 if h < 4 else 0
        odd.scales[blk, h, which, slot] = 255
        want[max(0, pos - c0):, 4 * h:4 * h + 4] = True
    announce(f"prefill_q8 rows without a scale, {how}")
    check_spoilt(arranged(odd, how), arranged(q8, how), want, how)
