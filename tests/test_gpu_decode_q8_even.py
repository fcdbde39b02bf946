"""The even split of bros_attn_decode_q8 for every number of query heads to a KV head and of KV
heads side by side (1, 2, 4), and single waves for two heads. A loose bound over wide tables
takes the calls to the even split. And in every arrangement: a NaN stays in its row and head."""

import dataclasses

import numpy as np
import pytest

import oracle
from paper_2504_09590_amd import workload as W
from tests import q8_helpers as Q
from tests.gpu_helpers import announce, owned_mask, with_direction_table
from tests.test_gpu_decode_q8 import WEIGHTS, check, masked_reference, run
from tests.test_gpu_prefill_q8_edges import check_spoilt, wide

pytestmark = pytest.mark.gpu

BOUND = 30000


def even(q8, **kw):
    return run(dataclasses.replace(q8, batch=wide(q8.batch)), max_ctx=BOUND, **kw)


@pytest.mark.parametrize("hkv", [3, 2, 4])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_groups_and_heads(group, hkv):
    rng = np.random.default_rng(10 * group + hkv)
    ctx = rng.integers(1, 400, 70)
    ctx[:12] = 1, 15, 16, 17, 31, 32, 33, 64, 65, 3000, 1, 2500
    b = W.custom(ctx, (rng.random(70) < 0.5).astype(np.uint8), hkv * group, hkv, seed=group, spare_blocks=5)
    q8 = Q.poison(Q.held(b, group), owned_mask(b))
    announce(f"decode_q8 even split, G={group} Hkv={hkv}")
    one, two = even(q8, repeat=2)
    assert np.array_equal(one, two)
    check(q8, one, f"G={group} Hkv={hkv}")


@pytest.mark.parametrize("group,hkv", [(1, 2), (8, 1)])
def test_empty_contexts_and_invalid_entries(group, hkv):
    rng = np.random.default_rng(group)
    ctx = rng.integers(1, 700, 130)
    b = with_direction_table(W.custom(ctx, (rng.random(130) < 0.5).astype(np.uint8), hkv * group, hkv, seed=3, spare_blocks=5))
    q8 = Q.poison(Q.held(b, 3), owned_mask(b))
    b = q8.batch
    empty = np.array([0, 1, 64, 129])
    b.ctx_lens[empty] = 0, -5, 0, 0
    gone = np.array([2, 50, 128])
    b.block_tables[gone, 0] = b.num_blocks + 3, -1, 2 ** 31 - 1
    announce(f"decode_q8 even split, empty contexts and invalid entries, G={group} Hkv={hkv}")
    got = even(q8)
    assert (got[empty] == 0).all()
    Q.check(got, masked_reference(q8, b.block_tables), b.q_decode, b, np.arange(130), WEIGHTS, f"G={group}")


def test_single_waves_of_two_heads():
    rng = np.random.default_rng(2)
    ctx = rng.integers(1, 120, 130)
    b = W.custom(ctx, (rng.random(130) < 0.5).astype(np.uint8), 16, 8, seed=4, spare_blocks=5)
    q8 = Q.poison(Q.held(b, 4), owned_mask(b))
    announce("decode_q8 by single waves, G=2")
    check(q8, run(q8), "G=2")


@pytest.mark.parametrize("how", ["whole", "pieces", "waves", "even"])
def test_a_nan_stays_in_its_row_and_head(how):
    rng = np.random.default_rng(6)
    rows, hi = {"whole": (20, 300), "pieces": (4, 3000), "waves": (130, 100), "even": (130, 400)}[how]
    ctx = rng.integers(hi // 3, hi + 1, rows)
    b = W.custom(ctx, [W.RT] * rows, 32, 8, seed=5, spare_blocks=5, share_tails=False)
    q8 = Q.held(b, 5)
    odd = dataclasses.replace(q8, k=q8.k.copy(), v=q8.v.copy(), scales=q8.scales.copy())
    want = np.zeros((rows, 32, 128), dtype=bool)
    for row, h, what in ((1, 0, "value"), (1, 7, "key"), (2, 3, "scale"), (rows - 1, 5, "value"), (rows - 1, 2, "key scale"),
                         (0, 6, "scale of zeros")):
        pos = int(ctx[row]) // 2
        blk, slot = oracle.physical_location(b.block_tables, b.dir, row, np.array([pos]))
        dims = slice(None)
        if what == "value":
            dims = 99
            odd.v[blk, h, slot, dims] = 0x7F
        elif what == "key":
            odd.k[blk, h, slot, 3] = 0xFF
        elif what.startswith("scale"):
            odd.v[blk, h, slot] = 0x30 if what == "scale" else 0
            odd.scales[blk, h, 1, slot] = 255
        else:
            odd.k[blk, h, slot] = 0x30
            odd.scales[blk, h, 0, slot] = 255
        want[row, 4 * h:4 * h + 4, dims] = True
    announce(f"decode_q8 NaNs, {how}")
    go = even if how == "even" else run
    check_spoilt(go(odd), go(q8), want, how)
