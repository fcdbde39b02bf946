"""bros_attn_prefill_chunk_q8 over long contexts of which every tile counts (q8_planted.py):
pieces of groups of 16 columns, units of 128 rows in pieces and whole, and tables that run through the
ring in LDS, refills among them."""

import dataclasses

import numpy as np
import pytest

from paper_2504_09590_amd import workload as W
from tests import q8_helpers as Q
from tests.gpu_helpers import announce, owned_mask
from tests.q8_planted import planted
from tests.test_gpu_prefill_q8 import WEIGHTS, check, chunks, run
from tests.test_gpu_prefill_q8_edges import wide

# name: heads to a KV head, KV heads, cached tokens and new rows of the chunks
CASES = {
    "groups-4": (4, 2, [4000, 30, 900], [20, 3, 9]),
    "groups-8": (8, 1, [9000], [9]),
    "groups-1": (1, 8, [1500, 0], [16, 7]),
    "groups-2": (2, 3, [20000, 5], [32, 33]),
    "units-4": (4, 2, [9000, 0, 7], [200, 64, 1]),
    "units-1": (1, 8, [9000, 0], [200, 64]),
    "units-8": (8, 1, [9000, 7], [200, 1]),
    "ring": (4, 2, [40000, 100], [70, 30]),
}


def batch(name):
    group, hkv, c0s, ns = CASES[name]
    return chunks(c0s, ns, group, hkv, seed=len(name), cls=[W.RT, W.BE, W.RT][:len(ns)])


def poisoned(name):
    b = batch(name)
    return Q.poison(planted(b, 1), owned_mask(b))


def with_empty_chunks(b, more=600):
    """The batch with `more` chunks of no rows behind it: units enough for the chip, so that none is split."""
    pad = lambda x: np.concatenate([x, np.full(more, x[-1], dtype=x.dtype)])  # noqa: E731
    return dataclasses.replace(b, block_tables=np.concatenate([b.block_tables, np.full((more, b.block_tables.shape[1]), -1, np.int32)]),
                               dir=pad(b.dir), cls=pad(b.cls), ctx_lens=np.concatenate([b.ctx_lens, np.ones(more, np.int32)]),
                               cu_q=pad(b.cu_q))


@pytest.mark.gpu
@pytest.mark.parametrize("name", [n for n in CASES if n.startswith("groups")])
def test_groups_of_columns_in_pieces(name):
    q8 = poisoned(name)
    announce(f"prefill_q8 long contexts, {name}")
    check(q8, run(q8), name)


@pytest.mark.gpu
@pytest.mark.parametrize("name", [n for n in CASES if n.startswith("units")])
def test_units_in_pieces_and_whole(name):
    q8 = poisoned(name)
    loose = dataclasses.replace(q8, batch=wide(q8.batch))
    announce(f"prefill_q8 long contexts, {name}")
    split, whole = run(loose, max_ctx=30000), run(loose, max_ctx=30000, with_ws=False)
    check(q8, split, f"{name} in pieces")
    check(q8, whole, f"{name} whole")
    assert not np.array_equal(split, whole)


@pytest.mark.gpu
def test_tables_beyond_lds():
    q8 = poisoned("ring")
    announce("prefill_q8 long contexts, a ring of table entries, in pieces")
    split = run(q8)
    check(q8, split, "in pieces")
    # whole units: 1253 tiles, entries refilled at 512 and 1024
    announce("prefill_q8 long contexts, a ring of table entries, whole")
    whole = run(dataclasses.replace(q8, batch=with_empty_chunks(q8.batch)))
    check(q8, whole, "whole")
    assert not np.array_equal(split, whole)
