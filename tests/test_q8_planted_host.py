"""The long contexts of the 8-bit prefill's tests show a lost tile: their check turns down the
attention with any one tile of 32 cached keys left out (no GPU)."""

import numpy as np
import pytest

import oracle
from paper_2504_09590_amd import workload as W
from tests import q8_helpers as Q
from tests.q8_planted import cached, planted, without_a_tile
from tests.test_gpu_prefill_q8_long import CASES, WEIGHTS, batch


def largest(b, s):
    """Q.check's largest norms of K and values of V, of sequence s (it looks for all sequences' in every call otherwise)."""
    kmax, vmax = np.zeros((b.num_seqs, b.num_kv_heads)), np.zeros((b.num_seqs, b.num_kv_heads))
    k, v = (oracle.widen(oracle.gather_kv(p, b.block_tables, b.dir, s, int(b.ctx_lens[s])), "bf16") for p in (b.k_pool, b.v_pool))
    kmax[s], vmax[s] = np.linalg.norm(k, axis=-1).max(0), np.abs(v).max((0, 2))
    return kmax, vmax


@pytest.mark.parametrize("name", CASES)
def test_every_tile_is_seen(name):
    group, hkv, c0s, ns = CASES[name]
    b = batch(name)
    q8 = planted(b, 1)
    b = q8.batch
    want = oracle.prefill_chunk(b.q_prefill, b.cu_q, b.k_pool, b.v_pool, b.block_tables, b.dir, b.ctx_lens, "bf16")
    seq = np.repeat(np.arange(b.num_prefill), np.diff(b.cu_q))
    stored = lambda x: W._to_bf16_bits(x.astype(np.float32))  # noqa: E731
    Q.check(stored(want), want, b.q_prefill, b, seq, WEIGHTS, "the attention itself")
    tiles = 0
    for s in range(b.num_prefill):
        n, c0 = cached(b, s)
        if c0 < 900 or n == 0:
            continue
        most = largest(b, s)
        for g in {0, hkv - 1}:
            for row, head, out in without_a_tile(q8, s, g, want):
                got = want[row:row + 1].copy()
                got[0, head] = out
                with pytest.raises(AssertionError, match="off"):
                    Q.check(stored(got), want[row:row + 1], b.q_prefill[row:row + 1], b, seq[row:row + 1], WEIGHTS, name, *most)
                tiles += 1
    assert tiles >= min(hkv, 2) * (max(c0s) // 32)
