"""Long contexts of which every tile counts. Over thousands of like keys an output is
small against the tolerance, and a tile of 32 keys lost in it cannot be seen. Here each
tile of cached keys holds one key that is some query's own direction, with a score of
about 25: a query's softmax rests on a few such keys (exp(25) against the sum of the
others, exp(ln 40000 + 0.5)), so a tile that is lost, or read from another block, moves an
output by a tenth of |v| at least where a query has up to ten of them."""

import dataclasses

import numpy as np

import oracle
from paper_2504_09590_amd import workload as W
from tests import q8_helpers as Q

SCORE = 25.0
TILE = 32


def owners(b, s):
    """[tiles]: per tile of sequence s's cached positions its query, as (row of the chunk) * G + head of the group."""
    n, c0 = cached(b, s)
    group = b.num_q_heads // b.num_kv_heads
    return np.arange((c0 + TILE - 1) // TILE) % (n * group) if n else np.zeros(0, dtype=int)


def cached(b, s):
    n = int(b.cu_q[s + 1] - b.cu_q[s])
    return n, int(b.ctx_lens[s]) - n


def planted(b, seed):
    """The batch in 8 bits with such keys in every sequence and KV head."""
    k = oracle.widen(b.k_pool, "bf16").copy()
    q = oracle.widen(b.q_prefill, "bf16")
    group = b.num_q_heads // b.num_kv_heads
    for s in range(b.num_prefill):
        n, c0 = cached(b, s)
        own = owners(b, s)
        tile = np.arange(len(own))
        pos = np.minimum(tile * TILE + tile * 7 % TILE, c0 - 1)
        if len(own) == 0:
            continue
        blk, slot = oracle.physical_location(b.block_tables, b.dir, s, pos)
        for g in range(b.num_kv_heads):
            x = q[b.cu_q[s] + own // group, g * group + own % group]
            k[blk, g, slot] = x * (SCORE * np.sqrt(128) / (x * x).sum(-1, keepdims=True))
    return Q.held(dataclasses.replace(b, k_pool=W._to_bf16_bits(k.astype(np.float32))), seed, spread=0.0)


def without_a_tile(q8, s, g, want):
    """For each tile of sequence s's cached positions its owner's row of `want`, its head, and that output with
    the tile's keys left out: (row, head, output)."""
    b = q8.batch
    n, c0 = cached(b, s)
    group = b.num_q_heads // b.num_kv_heads
    ctx = c0 + n
    k, v = (oracle.widen(oracle.gather_kv(p, b.block_tables, b.dir, s, ctx), "bf16")[:, g] for p in (b.k_pool, b.v_pool))
    own = owners(b, s)
    for query in np.unique(own):
        row, head = int(b.cu_q[s]) + query // group, g * group + query % group
        last = c0 + query // group + 1
        score = k[:last] @ oracle.widen(b.q_prefill[row, head], "bf16") / np.sqrt(128)
        w = np.exp(score - score.max())
        total, out = w.sum(), want[row, head]
        for t in np.nonzero(own == query)[0]:
            at = slice(t * TILE, min(t * TILE + TILE, last))
            yield row, head, (out * total - w[at] @ v[at]) / (total - w[at].sum())
