"""Batches of new rows over a paged cache, and their attention in 64 bits (plain NumPy and torch
on the CPU, from the definition), for the tests of drafts and of the latent cache."""

from __future__ import annotations

import numpy as np
import torch

BLOCK = 16


class Rows:
    """Tables, directions and lengths of sequences with n new rows behind c0 tokens each."""

    def __init__(self, n, c0, seed=0, directions="sequence", spare=3, num_blocks=None, skip=()):
        self.n, self.c0 = np.asarray(n, dtype=np.int64), np.asarray(c0, dtype=np.int64)
        rng = np.random.default_rng(seed)
        self.S, self.ctx = len(self.n), self.n + self.c0
        need = (self.ctx + BLOCK - 1) // BLOCK
        self.num_blocks = int(need.sum()) + spare if num_blocks is None else num_blocks
        ids = rng.permutation(self.num_blocks).astype(np.int32) if num_blocks is None else \
            rng.choice(num_blocks - 1, int(need.sum()), replace=False).astype(np.int32) + 1
        self.tables = np.full((self.S, max(1, int(need.max()))), -1, dtype=np.int32)
        at = 0
        for s, m in enumerate(need):
            self.tables[s, :m] = ids[at:at + m]
            at += m
        self.dir = np.where(rng.random(self.S) < 0.5, 1, -1).astype(np.int8)
        if directions == "table":
            self.dir = np.where(rng.random(self.tables.shape) < 0.5, 1, -1).astype(np.int8)
        self.cu = np.concatenate([[0], np.cumsum(self.n)]).astype(np.int32)
        self.rows, self.max_ctx, self.max_n = int(self.cu[-1]), int(self.ctx.max()), int(self.n.max())

    def places(self, s, pos):
        """(blocks, slots) of positions of sequence s."""
        pos = np.asarray(pos)
        e = pos // BLOCK
        d = self.dir[s, e] if self.dir.ndim == 2 else np.full(pos.shape, self.dir[s])
        return self.tables[s, e].astype(np.int64), np.where(d > 0, pos % BLOCK, BLOCK - 1 - pos % BLOCK)

    def owned(self):
        mask = np.zeros((self.num_blocks, BLOCK), dtype=bool)
        for s in range(self.S):
            if self.ctx[s]:
                mask[self.places(s, np.arange(self.ctx[s]))] = True
        return mask

    def cuda(self):
        up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
        return up(self.tables), up(self.dir), up(self.ctx.astype(np.int32)), up(self.cu)


def bf16(rng, shape, gain=1.0):
    return torch.from_numpy((rng.standard_normal(shape, dtype=np.float32) * gain)).bfloat16()


def tree_bits(rng, n, words):
    """Rows of bits of a random tree for each sequence: a draft sees itself and its ancestors."""
    out = []
    for m in n:
        seen = []
        for j in range(m):
            up = int(rng.integers(-1, j)) if j else -1
            seen.append((1 << j) | (seen[up] if up >= 0 else 0))
        out += seen
    return pack(out, words)


def pack(rows, words):
    """Python integers to int64 [rows][words]."""
    a = np.array([[(x >> (64 * w)) & ((1 << 64) - 1) for w in range(words)] for x in rows], dtype=np.uint64)
    return a.reshape(len(rows), words).view(np.int64)


def visible(b: Rows, s, bits, max_ctx=None):
    """[n][ctx] truth values: what each row of sequence s sees (bits None: causal)."""
    n, ctx, c0 = int(b.n[s]), int(b.ctx[s]), int(b.c0[s])
    see = np.zeros((n, ctx), dtype=bool)
    for j in range(n):
        see[j, :c0] = True
        if bits is None:
            see[j, :c0 + j + 1] = True
        else:
            word = sum((int(w) & ((1 << 64) - 1)) << (64 * i) for i, w in enumerate(bits[int(b.cu[s]) + j]))
            see[j, c0:] = [bool((word >> i) & 1) for i in range(n)]
    if max_ctx is not None:
        see[:, max_ctx:] = False
    bad = b.tables[s, np.arange(ctx) // BLOCK]
    see[:, (bad < 0) | (bad >= b.num_blocks)] = False
    return see


def attention(q, k, v, see, scale, key_error=None):
    """q [rows][dk], k [keys][dk], v [keys][dv] in fp64; see [rows][keys]. Gives the result and, for each
    value, how far a kernel may be off that rounds softmax weights and outputs to bf16 (2^-8 of
    a value at most each) and computes the rest in 32 bits:

    - weights w_i (1 + d_i), |d_i| <= 2^-8, over their own sum: 2 * 2^-8 / (1 - 2^-8) of A = sum w |v|;
    - a score's error e (products exact in 32 bits, dk of them added, each addition off by 2^-24 of the sum
      of magnitudes; the argument's rounding and the exponential's, 2^-22 of the score and of one)
      changes each weight by at most e^(2 e) - 1 of it: 2.1 e of A for e < 0.05;
    - the output's rounding, 2^-8 of it, and the sums' over the keys, 2^-24 of A each.
    key_error: the score's error from rounded keys, per row, to be added to e."""
    w = (q @ k.t()) * scale
    big = (q.abs() @ k.abs().t()) * scale
    see = torch.from_numpy(see)
    w = w.masked_fill(~see, -np.inf)
    e = (q.shape[1] + 4) * 2.0 ** -24 * big.masked_fill(~see, 0).amax(1) + 2.0 ** -22 * (1 + w.abs().masked_fill(~see, 0).amax(1))
    if key_error is not None:
        e = e + key_error.masked_fill(~see, 0).amax(1)
    none = ~see.any(1)
    w = torch.where(none[:, None], torch.zeros_like(w), w.softmax(1))
    y, A = w @ v, w @ v.abs()
    tol = A * (2.02 * 2.0 ** -8 + 2.1 * e[:, None] + k.shape[0] * 2.0 ** -23) + 2.0 ** -8 * y.abs() * 1.01
    return y, tol


def check(got, want, tol, what):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    off = (got - want).abs() - tol
    assert (off <= 0).all(), f"{what}: {int((off > 0).sum())} of {off.numel()} values beyond, most {float(off.max()):.3g} over {float(tol.max()):.3g}"


# Shapes that take each way of running the attention of few rows on a card of 256 compute units (index of the way,
# narrowest units first): drafts (n, c0, hq, hkv) over a K/V pool, rows (n, c0, hq) over a latent pool.
WAYS_TREE = [(0, [6] * 3, [480, 17, 300], 8, 2), (0, [2] * 150, [240] * 150, 8, 2), (0, [20], [2000], 8, 2), (1, [16] * 8, [4000] * 8, 16, 4), (2, [30] * 16, [8000] * 16, 16, 4)]
WAYS_LATENT = [(0, [1] * 2, [600] * 2, 64), (1, [1] * 8, [5000] * 8, 64), (2, [2] * 40, [4000] * 40, 32), (3, [1] * 90, [4000] * 90, 128)]
# Shapes whose units of 128 columns stand side by side in teams (workgroups of a team; the rest as above, chunks of a
# latent cache as (n, c0, heads)).
TEAMS_TREE = [(4, [64] * 3, [9000, 12000, 700], 64, 8), (4, [128] * 100, [250] * 100, 16, 4), (2, [64, 50, 41, 60] * 6, [4000, 900, 6000, 33] * 6, 16, 4),
              (2, [150, 0, 160], [9000, 5, 8000], 32, 8)]
TEAMS_CHUNKS = [(4, [512, 512], [1000, 1300], 2), (4, [1024], [1100], 3), (2, [256, 250], [1500, 40], 3), (2, [700, 600, 1], [900, 1100, 1024], 2),
                (2, [641], [2000], 2)]
