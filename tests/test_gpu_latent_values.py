"""The expanded form over values of any size: a head's small or large values, tiles and rows of different sizes, and
queries that put their weight on any of them.

Half of the latent dims make the keys and half the values, so that a position's values have any size without a change of
its scores; the rotated dims add to a position's score."""

import numpy as np
import pytest

from tests.gpu_helpers import announce, require_gpu
from tests.rows_helpers import check, visible
from tests.test_gpu_latent import LATENT, SCALE, Chunks, latent_rows

pytestmark = pytest.mark.gpu
NARROW = ([70, 33], [200, 0])                  # units of 64 rows, whole
WIDE = ([70, 33], [1200, 90])                  # of 128 rows, cut
SHAPES = [NARROW, WIDE]


class Values(Chunks):
    """sizes: of sequence s and its positions, the exponent of two that its values are multiplied by; raise_: what is added
    to its scores (natural units, times `lift`, one for each row's query)."""

    def __init__(self, n, c0, hq, sizes, raised=None, seed=0, directions="table"):
        import torch
        super().__init__(n, c0, hq, seed, directions)
        self.w[:, :128, LATENT // 2:] = 0
        self.w[:, 128:, :LATENT // 2] = 0
        rng = np.random.default_rng(seed)
        for s in range(self.b.S):
            if self.b.ctx[s] == 0:
                continue
            pos = np.arange(self.b.ctx[s])
            blk, slot = self.b.places(s, pos)
            rows = self.pool[blk, slot].float()
            rows[:, LATENT // 2:LATENT] *= torch.from_numpy(2.0 ** np.broadcast_to(sizes(s, pos, rng), pos.shape).astype(np.float64)).float()[:, None]
            if raised is not None:             # one rotated dim: 8 of the query's against the rest of the key's
                self.q[int(self.b.cu[s]):int(self.b.cu[s + 1]), :, 128:] = 0
                self.q[int(self.b.cu[s]):int(self.b.cu[s + 1]), :, 130] = 8.0
                rows[:, LATENT:] = 0
                rows[:, LATENT + 2] = torch.from_numpy(np.broadcast_to(raised(s, pos, rng), pos.shape).astype(np.float32)) / (8 * SCALE)
            self.pool[blk, slot] = rows.bfloat16()

    def steps(self):
        """How far halves may be off where few bits are left of them (kernel and definition differ by at most the first of these in
        tiles of 32 positions that stand behind exponents, by the second in the others).

        Behind exponents each tile's products are made of weights w' <= 1 and values v' <= 2^14 in halves, of which the largest
        w' |v'| of the seen keys is 2^13 at least: a weight that is rounded to steps of 2^-24 is off by 2^-25 at most, its
        product by 2^-24 of that largest one, the 32 of a tile by 2^-19. So 2^-19 of the sum over all keys of weight times the
        largest magnitude among the key's values; as much again for the values' own steps.

        A tile is stored as it is where each row's largest magnitude is zero or 2^-6 .. 2^5 (a per cent aside, for that
        magnitude's own roundings). Tiles like that next to each other may share a largest weight, that of one of their keys: 2^-25
        of it for each seen key times the key's value."""
        import torch
        b = self.b
        out = torch.zeros((b.rows, self.hq, 128), dtype=torch.float64)
        for s in range(b.S):
            lo, hi = int(b.cu[s]), int(b.cu[s + 1])
            if hi == lo:
                continue
            see = torch.from_numpy(visible(b, s, None))
            c = latent_rows(b, self.pool, s, see.numpy())
            for h in range(self.hq):
                w, q = self.w[h].double(), self.q[lo:hi, h].double()
                kv = c[:, :LATENT] @ w.t()
                k, v = torch.cat([kv[:, :128], c[:, LATENT:]], 1), kv[:, 128:].abs()
                p = ((q @ k.t()) * SCALE).masked_fill(~see, -np.inf).softmax(1).nan_to_num(0.0)
                most = v.amax(1)
                out[lo:hi, h] = (p @ most[:, None]) * 2.0 ** -18
                as_is = ((most == 0) | (most >= 0.99 * 2.0 ** -6) & (most < 1.01 * 2.0 ** 5)).numpy()
                tiles = [as_is[i:i + 32].all() for i in range(0, len(as_is), 32)]
                i = 0
                while i < len(tiles):
                    n = next((x for x in range(i, len(tiles)) if not tiles[x]), len(tiles))
                    if n > i:
                        run = slice(32 * i, 32 * n)
                        out[lo:hi, h] += 2.0 ** -25 * p[:, run].amax(1, keepdim=True) * (see[:, run].double() @ v[run])
                    i = n + 1
        return out

    def compare(self, what, **kw):
        import torch
        announce(what)
        got = self.run(**kw)
        want, tol = self.want()
        check(got, want, tol + self.steps(), what)
        # (row by row and head by head: roundings are independent, and their sum stays near 2^-8 of a row)
        off, size = (got.double().cpu() - want).norm(dim=-1), want.norm(dim=-1)
        assert (off <= 2.0 ** -7 * size).all(), f"{what}: {float((off / size.clamp(min=1e-300)).max()):.3g} of a row"
        assert torch.equal(got, self.run(**kw))
        return got


@pytest.mark.parametrize("shape", SHAPES, ids=["narrow", "wide"])
@pytest.mark.parametrize("size", [-100, -20, -9, -8, -7.7, -7.5, -7.3, -7, -6, 3, 4, 5, 14, 16, 100])
def test_all_of_one_size(shape, size):
    """Among them sizes near which some rows' values lie within what halves hold as they are, and others do not."""
    require_gpu()
    Values(*shape, 2, lambda s, pos, rng: size, seed=3).compare(f"latent values of 2^{size}")


@pytest.mark.parametrize("shape", SHAPES, ids=["narrow", "wide"])
@pytest.mark.parametrize("spread", [3, 12, 30, 60])
def test_any_size_in_any_row(shape, spread):
    require_gpu()
    Values(*shape, 2, lambda s, pos, rng: rng.uniform(-spread, spread, pos.shape), seed=4).compare(f"latent values spread over 2^{spread}")


@pytest.mark.parametrize("shape", SHAPES, ids=["narrow", "wide"])
@pytest.mark.parametrize("first,then", [(0, -9), (0, -20), (0, -60), (12, -5), (20, -20), (40, 0), (-20, 20)])
@pytest.mark.parametrize("raised", [False, True])
def test_small_values_behind_large_ones(shape, first, then, raised):
    """The first two tiles are of one size, the others of another, on which the queries put nearly all of their weight or
    not: 2^-43 of it stays on the first."""
    require_gpu()
    Values(*shape, 2, lambda s, pos, rng: np.where(pos < 64, first, then), (lambda s, pos, rng: np.where(pos < 64, -30.0, 0.0)) if raised else None,
           seed=5).compare(f"latent values of 2^{first}, then 2^{then}, raised {raised}")


@pytest.mark.parametrize("shape", SHAPES, ids=["narrow", "wide"])
@pytest.mark.parametrize("size", [-9, -20, 0])
def test_zeros_and_missing_blocks_before_small_values(shape, size):
    """Tiles of zeros and without context have no size of their own."""
    require_gpu()
    n, c0 = [70, 33, 40], [*shape[1], 300]
    c = Values(n, c0, 2, lambda s, pos, rng: np.where((pos >= 32) & (pos < 64) | (pos % 7 == 3), -np.inf, size), seed=6)
    c.b.tables[0, [0, 1, 7]] = [-1, c.b.num_blocks, -5]
    c.b.tables[2, 0:4] = -1
    c.compare(f"latent values of 2^{size} behind zeros")


@pytest.mark.parametrize("shape", SHAPES, ids=["narrow", "wide"])
@pytest.mark.parametrize("size", [20, 40, 100])
def test_a_row_of_another_size(shape, size):
    """One row's values are 2^20 times the others' and more. The rows before it, in its tile and others, are as near to the
    definition as without it; those behind it see it, with the weight that it has or with next to none."""
    require_gpu()
    for raised in (None, lambda s, pos, rng: np.where(pos == shape[1][s] + 20, -60.0, 0.0)):
        Values(*shape, 2, lambda s, pos, rng: np.where(pos == shape[1][s] + 20, size, 0), raised, seed=7).compare(f"latent values, one of 2^{size}")


def test_heads_and_sequences_of_different_sizes():
    """Chunks in teams, in passes: a head's and a sequence's sizes are its own."""
    require_gpu()
    c = Values([700, 1, 130], [900, 1024, 1500], 3, lambda s, pos, rng: (0, -30, 12)[s] - (pos > 800) * 9, seed=8)
    c.w[1, 128:] = (c.w[1, 128:].float() * 2.0 ** -8).bfloat16()
    c.w[2, 128:] = (c.w[2, 128:].float() * 2.0 ** 20).bfloat16()
    c.compare("latent values of different sizes")
    c.compare("latent values of different sizes, a head a pass", heads=1)
