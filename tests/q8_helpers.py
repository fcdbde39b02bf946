"""Shared pieces of the tests of attention over an 8-bit pool: a batch whose pool
is held in 8 bits, the fp64 attention over the values it stands for, and the
tolerance.

Tolerance per output value y of a head, n keys, vmax the largest |value| of its V:
  2^-8 |y|                      the rounding to bf16
  vmax * 2 d                    scores: 128 products summed in fp32 are off by at most
                                d = 132 * 2^-24 * scale * |q| |k|max (norms), a weight by
                                the factor e^d, numerator and denominator alike
  vmax * w                      the weights' rounding: 2^-16 where a weight is two bf16
                                parts (decode), 2^-7 for one part (prefill: up to half a
                                step, 2^-8, in the weights and again in their sum)
  vmax * (2^-20 + n 2^-27)      exponentials, and sums over n keys in steps of 32 or fewer
"""

import dataclasses

import numpy as np

import oracle
from paper_2504_09590_amd import workload as W


@dataclasses.dataclass
class Q8Batch:
    batch: object          # the batch; its pools hold the (exact, bf16) values of the codes
    k: np.ndarray          # uint8 [nb][Hkv][16][D]
    v: np.ndarray
    scales: np.ndarray     # uint8 [nb][Hkv][2][16]


def held(batch, seed=0, spread=3.0):
    """The batch with its pools held in 8 bits, rows scaled by 2^U(-spread, spread)."""
    rng = np.random.default_rng(seed + 77)
    out = []
    for pool, by in ((batch.k_pool, 0.5), (batch.v_pool, 1.0)):
        x = oracle.widen(pool, batch.dtype) * np.exp2(rng.uniform(-spread, spread, pool.shape[:3] + (1,)) * by)
        codes, scales = oracle.encode(x)
        out.append((codes, scales, W._to_bf16_bits(oracle.decode_rows(codes, scales).astype(np.float32))))
    (k, ks, kb), (v, vs, vb) = out
    b = dataclasses.replace(batch, k_pool=kb, v_pool=vb)
    return Q8Batch(b, k, v, np.ascontiguousarray(np.stack([ks, vs], axis=2)))


def poison(q8, mask):
    """NaN codes and the largest scale byte where mask [nb][16] is False."""
    blocks, slots = np.nonzero(~mask)
    q8.k[blocks, :, slots] = 0x7F
    q8.v[blocks, :, slots] = 0xFF
    q8.scales[blocks, :, :, slots] = 255
    return q8


def check(got_bits, want, q, batch, seq_of_row, w, what, kmax=None, vmax=None, dtype="bf16"):
    """got [rows][Hq][D] as stored against fp64 `want`; q as stored, seq_of_row: each row's sequence.
    dtype "f32": the same tolerance with a rounding of 2^-24 at the end."""
    got = oracle.widen(got_bits, dtype)
    assert np.isfinite(got).all(), f"{what}: not finite"
    qn = np.linalg.norm(oracle.widen(q, dtype), axis=-1)                      # [rows][Hq]
    hq, hkv = qn.shape[1], batch.num_kv_heads
    if kmax is None:
        kmax, vmax = np.zeros((batch.num_seqs, hkv)), np.zeros((batch.num_seqs, hkv))
        for s in range(batch.num_seqs):
            n = min(int(batch.ctx_lens[s]), batch.block_tables.shape[1] * 16)
            tab = np.where((batch.block_tables >= 0) & (batch.block_tables < batch.num_blocks), batch.block_tables, 0)
            if n > 0:
                kmax[s] = np.linalg.norm(oracle.widen(oracle.gather_kv(batch.k_pool, tab, batch.dir, s, n), dtype), axis=-1).max(0)
                vmax[s] = np.abs(oracle.widen(oracle.gather_kv(batch.v_pool, tab, batch.dir, s, n), dtype)).max((0, 2))
    group = np.arange(hq) // (hq // hkv)
    k_row, v_row = kmax[seq_of_row][:, group], vmax[seq_of_row][:, group]
    n = np.maximum(batch.ctx_lens[seq_of_row], 0)[:, None]
    d = 132 * 2.0 ** -24 * qn * k_row / np.sqrt(batch.head_dim)
    tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want) + (v_row * (2 * d + w + 2.0 ** -20 + n * 2.0 ** -27))[..., None]
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.abs(got - want)[bad].max():.3g}"
