"""Shared pieces of the append tests: a seeded batch of projected rows, the call,
and the check of everything it wrote against the fp64 oracle.

Tolerance, relative to |a| + |b| of a value's normed pair: the sum of 128 squares in
fp32 (16 fused steps, 3 exchanges) is off by at most 20 half steps of 2^-24, its
root by half of that, the reciprocal root by 4 more; the product with the factor and
with the weight add 2, the rotation's product and fused sum 2: at most 18 in all.
32 * 2^-24 is allowed. A result of bf16 adds its own rounding, 2^-8 of the value; a
row in 8 bits half an e4m3 step, 2^-4 of the value or 2^-10 of the scale.
"""

import dataclasses

import numpy as np

import oracle
from paper_2504_09590_amd import workload as W

ARITH = 32 * 2.0 ** -24
OWN = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@dataclasses.dataclass
class Rows:
    batch: object
    dtype: str
    q: np.ndarray            # [Tn][Hq][D] as stored (bf16: bit patterns), like k and v
    k: np.ndarray
    v: np.ndarray
    q_norm: object = None    # [D] as stored, or None
    k_norm: object = None
    eps: float = 1e-6
    table: object = None     # float32 [rows][R], or None
    adjacent: bool = False
    sections: object = None
    pos: object = None       # int32 [axes][Tn], or None


def _store(x, dtype):
    x = np.ascontiguousarray(x, dtype=np.float32)
    return x if dtype == "f32" else W._to_bf16_bits(x)


def make_table(rows, rotary, seed=0):
    """Cosines and sines of seeded angles (any table will do; these are unit pairs)."""
    angles = np.random.default_rng(seed).uniform(-np.pi, np.pi, (rows, rotary // 2))
    return np.concatenate([np.cos(angles), np.sin(angles)], axis=1).astype(np.float32)


def make_rows(batch, hq, dtype="bf16", q_norm=False, k_norm=False, rotary=0, adjacent=False, sections=None, seed=0):
    rng = np.random.default_rng(seed + 1000)
    tn, hkv, d = int(batch.cu_new[-1]), batch.num_kv_heads, batch.head_dim
    size = np.exp2(rng.uniform(-3, 3, (tn, 1, 1)))
    r = Rows(batch, dtype, *(_store(rng.standard_normal((tn, h, d)) * size, dtype) for h in (hq, hkv, hkv)))
    if q_norm:
        r.q_norm = _store(rng.uniform(0.5, 1.5, d), dtype)
    if k_norm:
        r.k_norm = _store(rng.uniform(0.5, 1.5, d), dtype)
    if rotary:
        last = int(batch.ctx_lens.max()) if len(batch.ctx_lens) else 1
        r.table, r.adjacent, r.sections = make_table(last + 3, rotary, seed), adjacent, sections
        if sections is not None:
            r.pos = rng.integers(0, last + 3, (len(sections), tn)).astype(np.int32)
    return r


def tokens(batch):
    """(sequence, logical position) of every new token."""
    cu = batch.cu_new.astype(np.int64)
    seq = np.repeat(np.arange(batch.num_seqs), np.diff(cu))
    return seq, np.arange(cu[-1]) - cu[seq] + batch.pos0[seq]


def expected(r, seq, pos):
    """((q, |a|+|b| of its pairs), (k, ...)) in float64 for tokens at logical positions pos."""
    out = []
    for x, w in ((r.q, r.q_norm), (r.k, r.k_norm)):
        n = oracle.widen(x, r.dtype)
        if w is not None:
            n = oracle.norm(n, oracle.widen(w, r.dtype), r.eps)
        reach = np.abs(n)
        y = n
        if r.table is not None:
            half = r.table.shape[1] // 2
            if r.pos is None:
                at = np.repeat(pos[:, None], half, axis=1)
            else:
                at = np.repeat(r.pos, r.sections if r.sections is not None else [half], axis=0).T
            y = oracle.rotate(n, at, r.table, r.adjacent)
            i = np.arange(half)
            a, b = (2 * i, 2 * i + 1) if r.adjacent else (i, i + half)
            both = reach[..., a] + reach[..., b]
            reach = reach.copy()
            reach[..., a] = both
            reach[..., b] = both
        out.append((y, reach))
    return out


def device_rows(r, packed=True):
    """(q, k, v) device tensors, views of one projection's rows when packed."""
    import torch
    from paper_2504_09590_amd import bros
    q, k, v = (bros._tensor(x, r.dtype, "cuda") for x in (r.q, r.k, r.v))
    if not packed:
        return q, k, v
    hq, hkv = q.shape[1], k.shape[1]
    qkv = torch.cat([q, k, v], dim=1).contiguous()
    return qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]


def options(r):
    from paper_2504_09590_amd import bros
    up = lambda x: None if x is None else bros._tensor(x, r.dtype, "cuda")  # noqa: E731
    kw = {}
    if r.q_norm is not None or r.k_norm is not None:
        kw["norm"] = bros.QkNorm(up(r.q_norm), up(r.k_norm), r.eps)
    if r.table is not None:
        kw["rope"] = bros.Rope(bros._tensor(r.table, None, "cuda"), bros.BROS_ROPE_ADJACENT if r.adjacent else
                               bros.BROS_ROPE_HALF, r.sections)
        if r.pos is not None:
            kw["rope_pos"] = bros._tensor(r.pos, None, "cuda")
    return kw


def check_close(got, want, reach, dtype, what, tokens_live=None):
    g = oracle.widen(got, dtype)
    tol = OWN[dtype] * np.abs(want) + ARITH * reach
    if tokens_live is not None:
        g, want, tol = g[tokens_live], want[tokens_live], tol[tokens_live]
    bad = ~(np.abs(g - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} values off, worst {np.abs(g - want)[bad].max():.3g}"


def check_codes(codes, scales, want, reach, what):
    """Codes and scale bytes of rows whose exact values are `want`."""
    err = ARITH * reach
    e = scales.astype(np.int64) - 127
    assert (e >= -100).all() and (e <= 120).all(), what
    amax, slack = np.abs(want).max(-1), err.max(-1)
    top = 448.0 * 2.0 ** e.astype(np.float64)
    assert (amax - slack <= top).all(), f"{what}: a scale is too small"
    assert ((amax + slack > top / 2) | (e == -100)).all(), f"{what}: a scale is too large"
    got = oracle.decode_rows(codes, scales)
    tol = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** (e - 10.0)[..., None]) + err * (1 + 2.0 ** -4)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} values off"
