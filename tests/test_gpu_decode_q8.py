"""bros_attn_decode_q8 against the fp64 oracle over the values the 8-bit pool
stands for: lengths, groups, directions, slots and entries that hold nothing."""

import dataclasses

import numpy as np
import pytest

import oracle
from paper_2504_09590_amd import workload as W
from tests import q8_helpers as Q
from tests.gpu_helpers import announce, owned_mask, require_gpu, with_direction_table

pytestmark = pytest.mark.gpu

WEIGHTS = 2.0 ** -16


def device(q8):
    import torch
    from paper_2504_09590_amd import bros
    b = q8.batch
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    return dict(q=bros._tensor(b.q_decode, "bf16", "cuda"), pools=(up(q8.k), up(q8.v), up(q8.scales)),
                tables=up(b.block_tables), dir=up(b.dir), cls=up(b.cls), ctx=up(b.ctx_lens))


def workspace(rows, hq, max_ctx):
    """The queried size, full of NaNs: nothing may read a partial that the call did not write."""
    import torch
    from paper_2504_09590_amd import bros
    size = bros.bros_attn_workspace_size(bros.BROS_WS_DECODE, bros.BROS_BF16, rows, hq, 128, max_ctx)
    return torch.full((size,), 255, dtype=torch.uint8, device="cuda")


def run(q8, max_ctx=None, use_dir=True, repeat=1, scale=0.0):
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    b, d = q8.batch, device(q8)
    max_ctx = int(b.ctx_lens.max()) if max_ctx is None else max_ctx
    ws = workspace(b.num_seqs, b.num_q_heads, max_ctx)
    outs = []
    for _ in range(repeat):
        out = torch.full_like(d["q"], float("nan"))
        bros.bros_attn_decode_q8(out, d["q"], *d["pools"], d["tables"], d["dir"] if use_dir else None, d["cls"], d["ctx"],
                                 max_ctx, scale=scale, workspace=ws)
        torch.cuda.synchronize()
        outs.append(bros.to_host_bits(out))
    return outs if repeat > 1 else outs[0]


def want(b, seqs=None):
    return oracle.decode(b.q_decode, b.k_pool, b.v_pool, b.block_tables, b.dir, b.ctx_lens, "bf16", seqs=seqs)


def check(q8, got, what):
    b = q8.batch
    Q.check(got, want(b), b.q_decode, b, np.arange(b.num_seqs), WEIGHTS, what)


EDGE_CTX = [1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129, 255, 511, 512, 513, 1000, 4097, 20000]


@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_edge_lengths_and_groups(group):
    cls = [W.RT if i % 2 == 0 else W.BE for i in range(len(EDGE_CTX))]
    b = W.custom(EDGE_CTX, cls, 2 * group, 2, seed=100 + group, spare_blocks=7)
    q8 = Q.poison(Q.held(b, group), owned_mask(b))
    announce(f"decode_q8 edges G={group}")
    check(q8, run(q8), f"edges G={group}")


@pytest.mark.parametrize("ctx", [[1], [16], [17], [200], [300, 7], [5, 900], [2000], [8000], [3, 3000, 40]])
@pytest.mark.parametrize("hq,hkv", [(8, 1), (32, 8)])
def test_few_rows(hq, hkv, ctx):
    cls = [W.BE if i % 2 else W.RT for i in range(len(ctx))]
    b = W.custom(ctx, cls, hq, hkv, seed=sum(ctx), spare_blocks=2)
    q8 = Q.poison(Q.held(b, 1), owned_mask(b))
    announce(f"decode_q8 {hq}/{hkv} ctx={ctx}")
    check(q8, run(q8), f"ctx={ctx}")


@pytest.mark.parametrize("rows,lo,hi,hq,hkv", [(700, 1, 90, 16, 2), (300, 1, 900, 32, 8), (96, 500, 6000, 8, 1)])
def test_many_rows(rows, lo, hi, hq, hkv):
    rng = np.random.default_rng(rows)
    ctx = rng.integers(lo, hi + 1, rows)
    b = W.custom(ctx, (rng.random(rows) < 0.5).astype(np.uint8), hq, hkv, seed=rows, spare_blocks=5)
    q8 = Q.poison(Q.held(b, rows), owned_mask(b))
    announce(f"decode_q8 {rows} rows of {lo} to {hi}, {hq}/{hkv}")
    check(q8, run(q8), f"{rows} rows")


@pytest.mark.parametrize("rows,hi,hq,hkv", [(300, 128, 12, 3), (130, 100, 64, 8), (900, 40, 8, 1), (300, 380, 8, 8), (1800, 33, 8, 2), (125, 250, 32, 8)])
def test_short_contexts_by_single_waves(rows, hi, hq, hkv):
    rng = np.random.default_rng(rows + hi)
    ctx = rng.integers(1, hi + 1, rows)
    ctx[:5] = hi, 1, 16, 17, 32
    b = W.custom(ctx, (rng.random(rows) < 0.5).astype(np.uint8), hq, hkv, seed=rows, spare_blocks=7)
    b = with_direction_table(b) if hkv == 3 else b
    q8 = Q.poison(Q.held(b, rows), owned_mask(b))
    empty = rng.integers(0, rows, 9)
    b = q8.batch
    b.ctx_lens[empty] = rng.choice([0, -3], 9)
    gone = np.setdiff1d(rng.integers(0, rows, 9), empty)
    b.block_tables[gone, 0] = b.num_blocks + 3        # a first block outside the pool: its positions are not seen
    announce(f"decode_q8 {rows} rows of up to {hi}, {hq}/{hkv}, a wave each")
    got = run(q8, max_ctx=hi)
    assert (got[empty] == 0).all()
    Q.check(got, masked_reference(q8, b.block_tables), b.q_decode, b, np.arange(rows), WEIGHTS, "short contexts")


def test_more_rows_than_the_prefix_holds():
    rng = np.random.default_rng(12)
    ctx = rng.integers(1, 40, 5001)
    ctx[[7, 2500, 5000]] = 6000, 4100, 900
    b = W.custom(ctx, (rng.random(5001) < 0.5).astype(np.uint8), 4, 1, seed=12, spare_blocks=5)
    q8 = Q.poison(Q.held(b, 12), owned_mask(b))
    announce("decode_q8 5001 rows, three of them long")
    check(q8, run(q8), "5001 rows")


def test_one_long_context_among_short_ones():
    ctx = [50] * 40 + [60000] + [17] * 23
    b = W.custom(ctx, [W.BE] * 64, 8, 2, seed=11, share_tails=False)
    q8 = Q.held(b, 11)
    announce("decode_q8 60000 tokens among short contexts")
    check(q8, run(q8), "one long context")


def test_directions():
    ctx = [5, 40, 17, 70, 16, 3, 333]
    cls = [W.RT, W.RT, W.BE, W.BE, W.RT, W.BE, W.BE]
    b = W.custom(ctx, cls, 16, 4, dirs=[-1, -1, 1, 1, 1, -1, 1], share_tails=False, seed=7, spare_blocks=3)
    q8 = Q.poison(Q.held(b, 7), owned_mask(b))
    announce("decode_q8 explicit directions")
    check(q8, run(q8), "explicit directions")
    b = W.custom(ctx, cls, 16, 4, seed=8, spare_blocks=3)
    q8 = Q.poison(Q.held(b, 8), owned_mask(b))
    announce("decode_q8 directions from classes")
    assert np.array_equal(run(q8, use_dir=False), run(q8))
    t = with_direction_table(b)
    q8 = Q.poison(Q.held(t, 8), owned_mask(t))
    announce("decode_q8 direction table")
    check(q8, run(q8), "direction table")


def test_empty_contexts():
    b = W.custom([40, 1, 20, 700], [W.RT, W.BE, W.RT, W.BE], 8, 4, seed=9)
    q8 = Q.held(b, 9)
    b.ctx_lens[1] = q8.batch.ctx_lens[1] = 0
    q8.batch.ctx_lens[3] = -5
    announce("decode_q8 empty contexts")
    got = run(q8, max_ctx=700)
    assert (got[[1, 3]] == 0).all()
    live = dataclasses.replace(q8.batch, ctx_lens=np.array([40, 0, 20, 0], dtype=np.int32))
    Q.check(got, want(live), live.q_decode, live, np.arange(4), WEIGHTS, "empty contexts")
    q8.batch.ctx_lens[:] = 0
    announce("decode_q8 nothing but empty contexts")
    assert (run(q8, max_ctx=0) == 0).all() and (run(q8, max_ctx=5000) == 0).all()


def masked_reference(q8, tables):
    """fp64 attention where entries outside the pool contribute nothing."""
    b = q8.batch
    out = np.zeros(b.q_decode.shape)
    for s in range(b.num_seqs):
        n = min(int(b.ctx_lens[s]), tables.shape[1] * 16)
        pos = np.arange(n)
        e = tables[s][pos // 16]
        pos = pos[(e >= 0) & (e < b.num_blocks)]
        if not len(pos):
            continue
        blk, slot = oracle.physical_location(tables, b.dir, s, pos)
        k, v = (oracle.widen(p[blk, :, slot], "bf16") for p in (b.k_pool, b.v_pool))
        q = oracle.widen(b.q_decode[s:s + 1], "bf16")
        out[s] = oracle.softmax_attention(q, k, v, np.array([len(pos)]), oracle.default_scale(128))[0]
    return out


@pytest.mark.parametrize("rows", [5, 400])
def test_invalid_entries(rows):
    rng = np.random.default_rng(rows)
    ctx = np.concatenate([[300, 40, 33, 16, 700], rng.integers(1, 400, rows - 5)])
    b = W.custom(ctx, [W.BE] * rows, 16, 4, seed=12, share_tails=False, spare_blocks=2)
    tables = b.block_tables.copy()
    tables[0, [0, 7, 18]] = [-1, b.num_blocks, 2 ** 31 - 1]
    tables[1, 2] = -7
    tables[2, :3] = -1                      # nothing left: zeros
    tables[3, 0] = b.num_blocks + 5
    tables[4, 5:30] = -1
    b = dataclasses.replace(b, block_tables=tables)
    q8 = Q.held(b, 12)
    announce(f"decode_q8 invalid entries, {rows} rows")
    got = run(q8)
    assert (got[[2, 3]] == 0).all()
    Q.check(got, masked_reference(q8, tables), b.q_decode, q8.batch, np.arange(rows), WEIGHTS, "invalid entries")
    # a table shorter than the contexts: the rest contributes nothing
    short = dataclasses.replace(q8.batch, block_tables=np.ascontiguousarray(tables[:, :9]))
    q8 = dataclasses.replace(q8, batch=short)
    announce(f"decode_q8 tables shorter than the contexts, {rows} rows")
    Q.check(run(q8), masked_reference(q8, short.block_tables), b.q_decode, short, np.arange(rows), WEIGHTS, "short tables")


def test_contexts_above_the_bound_are_cut():
    b = W.custom([500, 90, 33], [W.BE] * 3, 8, 2, seed=13, share_tails=False)
    q8 = Q.held(b, 13)
    announce("decode_q8 max_ctx below the contexts")
    for bound in (1, 33, 100, 499):
        cut = dataclasses.replace(q8.batch, ctx_lens=np.minimum(b.ctx_lens, bound).astype(np.int32))
        Q.check(run(q8, max_ctx=bound), want(cut), b.q_decode, cut, np.arange(3), WEIGHTS, f"max_ctx={bound}")


def test_scale_and_large_scores():
    # one key far above the others; scores that span hundreds of powers of two
    b = W.custom([600, 70], [W.BE, W.RT], 8, 2, seed=14, share_tails=False)
    q8 = Q.held(b, 14, spread=5.0)
    announce("decode_q8 other softmax scales")
    for scale in (0.01, 1.0):
        got = run(q8, scale=scale)
        ref = np.zeros(b.q_decode.shape)
        for s in range(2):
            k, v = (oracle.widen(oracle.gather_kv(p, b.block_tables, b.dir, s, int(b.ctx_lens[s])), "bf16")
                    for p in (q8.batch.k_pool, q8.batch.v_pool))
            ref[s] = oracle.softmax_attention(oracle.widen(b.q_decode[s:s + 1], "bf16"), k, v, np.array([len(k)]), scale)[0]
        # (scores, and their error, grow with the scale)
        grown = dataclasses.replace(q8.batch, head_dim=128)
        kmax = np.array([[np.linalg.norm(oracle.widen(oracle.gather_kv(q8.batch.k_pool, b.block_tables, b.dir, s, int(b.ctx_lens[s])),
                                                      "bf16"), axis=-1).max(0)] for s in range(2)])[:, 0]
        vmax = np.array([np.abs(oracle.widen(oracle.gather_kv(q8.batch.v_pool, b.block_tables, b.dir, s, int(b.ctx_lens[s])),
                                             "bf16")).max((0, 2)) for s in range(2)])
        Q.check(got, ref, b.q_decode, grown, np.arange(2), WEIGHTS, f"scale={scale}", kmax * scale * np.sqrt(128), vmax)


@pytest.mark.parametrize("rows", [3, 200])
def test_a_query_that_is_not_finite_stays_alone(rows):
    # infinite scores have no softmax (inf - inf), NaNs neither: NaN in their own heads, nothing elsewhere
    rng = np.random.default_rng(rows)
    b = W.custom(rng.integers(700, 900, rows), rng.integers(0, 2, rows).astype(np.uint8), 16, 4, seed=29)
    q8 = Q.held(b, 29)
    odd = dataclasses.replace(q8, batch=dataclasses.replace(q8.batch, q_decode=q8.batch.q_decode.copy()))
    bad = [(0, 2, 0x7F80), (1, 15, 0x7FC0), (rows - 1, 0, 0xFF80)]        # +inf, NaN, -inf
    for r, h, bits in bad:
        odd.batch.q_decode[r, h, 17] = bits
    announce(f"decode_q8 {rows} rows, queries that are not finite")
    got, plain = run(odd), run(q8)
    for r, h, _ in bad:
        assert np.isnan(oracle.widen(got[r, h], "bf16")).all()
        got[r, h] = plain[r, h]
    check(q8, got, "the other rows")


def test_repeatable_and_a_stream_share():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    rng = np.random.default_rng(15)
    b = W.custom(rng.integers(100, 3000, 40), [W.BE] * 40, 32, 8, seed=15, share_tails=False)
    q8 = Q.held(b, 15)
    announce("decode_q8 twice, bitwise")
    first, second = run(q8, repeat=2)
    assert np.array_equal(first, second)
    check(q8, first, "40 rows")
    announce("decode_q8 on a share of the compute units")
    share = bros.bros_stream_create_cu_share(0, 64)
    try:
        with torch.cuda.stream(share):
            got = run(q8)
    finally:
        torch.cuda.synchronize()
        bros.bros_stream_destroy(share)
    check(q8, got, "64 compute units")


@pytest.mark.parametrize("rows,hi", [(3, 900), (120, 2500)])
def test_captured_and_replayed(rows, hi):
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    rng = np.random.default_rng(rows)
    b = W.custom(rng.integers(1, hi, rows), [W.BE] * rows, 32, 8, seed=16, share_tails=False)
    q8 = Q.held(b, 16)
    d, max_ctx = device(q8), int(b.ctx_lens.max())
    ws = workspace(rows, 32, max_ctx)
    out = torch.empty_like(d["q"])

    def call():
        bros.bros_attn_decode_q8(out, d["q"], *d["pools"], d["tables"], d["dir"], None, d["ctx"], max_ctx, workspace=ws)

    announce(f"decode_q8 captured, {rows} rows")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            call()
    fewer = np.maximum(b.ctx_lens // 3, 1).astype(np.int32)
    for ctx in (b.ctx_lens, fewer, b.ctx_lens):      # the contexts may change between replays
        d["ctx"].copy_(torch.from_numpy(ctx))
        out.zero_()
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        now = dataclasses.replace(q8, batch=dataclasses.replace(q8.batch, ctx_lens=ctx))
        check(now, bros.to_host_bits(out), "replay")


def test_far_blocks():
    # a pool beyond 4 GiB per tensor, the context in its last blocks
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    nb, hkv = 300000, 8
    b = W.custom([150, 2000], [W.BE, W.RT], 16, hkv, seed=17, share_tails=False)
    q8 = Q.held(b, 17)
    d = device(q8)
    far = [torch.full((nb,) + tuple(x.shape[1:]), 0x7F, dtype=torch.uint8, device="cuda") for x in d["pools"]]
    for x, y in zip(far, d["pools"]):
        x[nb - b.num_blocks:] = y
    tables = torch.where(d["tables"] >= 0, d["tables"] + (nb - b.num_blocks), d["tables"]).contiguous()
    out = torch.empty_like(d["q"])
    announce("decode_q8 in blocks beyond 4 GiB")
    bros.bros_attn_decode_q8(out, d["q"], *far, tables, d["dir"], None, d["ctx"], 2000, workspace=workspace(2, 16, 2000))
    torch.cuda.synchronize()
    check(q8, bros.to_host_bits(out), "far blocks")
