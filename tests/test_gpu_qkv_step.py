"""QkvStep: projected rows in, attention out, on 16-bit, 32-bit and 8-bit pools, and
the block manager driving an 8-bit cache step after step.

Checked in the order of the step: what the append wrote against fp64 (tests of the
append: their tolerances), every other byte of the pools unchanged, and the attention
against the fp64 oracle over the pool and the q rows that the append left.

The rows here differ in size by up to 2^6, so the attention's tolerance is the one of
q8_helpers, relative to the largest |v| that a row sees (a fixed bound for values near
one would be below half a bf16 step at 16). Weights: one bf16 part is off by 2^-8 and
its sum by as much again, 2^-7 (16-bit pools; 8-bit prefill); two parts, 2^-16 (8-bit
decode). 32-bit pools: weights are not rounded, but n terms summed one after another,
in the numerator and in the denominator, are off by up to 2 n 2^-24."""

import types

import numpy as np
import pytest

import oracle
from paper_2504_09590_amd import manager as M
from paper_2504_09590_amd import workload as W
from tests import append_helpers as A
from tests import q8_helpers as Q
from tests.gpu_helpers import announce, owned_mask, require_gpu

pytestmark = pytest.mark.gpu

RT, BE = 0, 1


def places(b):
    """(sequence, position, block, slot) of every new token of the batch."""
    seq, pos = A.tokens(b)
    at = [oracle.physical_location(b.block_tables, b.dir, int(s), np.array([p])) for s, p in zip(seq, pos)]
    return seq, pos, np.array([int(x[0]) for x, _ in at]), np.array([int(y[0]) for _, y in at])


def same(x, y):
    """Bit for bit (a NaN equals itself)."""
    return np.array_equal(np.ascontiguousarray(x).view(np.uint8), np.ascontiguousarray(y).view(np.uint8))


def check_append(r, b, q_rows, before, after, what):
    """before and after: (k, v) or (k, v, scales) pools on the host."""
    seq, pos, blk, slot = places(b)
    (q, q_reach), (k, k_reach) = A.expected(r, seq, pos)
    A.check_close(q_rows, q, q_reach, r.dtype, f"{what}: q")
    touched = np.zeros((b.num_blocks, 16), dtype=bool)
    touched[blk, slot] = True
    for was, now in zip(before, after):
        axes = (0, 3, 1, 2) if was.shape[2] == 2 else (0, 2, 1, 3)       # the slot behind the block
        assert same(was.transpose(axes)[~touched], now.transpose(axes)[~touched]), f"{what}: another slot changed"
    if len(after) == 3:
        A.check_codes(after[0][blk, :, slot], after[2][blk, :, 0, slot], k, k_reach, f"{what}: k")
        codes, scales = oracle.encode(oracle.widen(r.v, r.dtype))
        assert (after[1][blk, :, slot] == codes).all() and (after[2][blk, :, 1, slot] == scales).all(), f"{what}: v"
    else:
        A.check_close(after[0][blk, :, slot], k, k_reach, r.dtype, f"{what}: k")
        assert (after[1][blk, :, slot] == r.v).all(), f"{what}: v"


def values(codes, scales):
    """bf16 bits of the values of an 8-bit pool (exact) by the side of K (0) or V (1)."""
    return [W._to_bf16_bits(oracle.decode_rows(c, scales[:, :, i]).astype(np.float32)) for i, c in enumerate(codes)]


def check_attention(b, dtype, q_rows, pools, pre, dec, what):
    """The step's outputs over the pools (k, v or k, v, scales) it left."""
    P, n = b.num_prefill, int(b.cu_q[-1])
    k, v = pools[:2] if len(pools) == 2 else values(pools[:2], pools[2])
    view = types.SimpleNamespace(num_kv_heads=k.shape[1], head_dim=128, num_seqs=b.num_seqs, num_blocks=b.num_blocks,
                                 block_tables=b.block_tables, dir=b.dir, ctx_lens=b.ctx_lens, k_pool=k, v_pool=v)
    most = int(b.ctx_lens.max())
    weights = 2 * most * 2.0 ** -24 if dtype == "f32" else 2.0 ** -7
    parts = []
    if P:
        want = oracle.prefill_chunk(q_rows[:n], b.cu_q, k, v, b.block_tables[:P], b.dir[:P], b.ctx_lens[:P], dtype)
        parts.append((pre, want, q_rows[:n], np.repeat(np.arange(P), np.diff(b.cu_q)), weights, "prefill"))
    if b.num_seqs > P:
        want = oracle.decode(q_rows[n:], k, v, b.block_tables[P:], b.dir[P:], b.ctx_lens[P:], dtype)
        parts.append((dec, want, q_rows[n:], np.arange(P, b.num_seqs), 2.0 ** -16 if len(pools) == 3 else weights, "decode"))
    for got, want, q, seq, w, name in parts:
        Q.check(got, want, q, view, seq, w, f"{what}: {name}", dtype=dtype)


def pool_of(b, eight, seed):
    """Host pools in which no slot of a new token and none outside a sequence is a number."""
    _, _, blk, slot = places(b)
    mask = owned_mask(b)
    mask[blk, slot] = False
    if eight:
        q8 = Q.poison(Q.held(b, seed), mask)
        return q8.k, q8.v, q8.scales
    bad = np.float32("nan") if b.dtype == "f32" else np.uint16(0x7FC0)
    k, v = b.k_pool.copy(), b.v_pool.copy()
    blocks, slots = np.nonzero(~mask)
    k[blocks, :, slots] = bad
    v[blocks, :, slots] = bad
    return k, v


KINDS = [("bf16", False), ("f32", False), ("bf16", True)]


@pytest.mark.parametrize("dtype,eight", KINDS)
@pytest.mark.parametrize("ctx,new,pre", [([64 + 130, 45, 2000, 700, 31, 17, 1], [130, 45, 1, 1, 1, 1, 1], 2),
                                         ([300, 7], [1, 7], 2), ([5, 900, 33], [1, 1, 1], 0)])
def test_step(ctx, new, pre, dtype, eight):
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    from paper_2504_09590_amd.step import QkvStep
    hq, hkv = 16, 4
    b = W.custom(ctx, [i % 2 for i in range(len(ctx))], hq, hkv, dtype=dtype, seed=len(ctx), num_prefill=pre,
                 new_counts=new, spare_blocks=4)
    r = A.make_rows(b, hq, dtype, True, True, rotary=128, seed=5)
    before = pool_of(b, eight, 3)
    announce(f"qkv step ctx={ctx} new={new} {dtype} eight={eight}")
    dev = bros.to_device(b)
    pools = [bros._tensor(p, None if eight else dtype, "cuda") for p in before]
    dev.k_pool, dev.v_pool = pools[:2]
    kw = A.options(r)
    step = QkvStep(b, dev, rope=kw["rope"], norm=kw["norm"], kv_scales=pools[2] if eight else None)
    rows = A.device_rows(r)
    state = []
    for _ in range(2):                       # a step run again writes the same bytes
        out_pre, out_dec = step.run(*rows)
        torch.cuda.synchronize()
        host = bros.to_host_bits if not eight else lambda t: t.cpu().numpy()
        state.append([host(p) for p in pools] + [bros.to_host_bits(x) for x in (step.q, out_pre, out_dec)])
    assert all(same(x, y) for x, y in zip(*state)), "two runs of one step differ"
    after, (q, got_pre, got_dec) = state[0][:-3], state[0][-3:]
    check_append(r, b, q, before, after, "append")
    check_attention(b, dtype, q, after, got_pre, got_dec, "attention")
    # the step recorded once and replayed
    for p, was in zip(pools, before):
        p.copy_(bros._tensor(was, None if eight else dtype, "cuda"))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run(*rows)
    for _ in range(3):
        for t in (step.q, step.out):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        again = [host(p) for p in pools] + [bros.to_host_bits(x) for x in (step.q, out_pre, out_dec)]
        assert all(same(x, y) for x, y in zip(again, state[0])), "a replay differs"


def test_refusals():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    from paper_2504_09590_amd.step import QkvStep
    b = W.custom([40, 50], [0, 1], 8, 2, num_prefill=0, new_counts=[3, 1], spare_blocks=1)
    with pytest.raises(ValueError):
        QkvStep(b, bros.to_device(b))
    torch.cuda.synchronize()


def test_manager_drives_an_eight_bit_cache():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    from paper_2504_09590_amd.step import QkvStep
    from paper_2504_09590_amd.swap import PlanExecutor
    rng = np.random.default_rng(2025)
    nb, hkv, hq, d = 40, 4, 16, 128
    pools = [np.full((nb, hkv, 16, d), 0x7F, dtype=np.uint8), np.full((nb, hkv, 16, d), 0xFF, dtype=np.uint8),
             np.full((nb, hkv, 2, 16), 255, dtype=np.uint8)]           # nothing written yet: NaNs
    dev = [torch.from_numpy(p).cuda() for p in pools]
    mgr = M.BlockManager(nb)
    ex = PlanExecutor(dev[0], dev[1], max_rows=64, kv_scales=dev[2])
    store, cls, started = {}, {}, set()
    stats = {"victims": 0, "moves": 0, "restores": 0, "prefill": 0, "decode": 0}
    next_id = 1

    def drop(r):
        mgr.release(r)
        ex.drop(r)
        for key in [k for k in store if k[0] == r]:
            del store[key]
        del cls[r]

    def slot_rows(ids):
        blk, slot = np.asarray(ids) // 16, np.asarray(ids) % 16
        return pools[0][blk, :, slot], pools[1][blk, :, slot], pools[2][blk, :, :, slot]

    def put_rows(rows, ids):
        blk, slot = np.asarray(ids) // 16, np.asarray(ids) % 16
        pools[0][blk, :, slot], pools[1][blk, :, slot], pools[2][blk, :, :, slot] = rows

    def carry_out(req, plan):
        ex.execute(req, plan)
        for r, p, b, s in plan.victims:
            store[(int(r), int(p))] = [x[0].copy() for x in slot_rows([int(b) * 16 + int(s)])]
        if len(plan.move_src):
            put_rows([x.copy() for x in slot_rows(plan.move_src)], plan.move_dst)
        for p, dst in zip(plan.restore_pos, plan.restore_dst):
            put_rows([x[None] for x in store.pop((req, int(p)))], [int(dst)])
        stats["victims"] += len(plan.victims)
        stats["moves"] += len(plan.move_src)
        stats["restores"] += len(plan.restore_pos)

    for step in range(14):
        for _ in range(rng.integers(1, 4)):
            cls[next_id] = RT if rng.random() < 0.5 else BE
            mgr.add(next_id, cls[next_id])
            next_id += 1
        for r in [r for r in cls if r in started]:
            if rng.random() < 0.08:
                drop(r)
        ran = []
        for r in sorted((r for r in cls if rng.random() < 0.7), key=lambda r: cls[r]):
            n_new = int(rng.integers(20, 90)) if r not in started else 1
            try:
                if mgr.query(r)[2]:
                    carry_out(r, mgr.restore(r))
                p0 = mgr.query(r)[0]
                plan = mgr.grow(r, n_new)
            except bros.BrosError as e:
                if getattr(e, "plan", None) is not None:
                    carry_out(r, e.plan)
                drop(r)
                continue
            carry_out(r, plan)
            started.add(r)
            ran.append((r, p0, n_new))
        ran = sorted((x for x in ran if x[0] in cls and mgr.query(x[0])[2] == 0), key=lambda x: x[2] == 1)
        if not ran:
            continue
        ids = [x[0] for x in ran]
        tabs = [mgr.table(r) for r in ids]
        tables = np.zeros((len(ids), max(len(t) for t in tabs)), dtype=np.int32)
        for i, t in enumerate(tabs):
            tables[i, :len(t)] = t
        counts = np.array([x[2] for x in ran])
        cu_new = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        P = int(np.sum(counts > 1))
        b = types.SimpleNamespace(
            num_prefill=P, num_seqs=len(ids), num_blocks=nb, num_kv_heads=hkv, num_q_heads=hq, head_dim=d, dtype="bf16",
            block_tables=tables, dir=np.array([1 if cls[r] == RT else -1 for r in ids], dtype=np.int8),
            cls=np.array([cls[r] for r in ids], dtype=np.uint8),
            ctx_lens=np.array([mgr.query(r)[0] for r in ids], dtype=np.int32),
            pos0=np.array([x[1] for x in ran], dtype=np.int32), cu_new=cu_new, cu_q=cu_new[:P + 1].copy())
        bros.bros_check_batch(tables, b.dir, None, b.ctx_lens, nb)
        r = A.make_rows(b, hq, "bf16", True, True, rotary=128, seed=step)
        announce(f"8-bit manager step {step}: {len(ids)} sequences, {int(cu_new[-1])} new tokens, {P} prefill chunks")
        up = {n: torch.from_numpy(np.ascontiguousarray(getattr(b, n))).cuda() for n in
              ("block_tables", "dir", "cls", "ctx_lens", "cu_q", "cu_new", "pos0")}
        batch = bros.DeviceBatch(k_pool=dev[0], v_pool=dev[1], q_prefill=None, q_decode=None, k_new=None, v_new=None, **up)
        kw = A.options(r)
        run = QkvStep(b, batch, rope=kw["rope"], norm=kw["norm"], kv_scales=dev[2])
        pre, dec = run.run(*A.device_rows(r))
        torch.cuda.synchronize()
        after = [p.cpu().numpy() for p in dev]
        q = bros.to_host_bits(run.q)
        check_append(r, b, q, pools, after, f"step {step}")      # and every slot the plans filled
        check_attention(b, "bf16", q, after, bros.to_host_bits(pre), bros.to_host_bits(dec), f"step {step}")
        pools = after
        stats["prefill"] += P
        stats["decode"] += len(ids) - P
        mgr.validate()
    print("manager-driven steps on an 8-bit cache:", stats)
    assert all(stats[k] > 0 for k in ("victims", "restores", "prefill", "decode")), stats
