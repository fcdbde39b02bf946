"""Steps of drafts and of a latent cache as they are used: appended, scored, accepted, and again behind
what was kept; prompts in chunks and decode rows over what they left; and all of it captured."""

import types

import numpy as np
import pytest

from tests.gpu_helpers import announce, require_gpu
from tests.rows_helpers import Rows, attention, bf16, check, tree_bits, visible

pytestmark = pytest.mark.gpu
D, ROW, LATENT = 128, 576, 512


def make(n, c0, room, hq, num_prefill=0, seed=0, width=D):
    """A batch of n new rows behind c0 tokens whose tables hold `room` tokens more, and its device tensors."""
    import torch
    b = Rows([m + room for m in n], c0, seed)
    ctx = np.asarray(n) + np.asarray(c0)
    b.n, b.ctx = np.asarray(n), ctx
    b.cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    b.rows, b.max_n = int(b.cu[-1]), max(n)
    batch = types.SimpleNamespace(num_prefill=num_prefill, num_seqs=b.S, cu_new=b.cu, ctx_lens=ctx, num_q_heads=hq, head_dim=D,
                                  dtype="bf16")
    up = lambda x, dt: torch.from_numpy(np.ascontiguousarray(x).astype(dt)).cuda()  # noqa: E731
    dev = types.SimpleNamespace(block_tables=up(b.tables, np.int32), dir=up(b.dir, np.int8), cls=up(np.zeros(b.S), np.uint8),
                                ctx_lens=up(ctx, np.int32), cu_new=up(b.cu, np.int32), pos0=up(c0, np.int32))
    return b, batch, dev


def paths(rng, n, most):
    """Random drafts in rising order for each sequence, and their number."""
    path, lens = np.full((len(n), most), -1, dtype=np.int32), np.zeros(len(n), dtype=np.int32)
    for s, m in enumerate(n):
        keep = np.sort(rng.permutation(m)[:int(rng.integers(0, min(m, most) + 1))])
        path[s, :keep.size], lens[s] = keep, keep.size
    return path, lens


def kept(b, path, lens, pools, heads):
    """Moves the rows of `pools` (host) and the lengths of b as an accept does."""
    for s in range(b.S):
        src = b.places(s, b.c0[s] + path[s, :lens[s]])
        dst = b.places(s, b.c0[s] + np.arange(lens[s]))
        for p in pools:
            if heads:
                p[dst[0], :, dst[1]] = p[src[0], :, src[1]].clone()
            else:
                p[dst] = p[src].clone()
    b.c0 = b.c0 + lens
    b.ctx = b.c0 + b.n


def test_drafts_step_after_step():
    torch = require_gpu()
    from paper_2504_09590_amd.step import DraftStep
    rng = np.random.default_rng(1)
    n, hq, hkv = [5, 1, 0, 12], 8, 2
    b, batch, dev = make(n, [30, 0, 9, 500], 40, hq)
    host = [bf16(rng, (b.num_blocks, hkv, 16, D)) for _ in range(2)]
    dev.k_pool, dev.v_pool = (x.cuda() for x in host)
    step = DraftStep(batch, dev)
    for i in range(4):
        q, k, v = bf16(rng, (b.rows, hq, D)), bf16(rng, (b.rows, hkv, D)), bf16(rng, (b.rows, hkv, D))
        bits = tree_bits(rng, b.n, 1) if i % 2 == 0 else None
        for s in range(b.S):
            at = b.places(s, b.c0[s] + np.arange(b.n[s]))
            for p, x in zip(host, (k, v)):
                p[at[0], :, at[1]] = x[b.cu[s]:b.cu[s + 1]]
        announce(f"drafts, step {i}")
        out = step.run(q.cuda(), k.cuda(), v.cuda(), mask=None if bits is None else torch.from_numpy(bits).cuda())
        torch.cuda.synchronize()
        for s in range(b.S):
            lo, hi = int(b.cu[s]), int(b.cu[s + 1])
            if lo == hi:
                continue
            see = visible(b, s, bits)
            blk, slot = b.places(s, np.arange(b.ctx[s]))
            for h in range(hq):
                kk, vv = (p[blk, h // (hq // hkv), slot].double() for p in host)
                check(out[lo:hi, h], *attention(q[lo:hi, h].double(), kk, vv, see, D ** -0.5), f"step {i}, sequence {s}")
        path, lens = paths(rng, n, 6)
        step.accept(torch.from_numpy(path).cuda(), torch.from_numpy(lens).cuda())
        torch.cuda.synchronize()
        kept(b, path, lens, host, True)
        for p, x in zip(host, (dev.k_pool, dev.v_pool)):
            assert torch.equal(p, x.cpu())
        assert (dev.pos0.cpu().numpy() == b.c0).all() and (dev.ctx_lens.cpu().numpy() == b.ctx).all()


def rope_and_norm(rng, rows=2000):
    import torch
    from paper_2504_09590_amd import bros
    angles = rng.random((rows, 32)) * 6.28
    table = torch.from_numpy(np.concatenate([np.cos(angles), np.sin(angles)], 1).astype(np.float32)).cuda()
    return bros.Rope(table), bf16(rng, (LATENT,)).cuda()


def row_part(b, P):
    """The sequences from P on as a batch of their own (sharing the lengths at this time)."""
    r = types.SimpleNamespace(S=b.S - P, n=b.n[P:], c0=b.c0[P:], ctx=b.ctx[P:], cu=b.cu[P:] - b.cu[P], tables=b.tables[P:],
                              num_blocks=b.num_blocks)
    return r


@pytest.mark.parametrize("turned", [False, True])
def test_latent_prompts_then_rows(turned):
    """Chunks beside drafts: the pool that the append left (checked against its own tests' definition by
    the rows without norm and rotation), both forms of attention over it, and what accept keeps."""
    torch = require_gpu()
    from paper_2504_09590_amd.step import LatentStep
    rng = np.random.default_rng(2)
    hq, P, n = 6, 2, [50, 33, 4, 1, 7]
    b, batch, dev = make(n, [0, 64, 100, 3, 31], 30, hq, num_prefill=P)
    host = bf16(rng, (b.num_blocks, 16, ROW))
    pool = host.cuda()
    w = bf16(rng, (hq, 256, LATENT), LATENT ** -0.5)
    rope, norm = rope_and_norm(rng) if turned else (None, None)
    step = LatentStep(batch, dev, pool, w.cuda(), rope=rope, norm=norm, pass_heads=4)
    for i in range(3):
        kv, qc, qr = bf16(rng, (b.rows, ROW)), bf16(rng, (83, hq, 192)), bf16(rng, (b.rows - 83, hq, ROW), 0.6)
        bits = tree_bits(rng, b.n[P:], 1) if i != 1 else None
        dqc, dqr = qc.cuda(), qr.cuda()
        announce(f"latent, step {i}, {turned}")
        pos = torch.from_numpy(rng.integers(0, 2000, b.rows).astype(np.int32)).cuda() if turned else None
        chunks, rows = step.run(kv.cuda(), dqc, dqr, mask=None if bits is None else torch.from_numpy(bits).cuda(), rope_pos=pos)
        torch.cuda.synchronize()
        now = pool.cpu()
        touched = torch.zeros((b.num_blocks, 16), dtype=torch.bool)
        for s in range(b.S):
            touched[b.places(s, b.c0[s] + np.arange(b.n[s]))] = True
            if not turned:
                host[b.places(s, b.c0[s] + np.arange(b.n[s]))] = kv[b.cu[s]:b.cu[s + 1]]
        assert torch.equal(now[~touched], host[~touched])
        if turned:
            assert not torch.equal(dqc.cpu()[:, :, 128:], qc[:, :, 128:]) and torch.equal(dqc.cpu()[:, :, :128], qc[:, :, :128])
            assert not torch.equal(dqr.cpu()[:, :, 512:], qr[:, :, 512:]) and torch.equal(dqr.cpu()[:, :, :512], qr[:, :, :512])
            host = now.clone()
        else:
            assert torch.equal(now, host) and torch.equal(dqc.cpu(), qc) and torch.equal(dqr.cpu(), qr)
        qc, qr = dqc.cpu().double(), dqr.cpu().double()
        rest = row_part(b, P)
        for s in range(b.S):
            lo, hi = int(b.cu[s]), int(b.cu[s + 1])
            c = host[b.places(s, np.arange(b.ctx[s]))].double()
            if s >= P:
                see = visible(rest, s - P, bits)
                y, tol = attention(qr[lo - 83:hi - 83].reshape(-1, ROW), c, c[:, :LATENT], np.repeat(see, hq, axis=0), 192 ** -0.5)
                check(rows[lo - 83:hi - 83].reshape(-1, LATENT), y, tol, f"step {i}, rows of {s}")
                continue
            see = visible(b, s, None)
            for h in range(hq):
                kk = torch.cat([c[:, :LATENT] @ w[h, :128].double().t(), c[:, LATENT:]], 1)
                y, _ = attention(qc[lo:hi, h], kk, c[:, :LATENT] @ w[h, 128:].double().t(), see, 192 ** -0.5)
                # (bounds value by value are the expanded form's own tests'; here: the roundings together)
                assert float((chunks[lo:hi, h].cpu().double() - y).norm() / y.norm()) <= 2.0 ** -7
        path, lens = paths(rng, n[P:], 5)
        step.accept(torch.from_numpy(path).cuda(), torch.from_numpy(lens).cuda())
        torch.cuda.synchronize()
        full_path, full_lens = np.concatenate([np.zeros((P, 5), dtype=np.int32), path]), np.concatenate([np.zeros(P, dtype=np.int32), lens])
        kept(b, full_path, full_lens, [host], False)
        assert torch.equal(pool.cpu(), host)
        assert (dev.pos0.cpu().numpy() == b.c0).all() and (dev.ctx_lens.cpu().numpy() == b.ctx).all()


@pytest.mark.parametrize("kind", ["drafts", "latent"])
def test_steps_captured(kind):
    """Run and accept in one graph, replayed with other rows, masks and paths: the bits of the eager step."""
    torch = require_gpu()
    from paper_2504_09590_amd.step import DraftStep, LatentStep
    rng = np.random.default_rng(3)
    n, c0, hq = [6, 3, 9], [200, 17, 1500], 8
    both = []
    for _ in range(2):
        b, batch, dev = make(n, c0, 60, hq, seed=5)
        if kind == "drafts":
            dev.k_pool, dev.v_pool = (bf16(np.random.default_rng(s), (b.num_blocks, 2, 16, D)).cuda() for s in (7, 8))
            both.append((DraftStep(batch, dev), dev, [dev.k_pool, dev.v_pool]))
        else:
            pool = bf16(np.random.default_rng(7), (b.num_blocks, 16, ROW)).cuda()
            both.append((LatentStep(batch, dev, pool), dev, [pool]))
    shapes = [(18, hq, D), (18, 2, D), (18, 2, D)] if kind == "drafts" else [(18, ROW), (18, hq, ROW)]
    draw = lambda: [bf16(rng, s).cuda() for s in shapes] + [torch.from_numpy(tree_bits(rng, n, 1)).cuda()] + \
        [torch.from_numpy(x).cuda() for x in paths(rng, n, 4)]  # noqa: E731
    fixed = draw()

    def call(step, x):
        if kind == "drafts":
            out = step.run(*x[:3], mask=x[3])
        else:
            out = step.run(x[0], q_rows=x[1], mask=x[2])[1]
        step.accept(x[-2], x[-1])
        return out

    announce(f"step captured, {kind}")
    (eager, _, pools), (graphed, _, other) = both
    assert torch.equal(call(eager, fixed), call(graphed, fixed))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call(graphed, fixed)
    for i in range(4):
        x = draw()
        for a, c in zip(fixed, x):
            a.copy_(c)
        g.replay()
        want = call(eager, x)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        for a, c in zip(pools, other):
            assert torch.equal(a, c), i
