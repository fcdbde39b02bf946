"""The latent cache: append, absorbed and expanded attention against their definitions in 64 bits."""

import numpy as np
import pytest

from tests.gpu_helpers import announce, require_gpu
from tests.rows_helpers import Rows, attention, bf16, check, pack, tree_bits, visible

pytestmark = pytest.mark.gpu
LATENT, ROT, ROW = 512, 64, 576
SCALE = 192 ** -0.5


def new_pool(b, rng, poison=True):
    pool = bf16(rng, (b.num_blocks, 16, ROW))
    if poison:
        blk, slot = np.nonzero(~b.owned())
        pool[blk, slot] = float("nan")
    return pool


def latent_rows(b, pool, s, see):
    """fp64 rows [ctx][576] of sequence s, zeros where nothing sees them."""
    import torch
    blk, slot = b.places(s, np.arange(b.ctx[s]))
    rows = pool[np.clip(blk, 0, b.num_blocks - 1), slot].double()
    return torch.where(torch.from_numpy(see.any(0))[:, None], rows, 0.0)


class Absorbed:
    def __init__(self, n, c0, hq, bits="tree", seed=0, directions="sequence", words=None, **kw):
        rng = np.random.default_rng(seed + 1)
        self.b = b = Rows(n, c0, seed, directions, **kw)
        self.hq = hq
        words = words or max(1, (b.max_n + 63) // 64)
        self.bits = None if bits is None else tree_bits(rng, b.n, words) if isinstance(bits, str) else pack(bits, words)
        self.pool = new_pool(b, rng)
        self.q = bf16(rng, (b.rows, hq, ROW), 0.6)

    def run(self, max_ctx=None, cu=True, stream=None):
        import torch
        from paper_2504_09590_amd import bros
        b = self.b
        tables, dirs, ctx, cu_q = b.cuda()
        self.dev = q, pool = self.q.cuda(), self.pool.cuda()
        out = torch.full((b.rows, self.hq, LATENT), 7.0, dtype=torch.bfloat16, device="cuda")
        size = bros.bros_attn_workspace_size(bros.BROS_WS_LATENT, bros.BROS_BF16, max(b.rows, 1), self.hq, ROW, b.max_ctx)
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        bros.bros_attn_latent(out, q, cu_q if cu else None, b.max_n, pool, tables, dirs, None, ctx,
                              b.max_ctx if max_ctx is None else max_ctx,
                              mask=None if self.bits is None else torch.from_numpy(self.bits).cuda(), workspace=ws, stream=stream)
        torch.cuda.synchronize()
        return out

    def want(self, max_ctx=None):
        import torch
        b = self.b
        y, tol = (torch.zeros((b.rows, self.hq, LATENT), dtype=torch.float64) for _ in range(2))
        for s in range(b.S):
            lo, hi = int(b.cu[s]), int(b.cu[s + 1])
            if hi == lo:
                continue
            see = visible(b, s, self.bits, max_ctx)
            rows = latent_rows(b, self.pool, s, see)
            q = self.q[lo:hi].double().reshape(-1, ROW)
            a, t = attention(q, rows, rows[:, :LATENT], np.repeat(see, self.hq, axis=0), SCALE)
            y[lo:hi], tol[lo:hi] = a.view(hi - lo, self.hq, LATENT), t.view(hi - lo, self.hq, LATENT)
        return y, tol

    def check(self, what, **kw):
        announce(what)
        got = self.run(**kw)
        check(got, *self.want(kw.get("max_ctx")), what)
        return got


@pytest.mark.parametrize("hq", [1, 5, 16, 32, 33, 64, 128])
@pytest.mark.parametrize("n,c0", [([1], [0]), ([1, 1, 1, 1], [0, 31, 32, 700])])
def test_decode(n, c0, hq):
    require_gpu()
    c = Absorbed(n, c0, hq, None, seed=hq, directions="table" if hq % 2 else "sequence")
    assert (c.check(f"latent decode {n} {c0} {hq}") == c.run(cu=False)).all()


@pytest.mark.parametrize("hq,n,c0", [(16, [1, 1], [5000, 9000]), (48, [1], [12000]), (128, [1, 1, 1], [6000, 100, 3000])])
def test_decode_of_long_contexts(hq, n, c0):
    require_gpu()
    Absorbed(n, c0, hq, None, seed=hq).check(f"latent decode long {hq}")


@pytest.mark.parametrize("bits", ["tree", None])
@pytest.mark.parametrize("hq,n,c0", [(8, [4, 1, 3], [0, 40, 300]), (16, [4, 2], [17, 900]), (32, [8, 5, 0, 7], [200, 31, 5, 64]),
                                     (7, [70, 3], [20, 0])])
def test_drafts_and_chunks(hq, n, c0, bits):
    require_gpu()
    Absorbed(n, c0, hq, bits, seed=hq + 1, directions="table").check(f"latent rows {hq} {n} {bits}")


def test_many_sequences():
    require_gpu()
    rng = np.random.default_rng(5)
    Absorbed(rng.integers(0, 4, 270), rng.integers(0, 70, 270), 4, seed=6).check("latent 270 sequences")


@pytest.mark.parametrize("hq,n", [(8, 4), (16, 4), (40, 9)])
def test_edges(hq, n):
    """Rows that see nothing, missing blocks, contexts cut short."""
    require_gpu()
    rng = np.random.default_rng(n)
    rows = [int(rng.integers(0, 1 << n)) for _ in range(2 * n)]
    rows[1] = 0
    c = Absorbed([n, n], [0, 400], hq, rows, seed=3)
    c.b.tables[1, [2, 9]] = [-7, c.b.num_blocks]
    got = c.check(f"latent edges {hq} {n}")
    assert (got[1] == 0).all()
    c.check(f"latent edges {hq} {n}, max_ctx", max_ctx=190)
    c.check(f"latent edges {hq} {n}, nothing", max_ctx=0)


@pytest.mark.parametrize("hq", [8, 16, 40])
def test_what_is_not_finite(hq):
    torch = require_gpu()
    n, c0 = 4, 45
    rows = [0b0001, 0b0011, 0b0110, 0b1001]
    c = Absorbed([n], [c0], hq, rows, seed=hq)
    want, tol = c.want()
    blk, slot = c.b.places(0, [c0 + 1])
    c.pool[blk, slot, 100] = float("inf")
    announce(f"latent not finite {hq}")
    got = c.run().double().cpu()
    for j in range(n):
        if rows[j] & 2:
            assert not torch.isfinite(got[j]).all(-1).any()
        else:
            check(got[j], want[j], tol[j], f"row {j}")


def test_absorbed_on_a_stream_and_in_a_graph():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    c = Absorbed([1, 1, 1], [5000, 64, 300], 16, None, seed=21)
    first = c.check("latent first")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    announce("latent on a stream, in a graph")
    assert torch.equal(first, c.run(stream=side))
    tables, dirs, ctx, cu = c.b.cuda()
    q, pool = c.dev
    out = torch.zeros_like(first)
    ws = torch.empty(bros.bros_attn_workspace_size(3, 1, 1, 16, ROW, 0), dtype=torch.uint8, device="cuda")
    call = lambda: bros.bros_attn_latent(out, q, None, 1, pool, tables, dirs, None, ctx, c.b.max_ctx, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(3):
        out.fill_(i)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, out) and torch.equal(first, c.run())


class Chunks:
    def __init__(self, n, c0, hq, seed=0, directions="sequence"):
        rng = np.random.default_rng(seed + 1)
        self.b, self.hq = Rows(n, c0, seed, directions), hq
        self.pool = new_pool(self.b, rng)
        self.q = bf16(rng, (self.b.rows, hq, 192))
        self.w = bf16(rng, (hq, 256, LATENT), LATENT ** -0.5)

    def run(self, heads=None, total=None, max_ctx=None, out=None, stream=None):
        import torch
        from paper_2504_09590_amd import bros
        b = self.b
        tables, dirs, ctx, cu = b.cuda()
        q, pool, w = self.dev = self.q.cuda(), self.pool.cuda(), self.w.cuda()
        total = int(b.ctx.sum()) if total is None else total
        out = torch.full((b.rows, self.hq, 128), 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
        ws = torch.full((bros.bros_latent_prefill_workspace_size(b.S, total, heads or self.hq),), 255, dtype=torch.uint8, device="cuda")
        bros.bros_attn_latent_prefill(out, q, cu, b.max_n, w, pool, tables, dirs, None, ctx, b.max_ctx if max_ctx is None else max_ctx,
                                      total, workspace=ws, stream=stream)
        torch.cuda.synchronize()
        return out

    def want(self, max_ctx=None):
        """Keys and values are rounded to bf16 (2^-8 of a value, and 512 2^-24 of the sum of magnitudes they are
        made of): values add that to the result's error, keys |q| . |their error| to a score's."""
        import torch
        b = self.b
        y, tol = (torch.zeros((b.rows, self.hq, 128), dtype=torch.float64) for _ in range(2))
        for s in range(b.S):
            lo, hi = int(b.cu[s]), int(b.cu[s + 1])
            if hi == lo:
                continue
            see = visible(b, s, None, max_ctx)
            c = latent_rows(b, self.pool, s, see)
            for h in range(self.hq):
                w, q = self.w[h].double(), self.q[lo:hi, h].double()
                kv, big = c[:, :LATENT] @ w.t(), c[:, :LATENT].abs() @ w.abs().t()
                err = kv.abs() * 2.0 ** -8 * 1.01 + big * 516 * 2.0 ** -24
                k, v = torch.cat([kv[:, :128], c[:, LATENT:]], 1), kv[:, 128:]
                a, t = attention(q, k, v, see, SCALE, key_error=(q[:, :128].abs() @ err[:, :128].t()) * SCALE)
                y[lo:hi, h] = a
                seen = torch.from_numpy(see)
                p = ((q @ k.t()) * SCALE).masked_fill(~seen, -np.inf).softmax(1).nan_to_num(0.0)
                tol[lo:hi, h] = t + 1.2 * p @ err[:, 128:]
        return y, tol

    def check(self, what, **kw):
        announce(what)
        got = self.run(**kw)
        want, tol = self.want(kw.get("max_ctx"))
        check(got, want, tol, what)
        # (the bounds above are of the worst case; roundings are independent, and their sum stays near 2^-8)
        off = float((got.double().cpu() - want).norm() / want.norm().clamp(min=1e-30))
        assert off <= 2.0 ** -7, f"{what}: {off:.3g} of the result"
        return got


@pytest.mark.parametrize("hq", [1, 4])
@pytest.mark.parametrize("n,c0", [([1], [0]), ([33], [0]), ([5, 130, 64], [0, 17, 300]), ([300, 1], [0, 40]), ([129, 0, 128], [31, 5, 96])])
def test_chunks(n, c0, hq):
    require_gpu()
    Chunks(n, c0, hq, seed=len(n), directions="table" if hq == 4 else "sequence").check(f"latent prefill {n} {c0} {hq}")


def test_chunks_cut_and_in_passes():
    """Long units cut between workgroups; heads in several passes give the same rows."""
    torch = require_gpu()
    c = Chunks([200, 70], [3000, 1000], 3, seed=9)
    got = c.check("latent prefill long")
    assert torch.equal(got, c.run(heads=3)) 
    one = c.run(heads=1)
    want, tol = c.want()
    check(one, want, tol, "latent prefill, a head a pass")
    check(c.run(heads=2), want, tol, "latent prefill, two heads a pass")
    c = Chunks([40] * 60, [20] * 60, 2, seed=10)
    c.check("latent prefill 60 sequences")


def test_chunk_edges():
    torch = require_gpu()
    c = Chunks([70, 40], [100, 0], 2, seed=12)
    c.b.tables[0, [1, 8]] = [-1, c.b.num_blocks]
    got = c.check("latent prefill missing blocks")
    assert torch.equal(got, c.run(total=4000))
    c.check("latent prefill max_ctx", max_ctx=90)
    # a bound that the second sequence does not fit into (rows come in whole tiles of 32): zeros
    full = c.run()
    small = c.run(total=170 - 62)
    assert torch.equal(small[:70], full[:70]) and (small[70:] == 0).all()
    assert (c.run(total=0) == 0).all()
    # what is not finite reaches the rows that see it
    blk, slot = c.b.places(0, [126])
    c.pool[blk, slot, 7] = float("nan")
    got = c.run()
    assert not torch.isfinite(got[26:70]).any() and torch.equal(got[70:], full[70:]) and torch.isfinite(got[:26]).all()


def test_chunks_on_a_stream_and_in_a_graph():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    c = Chunks([150, 20], [40, 500], 2, seed=14)
    first = c.check("latent prefill first")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    announce("latent prefill on a stream, in a graph")
    assert torch.equal(first, c.run(stream=side))
    tables, dirs, ctx, cu = c.b.cuda()
    q, pool, w = c.dev
    out, total = torch.zeros_like(first), int(c.b.ctx.sum())
    ws = torch.empty(bros.bros_latent_prefill_workspace_size(2, total, 2), dtype=torch.uint8, device="cuda")
    call = lambda: bros.bros_attn_latent_prefill(out, q, cu, 150, w, pool, tables, dirs, None, ctx, 520, total, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(3):
        out.fill_(i)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, out) and torch.equal(first, c.run())


def test_both_forms_agree():
    """The absorbed form, its queries brought into the latent space and its output taken out of it in
    64 bits, against the expanded form: within both forms' bounds."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    c = Chunks([40, 9], [30, 200], 4, seed=17)
    want, tol = c.want()
    check(c.run(), want, tol, "expanded")
    announce("latent, both forms")
    tables, dirs, ctx, cu = c.b.cuda()
    w = c.w.double()
    absorbed = torch.stack([c.q[:, h, :128].double() @ w[h, :128] for h in range(4)], 1)
    q = torch.cat([absorbed, c.q[..., 128:].double()], -1).bfloat16().cuda()
    out = torch.empty((49, 4, LATENT), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(bros.bros_attn_workspace_size(3, 1, 49, 4, ROW, 0), dtype=torch.uint8, device="cuda")
    bros.bros_attn_latent(out, q, cu, 40, c.pool.cuda(), tables, dirs, None, ctx, 210, workspace=ws)
    torch.cuda.synchronize()
    got = torch.stack([out[:, h].double().cpu() @ w[h, 128:].t() for h in range(4)], 1)
    # roundings of queries, weights and outputs to bf16, each 2^-8 / sqrt(3) of the result or of a score of about one
    assert float((got - want).norm() / want.norm()) <= 2.0 ** -7


# --- append -------------------------------------------------------------------

def turned(x, cos, sin, adjacent):
    """fp64 rows [..., 64] turned pair by pair; cos and sin [..., 32]."""
    y = x.clone()
    a, b = (x[..., 0::2], x[..., 1::2]) if adjacent else (x[..., :32], x[..., 32:])
    u, v = a * cos - b * sin, b * cos + a * sin
    if adjacent:
        y[..., 0::2], y[..., 1::2] = u, v
    else:
        y[..., :32], y[..., 32:] = u, v
    return y


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("axes", [0, 1, 3])
@pytest.mark.parametrize("hq", [1, 6, 128])
@pytest.mark.parametrize("place", ["absorbed", "itself"])
def test_append(hq, axes, adjacent, place):
    append_case(hq, axes, adjacent, place, [1, 7, 0, 40, 1])


@pytest.mark.parametrize("hq,n", [(1, 33000), (16, 2100), (48, 1500), (128, 700)])
@pytest.mark.parametrize("axes", [1, 3])
def test_append_of_many_rows(hq, n, axes):
    """Threads of several query rows, of one token and of several."""
    append_case(hq, axes, False, "itself", [1, n, 0, 40, 1])


def append_case(hq, axes, adjacent, place, n):
    """Values are rounded once (2^-8 of each, and 32-bit arithmetic before it); slots that get nothing keep their bits."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    rng = np.random.default_rng(hq + axes)
    b = Rows(n, [0, 30, 5, 3, 100], hq, "table" if axes else "sequence")
    tn, pad = b.rows, 3                       # rows of padding behind the last sequence
    kv_all = bf16(rng, (tn + pad, 704))
    kv = kv_all.cuda()[:, 104:680] if axes != 1 else kv_all.cuda()[:, 104:680].contiguous()
    q = bf16(rng, (tn + pad, hq, 192)).cuda()
    norm = None if axes == 1 else bf16(rng, (LATENT,))
    pool = bf16(rng, (b.num_blocks, 16, ROW)).cuda()
    rows = 64
    angles = rng.random((rows, 32)) * 6.28
    table = torch.from_numpy(np.concatenate([np.cos(angles), np.sin(angles)], 1).astype(np.float32)).cuda()
    sections = (4, 17, 11) if axes == 3 else None
    rope = None if axes == 0 else bros.Rope(table, bros.BROS_ROPE_ADJACENT if adjacent else bros.BROS_ROPE_HALF, sections)
    pos = rng.integers(0, rows, (max(axes, 1), tn + pad)).astype(np.int32)
    pos[0, 4], pos[-1, 9] = -1, rows          # outside the table: zeros, not stored
    b.tables[3, 1] = b.num_blocks             # positions 16 .. 31 of the fourth sequence are not stored
    given = torch.from_numpy(pos).cuda() if axes else None
    before, q_before = pool.clone(), q.clone()
    if place == "absorbed":
        buf = torch.full((tn + pad, hq, ROW), 5.0, dtype=torch.bfloat16, device="cuda")
        q_out = buf[:, :, LATENT:]
    else:
        q_out = q[:, :, 128:]
    announce(f"latent append {hq} {axes} {adjacent} {place} {n}")
    tables, dirs, _, cu = b.cuda()
    bros.bros_latent_append(q_out, q[:, :, 128:], kv, pool, tables, dirs, None, torch.from_numpy(b.c0.astype(np.int32)).cuda(), cu,
                            rope=rope, rope_pos=given, norm=None if norm is None else norm.cuda(), eps=1e-5)
    torch.cuda.synchronize()

    x = kv.double().cpu()
    c = x[:, :LATENT]
    if norm is not None:
        c = c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt() * norm.double()
    k_r, qr = x[:, LATENT:], q_before[:, :, 128:].double().cpu()
    dropped = np.zeros(tn + pad, dtype=bool)
    if axes:
        axis = np.repeat(np.arange(max(axes, 1)), sections or (32,))
        at = pos[axis]                        # [32][tokens]
        dropped = ((pos < 0) | (pos >= rows)).any(0)
        at = np.clip(at, 0, rows - 1)
        t = table.double().cpu().numpy()
        cos, sin = (torch.from_numpy(np.stack([t[at[i], i + o] for i in range(32)], 1)) for o in (0, 32))
        k_r = turned(k_r, cos, sin, adjacent)
        qr = turned(qr, cos[:, None], sin[:, None], adjacent)
    want_q = torch.where(torch.from_numpy(dropped)[:, None, None], 0.0, qr)
    got_q = q_out.double().cpu()
    # (a pair's two products may cancel: 32-bit roundings are of their magnitudes, at most about 2 * 6)
    assert ((got_q - want_q).abs()[:tn] <= want_q.abs()[:tn] * 2.0 ** -8 * 1.01 + 12 * 2.0 ** -23).all()
    if place == "absorbed":
        assert (buf[:, :, :LATENT] == 5.0).all() and (buf[tn:] == 5.0).all() and torch.equal(q, q_before)
    else:
        assert torch.equal(q[:, :, :128], q_before[:, :, :128]) and torch.equal(q[tn:], q_before[tn:])
    want = before.double().cpu()
    stored = torch.zeros((b.num_blocks, 16), dtype=torch.bool)
    row = torch.cat([c, k_r], 1)
    for s in range(b.S):
        for i in range(int(b.n[s])):
            t, p = int(b.cu[s]) + i, int(b.c0[s]) + i
            if dropped[t] or not 0 <= b.tables[s, p // 16] < b.num_blocks:
                continue
            blk, slot = b.places(s, [p])
            want[blk, slot], stored[blk, slot] = row[t], True
    got = pool.double().cpu()
    assert torch.equal(got[~stored], before.double().cpu()[~stored])
    assert ((got - want).abs()[stored] <= want[stored].abs() * 2.0 ** -8 * 1.01 + 12 * 2.0 ** -23).all()


def test_append_without_queries():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    rng = np.random.default_rng(1)
    b = Rows([3], [20], 2)
    pool, kv = torch.zeros((b.num_blocks, 16, ROW), dtype=torch.bfloat16, device="cuda"), bf16(rng, (3, ROW)).cuda()
    announce("latent append without queries")
    tables, dirs, _, cu = b.cuda()
    bros.bros_latent_append(None, None, kv, pool, tables, dirs, None, torch.tensor([20], dtype=torch.int32).cuda(), cu)
    torch.cuda.synchronize()
    assert torch.equal(pool[b.places(0, [20, 21, 22])], kv)      # no norm, no rotation: the bits as they came
    assert int((pool != 0).any(-1).sum()) == 3
