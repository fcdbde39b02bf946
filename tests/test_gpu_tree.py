"""bros_attn_tree against its definition in 64 bits: heads, lengths, masks, directions, edges."""

import numpy as np
import pytest

from tests.gpu_helpers import announce, require_gpu
from tests.rows_helpers import Rows, attention, bf16, check, pack, tree_bits, visible

pytestmark = pytest.mark.gpu
D = 128


class Case:
    def __init__(self, n, c0, hq, hkv, bits="tree", seed=0, directions="sequence", poison=True, words=None, **kw):
        import torch
        self.torch = torch
        rng = np.random.default_rng(seed + 1)
        self.b = b = Rows(n, c0, seed, directions, **kw)
        self.hq, self.hkv = hq, hkv
        words = words or max(1, (b.max_n + 63) // 64)
        self.bits = None if bits is None else tree_bits(rng, b.n, words) if isinstance(bits, str) else pack(bits, words)
        self.k, self.v = (bf16(rng, (b.num_blocks, hkv, 16, D)) for _ in range(2))
        if poison:
            blk, slot = np.nonzero(~b.owned())
            self.k[blk, :, slot] = float("nan")
            self.v[blk, :, slot] = float("inf")
        self.q = bf16(rng, (b.rows, hq, D))

    def run(self, out=None, max_ctx=None, cu=True, ws=None, mask=None, stream=None):
        from paper_2504_09590_amd import bros
        torch, b = self.torch, self.b
        tables, dirs, ctx, cu_q = b.cuda()
        self.dev = [x.cuda() for x in (self.q, self.k, self.v)]
        q, k, v = self.dev
        out = torch.full_like(q, 7.0) if out is None else out
        if mask is None and self.bits is not None:
            mask = torch.from_numpy(self.bits).cuda()
        if ws is None:
            size = bros.bros_attn_workspace_size(bros.BROS_WS_TREE, bros.BROS_BF16, max(b.rows, 1), self.hq, D, b.max_ctx)
            ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        bros.bros_attn_tree(out, q, cu_q if cu else None, b.max_n, k, v, tables, dirs, None, ctx,
                            b.max_ctx if max_ctx is None else max_ctx, mask=mask, workspace=ws, stream=stream)
        torch.cuda.synchronize()
        return out

    def want(self, max_ctx=None):
        torch, b = self.torch, self.b
        y, tol = (torch.zeros((b.rows, self.hq, D), dtype=torch.float64) for _ in range(2))
        for s in range(b.S):
            lo, hi = int(b.cu[s]), int(b.cu[s + 1])
            if hi == lo:
                continue
            see = visible(b, s, self.bits, max_ctx)
            blk, slot = b.places(s, np.arange(b.ctx[s]))
            blk = np.clip(blk, 0, b.num_blocks - 1)
            for h in range(self.hq):
                g = h // (self.hq // self.hkv)
                any_row = torch.from_numpy(see.any(0))
                k, v = (torch.where(any_row[:, None], x[blk, g, slot].double(), 0.0) for x in (self.k, self.v))
                y[lo:hi, h], tol[lo:hi, h] = attention(self.q[lo:hi, h].double(), k, v, see, D ** -0.5)
        return y, tol

    def check(self, what, **kw):
        announce(what)
        got = self.run(**kw)
        check(got, *self.want(kw.get("max_ctx")), what)
        return got


HEADS = [(8, 8), (8, 4), (32, 8), (8, 1)]
# new rows and tokens before them: single rows, chains, ragged trees, trees of several masks' words
LENGTHS = [([1], [0]), ([1, 1, 1], [0, 15, 300]), ([4], [300]), ([3, 8, 1, 5], [0, 1, 16, 33]), ([16, 9], [100, 1000]),
           ([33, 64, 2], [31, 500, 2000]), ([130, 7], [40, 77])]


@pytest.mark.parametrize("bits", ["tree", None])
@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("n,c0", LENGTHS)
def test_lengths_and_heads(n, c0, hq, hkv, bits):
    require_gpu()
    Case(n, c0, hq, hkv, bits, seed=len(n) + hq, directions="table" if hkv == 8 else "sequence").check(f"tree {n} {c0} {hq}/{hkv} {bits}")


@pytest.mark.parametrize("n,hq,hkv", [([4, 2], 8, 2), ([13], 8, 2), ([40], 16, 4)])
def test_long_contexts_are_cut_and_merged(n, hq, hkv):
    require_gpu()
    Case(n, [9000 + 37 * i for i in range(len(n))], hq, hkv, seed=3).check(f"tree long {n} {hq}/{hkv}")


def test_many_sequences():
    require_gpu()
    rng = np.random.default_rng(5)
    n = rng.integers(0, 9, 300)
    n[[0, 7, 299]] = 0
    Case(n, rng.integers(0, 120, 300), 8, 2, seed=6).check("tree 300 sequences, some without rows")


def test_one_row_each_without_offsets():
    require_gpu()
    Case([1] * 5, [0, 3, 64, 200, 17], 8, 2, None, seed=8).check("tree without cu_q", cu=False)


@pytest.mark.parametrize("words", [1, 2, 4])
def test_any_bits(words):
    """Bits in any order, beyond the sequence's drafts, and rows that see nothing."""
    require_gpu()
    rng = np.random.default_rng(words)
    n, c0 = [64 * words, 1, 5, 30], [0, 0, 0, 50]
    rows = [int.from_bytes(rng.bytes(8 * words), "little") & int.from_bytes(rng.bytes(8 * words), "little") for _ in range(sum(n))]
    rows[0] = rows[64 * words + 3] = 0
    rows[64 * words] = 0          # a lone row that does not see itself
    c = Case(n, c0, 8, 2, rows, seed=words, words=words)
    got = c.check(f"tree any bits, {words} words")
    assert (got[0] == 0).all() and (got[64 * words] == 0).all() and (got[64 * words + 3] == 0).all()


def test_missing_blocks_see_nothing():
    require_gpu()
    for n in ([5], [12], [40]):
        c = Case(n, [700], 8, 2, seed=11)
        c.b.tables[0, [3, 20, 21]] = [-1, c.b.num_blocks, -2 ** 31]
        c.check(f"tree missing blocks {n}")


def test_context_bound():
    require_gpu()
    c = Case([6, 3], [500, 90], 8, 2, seed=12)
    c.check("tree max_ctx 300", max_ctx=300)
    c.check("tree max_ctx 0", max_ctx=0)


def test_rows_behind_and_inconsistent_lengths():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    c = Case([4, 6, 3], [30, 40, 50], 8, 2, seed=13)
    announce("tree rows behind, lengths that do not fit")
    tables, dirs, ctx, cu = c.b.cuda()
    q = torch.cat([c.q, c.q[:5]]).cuda()
    k, v = c.k.cuda(), c.v.cuda()
    mask = torch.from_numpy(np.concatenate([c.bits, c.bits[:5]])).cuda()
    ws = torch.empty(bros.bros_attn_workspace_size(2, 1, 18, 8, D, 128), dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, 7.0)
    ctx[1] = 5                      # fewer tokens than rows: they see nothing
    bros.bros_attn_tree(out, q, cu, 6, k, v, tables, dirs, None, ctx, 128, mask=mask, workspace=ws)
    torch.cuda.synchronize()
    want, tol = c.want()
    check(out[:4], want[:4], tol[:4], "first")
    check(out[10:13], want[10:], tol[10:], "third")
    assert (out[4:10] == 0).all() and (out[13:] == 7.0).all()
    out.fill_(7.0)
    cu[3] = 100                     # beyond the rows: left alone
    ctx[1] = int(c.b.ctx[1])
    bros.bros_attn_tree(out, q, cu, 18, k, v, tables, dirs, None, ctx, 128, mask=mask, workspace=ws)
    torch.cuda.synchronize()
    check(out[:10], want[:10], tol[:10], "others")
    assert (out[10:] == 7.0).all()


@pytest.mark.parametrize("n,c0", [(6, 0), (6, 50), (14, 100), (40, 7)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_what_is_not_finite_reaches_the_rows_that_see_it(n, c0, bad):
    """A value of draft 2 in dim 5, and all of draft 4's key: rows that do not see them are exact."""
    torch = require_gpu()
    rng = np.random.default_rng(n)
    rows = [int(rng.integers(0, 1 << n)) for _ in range(n)]
    rows = [(x & ~0b10100) | (0b100 if i % 3 == 0 else 0) | (0b10000 if i % 4 == 1 else 0) for i, x in enumerate(rows)]
    c = Case([n, 3], [c0, 9], 8, 2, rows + [1, 3, 7], seed=n)
    want, tol = c.want()
    (b2, s2), (b4, s4) = c.b.places(0, [c0 + 2]), c.b.places(0, [c0 + 4])
    c.v[b2, :, s2, 5] = bad
    c.k[b4, :, s4] = bad
    announce(f"tree not finite {n} {c0} {bad}")
    got = c.run().double().cpu()
    for j in range(n + 3):
        sees2, sees4 = j < n and rows[j] & 4, j < n and rows[j] & 16
        fine = torch.ones(D, dtype=torch.bool)
        if sees4:
            if np.isnan(bad):
                assert not torch.isfinite(got[j]).any()
            continue
        if sees2:
            fine[5] = False
            assert not torch.isfinite(got[j, :, 5]).any()
        check(got[j][:, fine], want[j][:, fine], tol[j][:, fine], f"row {j}")


def test_again_on_another_stream_and_in_a_graph():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    c = Case([5, 30, 1], [3000, 40, 900], 8, 2, seed=21)
    first = c.check("tree first")
    announce("tree on a stream, in a graph")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert torch.equal(first, c.run(stream=side))
    tables, dirs, ctx, cu = c.b.cuda()
    q, k, v = c.dev
    out, mask = torch.zeros_like(q), torch.from_numpy(c.bits).cuda()
    ws = torch.empty(bros.bros_attn_workspace_size(2, 1, 1, 8, D, 0), dtype=torch.uint8, device="cuda")
    call = lambda: bros.bros_attn_tree(out, q, cu, 30, k, v, tables, dirs, None, ctx, c.b.max_ctx, mask=mask, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(3):
        out.fill_(i)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, out)
        assert torch.equal(first, c.run())
    # other lengths and rows in the same buffers
    ctx[0], ctx[2] = 700, 801
    c.b.ctx[0], c.b.ctx[2], c.b.c0[0], c.b.c0[2] = 700, 801, 695, 800
    g.replay()
    torch.cuda.synchronize()
    check(out, *c.want(), "tree replayed with other lengths")


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB a tensor: the blocks used are its last."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    nb = (1 << 20) + 4000
    c = Case([5], [900], 8, 1, seed=31, poison=False)
    tables, dirs, ctx, cu = c.b.cuda()
    announce("tree offsets")
    k, v = (torch.empty((nb, 1, 16, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert k.numel() * 2 > 1 << 32
    k[nb - c.b.num_blocks:], v[nb - c.b.num_blocks:] = c.k.cuda(), c.v.cuda()
    q = c.q.cuda()
    out = torch.empty_like(q)
    ws = torch.empty(bros.bros_attn_workspace_size(2, 1, 1, 8, D, 0), dtype=torch.uint8, device="cuda")
    bros.bros_attn_tree(out, q, cu, 5, k, v, torch.where(tables >= 0, tables + (nb - c.b.num_blocks), tables), dirs, None, ctx,
                        c.b.max_ctx, mask=torch.from_numpy(c.bits).cuda(), workspace=ws)
    torch.cuda.synchronize()
    check(out, *c.want(), "tree offsets")


@pytest.mark.parametrize("kind", ["bf16", "f32", "latent"])
@pytest.mark.parametrize("seed", range(3))
def test_commit(kind, seed):
    """Rows move as if all were read first: paths that go back, repeat, or name no draft; nothing else changes."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    rng = np.random.default_rng(seed)
    n = [1, 8, 40, 256, 5, 0, 17]
    b = Rows(n, [0, 13, 100, 7, 31, 20, 64], seed, "table" if seed else "sequence")
    hkv = 1 if kind == "latent" else 3
    shape = (b.num_blocks, 16, 576) if kind == "latent" else (b.num_blocks, hkv, 16, D)
    dt = torch.float32 if kind == "f32" else torch.bfloat16
    pools = [torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(dt) for _ in range(1 if kind == "latent" else 2)]
    most = 256 if seed == 0 else 30
    path = rng.integers(-2, 60, (b.S, most)).astype(np.int32)
    if seed == 0:
        path[3] = rng.permutation(256)
        path[2, :40] = np.arange(40)[::-1]
    lens = np.array([1, 9, 40, 256, -3, 4, 6], dtype=np.int32)
    b.tables[6, 2] = -1                       # positions 32 .. 47 of the last sequence: none of its drafts' (64 on)
    want = [p.clone() for p in pools]
    for s in range(b.S):
        for i in range(min(int(lens[s]), int(b.n[s]), most)):
            if 0 <= path[s, i] < b.n[s]:
                src, dst = b.places(s, [b.c0[s] + path[s, i]]), b.places(s, [b.c0[s] + i])
                for w, p in zip(want, pools):
                    if kind == "latent":
                        w[dst] = p[src]
                    else:
                        w[dst[0], :, dst[1]] = p[src[0], :, src[1]]
    announce(f"commit {kind} {seed}")
    tables, dirs, ctx, cu = b.cuda()
    dev = [p.cuda() for p in pools]
    bros.bros_tree_commit(dev[0], dev[1] if len(dev) > 1 else None, tables, dirs, None, ctx, cu, torch.from_numpy(path).cuda(),
                          torch.from_numpy(lens).cuda())
    torch.cuda.synchronize()
    for d, w in zip(dev, want):
        assert torch.equal(d.cpu(), w)


def test_commit_leaves_positions_without_a_block():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    b = Rows([40], [10], 4)
    b.tables[0, 1] = b.num_blocks             # positions 16 .. 31: drafts 6 .. 21
    rng = np.random.default_rng(1)
    pool = bf16(rng, (b.num_blocks, 16, 576))
    path = np.array([[30, 7, 3, 39, 38, 37, 36, 35]], dtype=np.int32)   # draft 7 has no block, nor have positions 16 and 17
    want = pool.clone()
    for i in (0, 2, 3, 4, 5):
        want[b.places(0, [10 + i])] = pool[b.places(0, [10 + path[0, i]])]
    announce("commit without blocks")
    tables, dirs, ctx, cu = b.cuda()
    dev = pool.cuda()
    bros.bros_tree_commit(dev, None, tables, dirs, None, ctx, cu, torch.from_numpy(path).cuda(), torch.tensor([8], dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    assert torch.equal(dev.cpu(), want)
