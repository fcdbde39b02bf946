"""Drafted tokens over the paged cache, and a cache of one latent vector per token.

A case is one call that a serving loop makes:

  tree            rows of drafted tokens, each seeing the cache before the drafts and
                  the drafts its mask names, over a bf16 K/V pool
  commit          the accepted drafts' rows moved to the positions they now have, in a
                  K/V pool or a latent pool
  latent-append   norm of a step's new latent rows, rotation of their shared key and of
                  the queries' rotated dims, and the write into a latent pool
  latent          attention with queries in the latent space (absorbed form): one row
                  per sequence, short chunks, or drafts
  latent-prefill  causal chunks whose keys and values are made from the latents
                  (expanded form)

A latent pool holds one row of 576 values per slot, [blocks][16][576]: 512 of the latent
vector, which all heads share as key and value, and 64 of a rotated key. The expanded form's
weights w_kv [heads][256][512] give 128 key dims and 128 value dims of each head.

Lengths follow from the case alone (its "lengths" number); values, trees and physical blocks
follow from the seed.
"""

import math

import numpy as np
import torch

own = False

D = 128
BLOCK = 16
LATENT, ROT = 512, 64
ROW = LATENT + ROT

_DEFAULTS = {
    "kind": "tree", "hq": 32, "hkv": 8, "lengths": 1,
    "seqs": 1, "c0_lo": 0, "c0_hi": 0, "spread": "uniform",    # sequences and their tokens before the new rows
    "n_lo": 1, "n_hi": 1,                                      # new rows of a sequence
    "mask": "tree",                                            # or "causal" (no mask given)
    "direction": "sequence",                                   # or "table": a flag per table entry
    "pool": "kv",                                              # commit: or "latent"
    "q": "absorbed",                                           # latent-append: queries go to the absorbed form's
}                                                              # buffer, or "place": they stay where they are


def _case(name, **kw):
    return dict(_DEFAULTS, name=name, **kw)


def listed():
    return [
        # The smallest verification: one sequence, a chain of four drafts, where the launch counts.
        _case("tree-chain", hq=8, hkv=2, c0_lo=300, c0_hi=300, n_lo=4, n_hi=4, mask="causal"),
        # An ordinary verification step of an 8B model's attention: trees of up to 32 drafts.
        _case("tree-8b", seqs=16, c0_lo=128, c0_hi=8192, n_lo=17, n_hi=32, lengths=2),
        # Long documents and wide trees, a 70B model's heads, directions by table entry.
        _case("tree-70b-long", hq=64, seqs=6, c0_lo=8000, c0_hi=32000, n_lo=64, n_hi=64, direction="table", lengths=3),
        # What follows a verification: a few accepted drafts of each sequence move up.
        _case("commit-8b", kind="commit", seqs=64, c0_lo=128, c0_hi=4096, n_lo=17, n_hi=32, lengths=4),
        # The same in a latent pool, larger trees.
        _case("commit-latent", kind="commit", pool="latent", seqs=256, c0_lo=128, c0_hi=2048, n_lo=33, n_hi=64, lengths=5),
        # An ordinary decode step's new rows, queries into the absorbed form's buffer.
        _case("latent-append-decode", kind="latent-append", hq=32, seqs=64, c0_lo=128, c0_hi=8192, lengths=6),
        # A batch of prompts, all heads, queries turned in their place.
        _case("latent-append-prompts", kind="latent-append", hq=128, seqs=4, n_lo=1001, n_hi=1999, q="place", lengths=7),
        # One GPU's share of the heads: the cache's bytes decide.
        _case("latent-decode-16", kind="latent", hq=16, seqs=64, c0_lo=128, c0_hi=8192, lengths=8),
        # The largest decode step, all heads on one GPU: bytes and products are level.
        _case("latent-decode-128", kind="latent", hq=128, seqs=96, c0_lo=256, c0_hi=16384, lengths=9),
        # Verification of small trees over the latent cache, an interactive load.
        _case("latent-drafts", kind="latent", hq=32, seqs=5, c0_lo=200, c0_hi=4000, n_lo=5, n_hi=8, lengths=10),
        # A short prompt's only chunk, an odd row count: time to the first token.
        _case("latent-prefill-short", kind="latent-prefill", hq=32, n_lo=301, n_hi=301, lengths=11),
        # Chunks of long prompts, some with much of the prompt cached.
        _case("latent-prefill-chunks", kind="latent-prefill", hq=64, seqs=4, n_lo=601, n_hi=1400, c0_lo=0, c0_hi=6000, lengths=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above: a model's heads or one GPU's share of them, any length."""
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        n, c0 = _lengths(c)
        padded = len(n) * int((n + c0).max()) * (c["hq"] * int(n.max()) + 2 * ROW * c["hkv"])
        if c["kind"] == "latent-prefill":
            padded += len(n) * int((n + c0).max()) * c["hq"] * 2 * (2 * D + ROT)
        if c["kind"] in ("commit", "latent-append"):
            padded = 0
        if _cost(c) <= most and padded <= 4e9:     # (what the plain form lays out at once, in values)
            return c


def _draw(rng):
    c = dict(_DEFAULTS, lengths=rng.randrange(1, 1 << 20))
    c["kind"] = rng.choice(["tree", "tree", "tree", "commit", "latent-append", "latent", "latent", "latent", "latent-prefill",
                            "latent-prefill"])
    c["direction"] = rng.choice(["sequence", "table"])
    c["spread"] = rng.choice(["uniform", "uniform", "lognormal"])
    if c["kind"] in ("tree", "commit"):
        c["hq"], c["hkv"] = rng.choice([(32, 8), (32, 8), (64, 8), (8, 1), (16, 8), (8, 8)])
    else:
        c["hq"], c["hkv"] = rng.choice([8, 16, 16, 32, 64, 128]), 1
    c["c0_hi"] = _log(rng, 16, 32000)
    c["c0_lo"] = int(c["c0_hi"] * rng.uniform(0.02, 0.6))
    c["n_hi"] = _log(rng, 1, 128)
    c["n_lo"] = max(1, int(c["n_hi"] * rng.uniform(0.2, 1.0)))
    c["mask"] = rng.choice(["tree", "tree", "causal"])
    if c["kind"] == "tree":
        c["seqs"] = _log(rng, 1, 64)
    elif c["kind"] == "commit":
        c["seqs"] = _log(rng, 1, 512)
        c["c0_hi"], c["c0_lo"] = min(c["c0_hi"], 4096), min(c["c0_lo"], 2000)
        c["pool"] = rng.choice(["kv", "latent"])
    elif c["kind"] == "latent-append":
        if rng.random() < 0.5:
            c["seqs"], c["n_lo"], c["n_hi"] = _log(rng, 1, 512), 1, 1
        else:
            c["seqs"], c["n_hi"] = rng.randint(1, 6), _log(rng, 16, 2048)
            c["n_lo"] = max(1, int(c["n_hi"] * rng.uniform(0.3, 1.0)))
        c["c0_hi"], c["c0_lo"] = min(c["c0_hi"], 8192), min(c["c0_lo"], 4000)
        c["q"] = rng.choice(["absorbed", "place"])
    elif c["kind"] == "latent":
        c["seqs"] = _log(rng, 1, 128)
        if rng.random() < 0.5:
            c["n_lo"] = c["n_hi"] = 1
        else:
            c["n_hi"] = min(c["n_hi"], 64)
            c["n_lo"] = min(c["n_lo"], c["n_hi"])
    else:
        c["seqs"] = rng.randint(1, 6)
        c["n_hi"] = _log(rng, 64, 2048)
        c["n_lo"] = max(1, int(c["n_hi"] * rng.uniform(0.2, 1.0)))
        c["c0_hi"] = rng.choice([0, 0, rng.randint(1, 8000)])
        c["c0_lo"] = 0
        c["mask"] = "causal"
    return c


def _lengths(case):
    """(new rows, tokens before them) of every sequence, from the case alone."""
    rng = np.random.default_rng(case["lengths"])
    n = rng.integers(case["n_lo"], case["n_hi"] + 1, case["seqs"])
    if case["spread"] == "lognormal":
        sigma2 = math.log(1.0 + (500.0 / 600.0) ** 2)      # mean 600, standard deviation 500 before the clip
        c0 = np.rint(rng.lognormal(math.log(600.0) - sigma2 / 2, math.sqrt(sigma2), case["seqs"]))
        return n, np.clip(c0, case["c0_lo"], case["c0_hi"]).astype(np.int64)
    return n, rng.integers(case["c0_lo"], case["c0_hi"] + 1, case["seqs"])


def _accepted(case, n):
    """Accepted drafts of every sequence: one to eight of its tree."""
    rng = np.random.default_rng(case["lengths"] + 1)
    return np.minimum(n, rng.integers(1, 9, len(n)))


def work(case):
    n, c0 = _lengths(case)
    hq, hkv, rows, ctx = case["hq"], case["hkv"], int(n.sum()), n + c0
    tables = 4 * int(((ctx + BLOCK - 1) // BLOCK).sum())
    if case["kind"] == "commit":
        row = 2 * ROW if case["pool"] == "latent" else 2 * 2 * hkv * D
        return {"bytes": int(_accepted(case, n).sum()) * (2 * row + 4), "flops": 0}
    if case["kind"] == "latent-append":
        nbytes = rows * (2 * 2 * ROW + 2 * 2 * hq * ROT + 4 * ROT)
        return {"bytes": nbytes, "flops": rows * (4 * LATENT + 3 * ROT * (hq + 1))}
    # (drafts that a row's mask leaves out are at most n of its ctx keys; they are counted as seen)
    if case["kind"] == "tree":
        return {"bytes": int(ctx.sum()) * 2 * 2 * hkv * D + 2 * 2 * rows * hq * D + tables,
                "flops": 4 * hq * D * int((n * ctx).sum())}
    if case["kind"] == "latent":
        return {"bytes": int(ctx.sum()) * 2 * ROW + 2 * rows * hq * (ROW + LATENT) + tables,
                "flops": 2 * hq * (ROW + LATENT) * int((n * ctx).sum())}
    pairs = int((n * c0 + n * (n + 1) // 2).sum())
    return {"bytes": int(ctx.sum()) * 2 * ROW + 2 * rows * hq * (2 * D + ROT) + 2 * hq * 2 * D * LATENT + tables,
            "flops": 2 * hq * (2 * D + ROT) * pairs + 2 * hq * 2 * D * LATENT * int(ctx.sum())}


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 250)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

class _State:
    pass


def _randn(gen, shape, gain=1.0):
    """bf16 N(0, gain) values on the GPU, a slab at a time (a pool may hold billions)."""
    out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = out.view(-1)
    slab = 1 << 27
    for i in range(0, flat.numel(), slab):
        flat[i:i + slab] = torch.randn(min(slab, flat.numel() - i), generator=gen, device="cuda") * gain
    return out


def _tables(rng, ctx, dirs, num_blocks):
    """Random physical blocks; where the last blocks of a request that fills from
    the left and its neighbour that fills from the right fit into one, they share it."""
    need = (ctx + BLOCK - 1) // BLOCK
    tables = np.full((len(ctx), int(need.max())), -1, dtype=np.int32)
    ids = rng.permutation(num_blocks).astype(np.int32)
    at = 0
    for s, m in enumerate(need):
        share = (s > 0 and dirs[s] < 0 < dirs[s - 1] and ctx[s] % BLOCK and ctx[s - 1] % BLOCK
                 and ctx[s] % BLOCK + ctx[s - 1] % BLOCK <= BLOCK)
        fresh = int(m) - (1 if share else 0)
        tables[s, :fresh] = ids[at:at + fresh]
        at += fresh
        if share:
            tables[s, m - 1] = tables[s - 1, need[s - 1] - 1]
    return tables


def _trees(rng, n):
    """Parents of the drafts of every sequence (-1: the last cached token), breadth first,
    and each draft's row of bits, itself and its ancestors, in 64-bit words."""
    words = max(1, (int(n.max()) + 63) // 64)
    parents, rows = [], []
    for m in n:
        up = np.sort(np.minimum(rng.integers(-1, np.maximum(np.arange(m) // 2, 1)), np.arange(m) - 1))
        seen = []
        for j in range(m):
            seen.append((1 << j) | (seen[up[j]] if up[j] >= 0 else 0))
        parents.append(up)
        rows += [[(x >> (64 * w)) & ((1 << 64) - 1) for w in range(words)] for x in seen]
    return parents, np.array(rows, dtype=np.uint64).view(np.int64)


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    hq, hkv = case["hq"], case["hkv"]
    st = _State()
    st.case, st.kind = case, case["kind"]
    n, c0 = _lengths(case)
    S, ctx = len(n), n + c0
    dirs = np.where(np.arange(S) % 2 == 0, 1, -1).astype(np.int8)
    num_blocks = int(math.ceil(int(((ctx + BLOCK - 1) // BLOCK).sum()) / 0.9))
    tables = _tables(rng, ctx, dirs, num_blocks)
    if case["direction"] == "table":
        per = np.repeat(dirs[:, None], tables.shape[1], axis=1)
        full = np.arange(tables.shape[1])[None, :] < (ctx // BLOCK)[:, None]
        dirs = np.where(full & (rng.random(tables.shape) < 0.5), -per, per).astype(np.int8)
    cu = np.concatenate([[0], np.cumsum(n)])
    st.S, st.max_ctx, st.total_ctx, st.max_n, st.rows = S, int(ctx.max()), int(ctx.sum()), int(n.max()), int(cu[-1])
    st.n_host, st.ctx_host = n, ctx
    st.tables, st.dir, st.ctx, st.cu = up(tables), up(dirs), up(ctx.astype(np.int32)), up(cu.astype(np.int32))
    latent = st.kind.startswith("latent") or (st.kind == "commit" and case["pool"] == "latent")
    if latent:
        st.pool = _randn(gen, (num_blocks, BLOCK, ROW))
    else:
        st.k_pool, st.v_pool = (_randn(gen, (num_blocks, hkv, BLOCK, D)) for _ in range(2))
    parents, bits = _trees(rng, n) if case["mask"] == "tree" or st.kind == "commit" else (None, None)
    st.mask = up(bits) if case["mask"] == "tree" and st.kind in ("tree", "latent") else None
    if st.kind == "commit":
        # a path down each tree, as far as the sequence's accepted count or its leaf
        path, lens = np.full((S, 8), -1, dtype=np.int32), np.zeros(S, dtype=np.int32)
        for s, most in enumerate(_accepted(case, n)):
            at = -1
            for i in range(most):
                down = np.nonzero(parents[s] == at)[0]
                if not len(down):
                    down = np.arange(at + 1, n[s])       # (a leaf: any later draft, to keep the count)
                    if not len(down):
                        break
                at = path[s, i] = rng.choice(down)
                lens[s] = i + 1
        st.path, st.path_lens = up(path), up(lens)
    elif st.kind == "tree":
        st.q = _randn(gen, (st.rows, hq, D))
        st.out = torch.empty_like(st.q)
    elif st.kind == "latent":
        # (a score's spread is that of the model's own 192 dims, whose scale it gets)
        st.q = _randn(gen, (st.rows, hq, ROW), 0.6)
        st.out = torch.empty((st.rows, hq, LATENT), dtype=torch.bfloat16, device="cuda")
    elif st.kind == "latent-prefill":
        st.q = _randn(gen, (st.rows, hq, D + ROT))
        st.out = torch.empty((st.rows, hq, D), dtype=torch.bfloat16, device="cuda")
        st.w = _randn(gen, (hq, 2 * D, LATENT), LATENT ** -0.5)
    else:
        st.pos0 = up(c0.astype(np.int32))
        st.kv = _randn(gen, (st.rows, 3 * LATENT + ROW))[:, 3 * LATENT:]       # part of a projection's output
        st.norm = (1.0 + 0.1 * torch.randn(LATENT, generator=gen, device="cuda")).bfloat16()
        st.eps = 1e-6
        st.q = _randn(gen, (st.rows, hq, D + ROT))
        st.q_rot = st.q[:, :, D:]
        if case["q"] == "absorbed":
            st.q_all = torch.zeros((st.rows, hq, ROW), dtype=torch.bfloat16, device="cuda")
            st.q_out = st.q_all[:, :, LATENT:]
        else:
            st.q_all, st.q_out = st.q, st.q_rot
        half = ROT // 2
        angles = np.arange(st.max_ctx)[:, None] * (10000.0 ** (-np.arange(half) / half))[None, :]
        st.table = up(np.concatenate([np.cos(angles), np.sin(angles)], axis=1).astype(np.float32))
    return st


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _slots(st, seqs, pos):
    """Block and slot of positions of sequences (tensors of one shape)."""
    e = pos // BLOCK
    left = (st.dir[seqs, e] if st.dir.dim() == 2 else st.dir[seqs]) > 0
    return st.tables[seqs, e].long(), torch.where(left, pos % BLOCK, BLOCK - 1 - pos % BLOCK)


def _context_slots(st):
    """Blocks and slots of every sequence's positions, [S][max_ctx]; those past a context repeat its last one."""
    seqs = torch.arange(st.S, device="cuda")[:, None]
    pos = torch.minimum(torch.arange(st.max_ctx, device="cuda")[None, :], (st.ctx.long() - 1)[:, None])
    return _slots(st, seqs.expand(pos.shape), pos)


def _padded_rows(st):
    """Row of q of (sequence, new row), [S][max_n], and which of them are there."""
    n = (st.cu[1:] - st.cu[:-1]).long()
    j = torch.arange(st.max_n, device="cuda")[None, :]
    return st.cu[:-1].long()[:, None] + torch.minimum(j, n[:, None] - 1), j < n[:, None]


def _seen(st):
    """Which positions each padded row sees, [S][max_ctx][max_n]."""
    row, _ = _padded_rows(st)
    n = (st.cu[1:] - st.cu[:-1]).long()
    draft = torch.arange(st.max_ctx, device="cuda")[None, :] - (st.ctx.long() - n)[:, None]      # [S][ctx]
    if st.mask is None:
        return draft[:, :, None] <= (row - st.cu[:-1].long()[:, None])[:, None, :]
    at = draft.clamp(0, 64 * st.mask.shape[1] - 1)[:, :, None].expand(-1, -1, st.max_n)
    word = st.mask[row].transpose(1, 2).gather(1, at // 64)                                      # [S][ctx][n]
    bit = (word >> (at % 64)) & 1
    return (draft[:, :, None] < 0) | ((bit == 1) & (draft < n[:, None])[:, :, None])


def _softmax(w, seen):
    """Weights over dim 2 of [S][heads][keys][rows][...]: zeros where nothing is seen."""
    w = w.masked_fill_(~seen, -math.inf)
    w = torch.exp(w - w.amax(2, keepdim=True).clamp(min=-1e30))
    return w, w.sum(2).clamp(min=1e-30)


def _plain_tree(st):
    hq, hkv = st.case["hq"], st.case["hkv"]
    S, m, G = st.S, st.max_n, hq // hkv
    row, real = _padded_rows(st)
    blk, slot = _context_slots(st)
    q = st.q[row].float().view(S, m, hkv, G, D).permute(0, 2, 4, 1, 3).reshape(S, hkv, D, m * G)
    w = (st.k_pool[blk, :, slot].float().permute(0, 2, 1, 3).contiguous() @ q) / math.sqrt(D)
    w, total = _softmax(w.view(S, hkv, st.max_ctx, m, G), _seen(st)[:, None, :, :, None])
    w = w.view(S, hkv, st.max_ctx, m * G).transpose(2, 3).contiguous()
    y = w @ st.v_pool[blk, :, slot].float().permute(0, 2, 1, 3).contiguous()
    y = (y / total.view(S, hkv, m * G, 1)).view(S, hkv, m, G, D).permute(0, 2, 1, 3, 4).reshape(S, m, hq, D)
    return {"out": y[real].to(st.q.dtype)}


def _plain_commit(st):
    S, most = st.path.shape
    n = (st.cu[1:] - st.cu[:-1]).long()
    i = torch.arange(most, device="cuda")[None, :].expand(S, -1)
    seqs = torch.arange(S, device="cuda")[:, None].expand(-1, most)
    c0 = (st.ctx.long() - n)[:, None]
    keep = (i < st.path_lens[:, None]) & (i < n[:, None]) & (st.path >= 0) & (st.path < n[:, None])
    src = _slots(st, seqs[keep], (c0 + st.path)[keep])
    dst = _slots(st, seqs[keep], (c0 + i)[keep])
    if st.case["pool"] == "latent":
        st.pool[dst] = st.pool[src]
        return {"pool": st.pool}
    st.k_pool[dst[0], :, dst[1]] = st.k_pool[src[0], :, src[1]]
    st.v_pool[dst[0], :, dst[1]] = st.v_pool[src[0], :, src[1]]
    return {"k_pool": st.k_pool, "v_pool": st.v_pool}


def _turned(x, rows):
    half = ROT // 2
    a, b, cos, sin = x[..., :half], x[..., half:], rows[..., :half], rows[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _plain_latent_append(st):
    t = torch.arange(st.rows, device="cuda")
    seq = torch.searchsorted(st.cu[1:].long(), t, right=True)
    pos = st.pos0[seq].long() + t - st.cu[seq].long()
    x = st.kv.float()
    c = x[:, :LATENT]
    c = c * torch.rsqrt((c * c).mean(-1, keepdim=True) + st.eps) * st.norm.float()
    blk, slot = _slots(st, seq, pos)
    st.pool[blk, slot] = torch.cat([c, _turned(x[:, LATENT:], st.table[pos])], dim=-1).to(st.pool.dtype)
    st.q_out.copy_(_turned(st.q_rot.float(), st.table[pos][:, None]).to(st.q.dtype))
    return {"pool": st.pool, "q": st.q_all}


def _plain_latent(st):
    hq, S, m = st.case["hq"], st.S, st.max_n
    row, real = _padded_rows(st)
    c = st.pool[_context_slots(st)].float()                                       # [S][ctx][576]
    q = st.q[row].float().view(S, m * hq, ROW).transpose(1, 2)
    w = (c @ q) / math.sqrt(D + ROT)                                              # [S][ctx][m hq]
    w, total = _softmax(w.view(S, 1, st.max_ctx, m, hq), _seen(st)[:, None, :, :, None])
    w = w.view(S, st.max_ctx, m * hq).transpose(1, 2).contiguous()
    y = (w @ c[..., :LATENT].contiguous()) / total.view(S, m * hq, 1)
    return {"out": y.view(S, m, hq, LATENT)[real].to(st.q.dtype)}


def _plain_latent_prefill(st):
    hq, S, m, ctx = st.case["hq"], st.S, st.max_n, st.max_ctx
    row, real = _padded_rows(st)
    c = st.pool[_context_slots(st)].float()
    kv = (c[..., :LATENT].reshape(S * ctx, LATENT) @ st.w.float().view(hq * 2 * D, LATENT).t()).view(S, ctx, hq, 2 * D)
    k = torch.cat([kv[..., :D], c[:, :, None, LATENT:].expand(-1, -1, hq, -1)], dim=-1).permute(0, 2, 1, 3).contiguous()
    q = st.q[row].float().permute(0, 2, 3, 1)                                     # [S][hq][192][m]
    w, total = _softmax((k @ q) / math.sqrt(D + ROT), _seen(st)[:, None])
    w = w.transpose(2, 3).contiguous() @ kv[..., D:].permute(0, 2, 1, 3).contiguous()
    return {"out": (w / total[..., None]).permute(0, 2, 1, 3)[real].to(st.q.dtype)}


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------

def _kept(st):
    """What a serving loop makes once and keeps: the rotation, the workspace."""
    from paper_2504_09590_amd import bros
    hq, size = st.case["hq"], 0
    if st.kind == "latent-append":
        st.rope = bros.Rope(st.table)
    elif st.kind == "tree":
        size = bros.bros_attn_workspace_size(bros.BROS_WS_TREE, bros.BROS_BF16, st.rows, hq, D, st.max_ctx)
    elif st.kind == "latent":
        size = bros.bros_attn_workspace_size(bros.BROS_WS_LATENT, bros.BROS_BF16, st.rows, hq, ROW, st.max_ctx)
    elif st.kind == "latent-prefill":
        size = bros.bros_latent_prefill_workspace_size(st.S, st.total_ctx, hq)
    st.ws = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None
    st.bros = bros


def _own(st):
    if not hasattr(st, "bros"):
        _kept(st)
    bros = st.bros
    if st.kind == "tree":
        bros.bros_attn_tree(st.out, st.q, st.cu, st.max_n, st.k_pool, st.v_pool, st.tables, st.dir, None, st.ctx, st.max_ctx,
                            mask=st.mask, workspace=st.ws)
        return {"out": st.out}
    if st.kind == "commit":
        if st.case["pool"] == "latent":
            bros.bros_tree_commit(st.pool, None, st.tables, st.dir, None, st.ctx, st.cu, st.path, st.path_lens)
            return {"pool": st.pool}
        bros.bros_tree_commit(st.k_pool, st.v_pool, st.tables, st.dir, None, st.ctx, st.cu, st.path, st.path_lens)
        return {"k_pool": st.k_pool, "v_pool": st.v_pool}
    if st.kind == "latent-append":
        bros.bros_latent_append(st.q_out, st.q_rot, st.kv, st.pool, st.tables, st.dir, None, st.pos0, st.cu, rope=st.rope,
                                norm=st.norm, eps=st.eps)
        return {"pool": st.pool, "q": st.q_all}
    if st.kind == "latent":
        bros.bros_attn_latent(st.out, st.q, st.cu, st.max_n, st.pool, st.tables, st.dir, None, st.ctx, st.max_ctx,
                              mask=st.mask, workspace=st.ws)
        return {"out": st.out}
    bros.bros_attn_latent_prefill(st.out, st.q, st.cu, st.max_n, st.w, st.pool, st.tables, st.dir, None, st.ctx, st.max_ctx,
                                  st.total_ctx, workspace=st.ws)
    return {"out": st.out}


def run(st):
    if own:
        return _own(st)
    plain = {"tree": _plain_tree, "commit": _plain_commit, "latent-append": _plain_latent_append, "latent": _plain_latent,
             "latent-prefill": _plain_latent_prefill}
    return plain[st.kind](st)


# ---------------------------------------------------------------------------
# in 64 bits
# ---------------------------------------------------------------------------

def _places(st, s, pos):
    """Blocks and slots of positions of one sequence, from host copies of the metadata."""
    e = pos // BLOCK
    d = st.dirs_np[s, e] if st.dirs_np.ndim == 2 else st.dirs_np[s]
    return (torch.from_numpy(st.tables_np[s, e].astype(np.int64)).cuda(),
            torch.from_numpy(np.where(d > 0, pos % BLOCK, 15 - pos % BLOCK)).cuda())


def _exact_visible(st, s, lo, n, ctx):
    """Which of the ctx positions row j of sequence s sees, [n][ctx]."""
    c0 = ctx - n
    see = np.zeros((n, ctx), dtype=bool)
    for j in range(n):
        if st.mask is None:
            see[j, :c0 + j + 1] = True
        else:
            see[j, :c0] = True
            bits = sum((int(w) & ((1 << 64) - 1)) << (64 * i) for i, w in enumerate(st.mask_np[lo + j]))
            see[j, c0:] = [(bits >> i) & 1 for i in range(n)]
    return torch.from_numpy(see).cuda()


def _exact_attention(q, k, v, see, scale):
    """q [rows][heads][dims], k and v [keys][heads or 1][dims], all fp64; see [rows][keys]."""
    y = torch.empty((q.shape[0], q.shape[1], v.shape[2]), dtype=torch.float64, device="cuda")
    per = q.shape[1] // k.shape[1]
    for h in range(q.shape[1]):
        w = torch.mm(q[:, h], k[:, h // per].t().contiguous()) * scale
        w = w.masked_fill(~see, -math.inf).softmax(-1)
        y[:, h] = torch.mm(torch.where(see.any(1, keepdim=True), w, torch.zeros_like(w)), v[:, h // per])
    return y


def exact(case, seed):
    st = prepare(case, seed)
    if st.kind == "commit":
        return _plain_commit(st)
    st.tables_np, st.dirs_np, st.mask_np = st.tables.cpu().numpy(), st.dir.cpu().numpy(), None if st.mask is None else st.mask.cpu().numpy()
    cu = st.cu.cpu().numpy()
    if st.kind == "latent-append":
        pool, q_all = st.pool.double(), st.q_all.double()
        at = D if case["q"] == "place" else LATENT
        half, pos0 = ROT // 2, st.pos0.cpu().numpy()
        for s in range(st.S):
            lo, hi = int(cu[s]), int(cu[s + 1])
            p = np.arange(hi - lo) + pos0[s]
            blk, slot = _places(st, s, p)
            x, turn = st.kv[lo:hi].double(), st.table[torch.from_numpy(p).cuda()].double()
            c = x[:, :LATENT] / (x[:, :LATENT].square().mean(-1, keepdim=True) + st.eps).sqrt() * st.norm.double()
            pool[blk, slot, :LATENT] = c
            q = st.q_rot[lo:hi].double()
            for i in range(half):
                co, si = turn[:, i], turn[:, half + i]
                a, b = x[:, LATENT + i], x[:, LATENT + half + i]
                pool[blk, slot, LATENT + i], pool[blk, slot, LATENT + half + i] = a * co - b * si, a * si + b * co
                a, b, co, si = q[:, :, i], q[:, :, half + i], co[:, None], si[:, None]
                q_all[lo:hi, :, at + i], q_all[lo:hi, :, at + half + i] = a * co - b * si, a * si + b * co
        return {"pool": pool, "q": q_all}
    out = torch.empty(st.out.shape, dtype=torch.float64, device="cuda")
    for s in range(st.S):
        lo, n, ctx = int(cu[s]), int(st.n_host[s]), int(st.ctx_host[s])
        see = _exact_visible(st, s, lo, n, ctx)
        blk, slot = _places(st, s, np.arange(ctx))
        q = st.q[lo:lo + n].double()
        if st.kind == "tree":
            out[lo:lo + n] = _exact_attention(q, st.k_pool[blk, :, slot].double(), st.v_pool[blk, :, slot].double(), see, D ** -0.5)
            continue
        c = st.pool[blk, slot].double()
        if st.kind == "latent":
            # every row and head against the same keys: rows of one product
            see = see.repeat_interleave(case["hq"], dim=0)
            y = _exact_attention(q.reshape(-1, 1, ROW), c[:, None], c[:, None, :LATENT], see, (D + ROT) ** -0.5)
            out[lo:lo + n] = y.view(n, case["hq"], LATENT)
            continue
        for h in range(case["hq"]):
            kv = torch.mm(c[:, :LATENT], st.w[h].double().t().contiguous())
            k = torch.cat([kv[:, :D], c[:, LATENT:]], dim=1)
            out[lo:lo + n, h] = _exact_attention(q[:, h:h + 1], k[:, None], kv[:, None, D:], see, (D + ROT) ** -0.5)[:, 0]
    return {"out": out}
