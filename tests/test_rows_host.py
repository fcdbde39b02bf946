"""What the calls over drafted tokens and over a latent cache turn down (no GPU: every call here is
refused before a launch, or has nothing to do), and the rule that picks their units' width."""

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from tests.rows_helpers import TEAMS_CHUNKS, TEAMS_TREE, WAYS_LATENT, WAYS_TREE

bros = pytest.importorskip("paper_2504_09590_amd.bros", reason="libbros_attn.so not built")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_09590_amd", "csrc")

NULL, SHAPE, DTYPE, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4, -5
A = 1 << 24          # an address that nothing reads
HUGE = 1 << 40       # bytes of a workspace that nothing writes


def status(fn, base, **kw):
    assert set(kw) <= set(base), set(kw) - set(base)
    got = getattr(bros.LIB, fn)(*{**base, **kw}.values())
    if got:
        assert fn in bros.LIB.bros_last_error().decode()
    return got


TREE = dict(out=A, q=A, cu_q=A, rows=8, max_q_len=4, mask=A, words=1, k_pool=A, v_pool=A, num_blocks=10, tables=A, width=4, dir=A,
            cls=None, per_entry=0, ctx=A, max_ctx=64, seqs=2, hq=8, hkv=2, dim=128, block=16, scale=0.0, dtype=1, ws=A, bytes=HUGE,
            stream=None)
LATENT = dict(out=A, q=A, cu_q=A, rows=8, max_q_len=4, mask=A, words=1, pool=A, num_blocks=10, tables=A, width=4, dir=A, cls=None,
              per_entry=0, ctx=A, max_ctx=64, seqs=2, hq=8, row_dim=576, block=16, scale=0.0, dtype=1, ws=A, bytes=HUGE, stream=None)
PREFILL = dict(out=A, q=A, cu_q=A, rows=8, max_q_len=4, w_kv=A, pool=A, num_blocks=10, tables=A, width=4, dir=A, cls=None,
               per_entry=0, ctx=A, max_ctx=64, total=100, seqs=2, hq=8, row_dim=576, block=16, scale=0.0, dtype=1, ws=A, bytes=HUGE,
               stream=None)
COMMIT = dict(k_pool=A, v_pool=A, num_blocks=10, tables=A, width=4, dir=A, cls=None, per_entry=0, ctx=A, cu_q=A, path=A, lens=A,
              max_path=4, seqs=2, hkv=2, row_dim=128, block=16, dtype=1, stream=None)
APPEND = dict(q_out=16 * A, q=2 * A, out_stride=8 * 576, out_head=576, q_stride=8 * 192, q_head=192, kv=4 * A, kv_stride=576, tokens=5,
              hq=8, norm=A, eps=1e-6, rope=None, rope_pos=None, pool=64 * A, num_blocks=10, tables=A, width=4, dir=A, cls=None,
              per_entry=0, pos0=A, cu_new=A, seqs=2, row_dim=576, block=16, dtype=1, stream=None)
ROWS_CALLS = [("bros_attn_tree", TREE), ("bros_attn_latent", LATENT), ("bros_attn_latent_prefill", PREFILL)]

COMMON = [
    (dict(dtype=7), DTYPE), (dict(dtype=0), UNSUPPORTED), (dict(block=32), UNSUPPORTED), (dict(hq=0), SHAPE), (dict(hq=-8), SHAPE),
    (dict(hq=2048), UNSUPPORTED), (dict(seqs=-1), SHAPE), (dict(rows=-1), SHAPE), (dict(max_q_len=-1), SHAPE), (dict(max_ctx=-1), SHAPE),
    (dict(max_q_len=0), SHAPE), (dict(out=None), NULL), (dict(q=None), NULL), (dict(ctx=None), NULL), (dict(tables=None), NULL),
    (dict(width=0), SHAPE), (dict(num_blocks=0), SHAPE), (dict(out=A + 8), SHAPE), (dict(q=A + 2), SHAPE),
    (dict(cu_q=A + 2), SHAPE), (dict(ctx=A + 1), SHAPE), (dict(per_entry=2), SHAPE), (dict(ws=None), WORKSPACE), (dict(ws=A + 8), WORKSPACE),
    (dict(bytes=1 << 20), WORKSPACE), (dict(rows=2 ** 31 - 1, max_q_len=2 ** 31 - 1, hq=1024), SHAPE),
]
MASKS = [(dict(words=0), SHAPE), (dict(words=5), SHAPE), (dict(words=1, rows=100, max_q_len=65), SHAPE), (dict(mask=A + 4), SHAPE),
         (dict(cu_q=None), SHAPE)]


@pytest.mark.parametrize("fn,base", ROWS_CALLS)
@pytest.mark.parametrize("kw,want", COMMON)
def test_rows_refusals(fn, base, kw, want):
    if kw.get("hq") == 1024:
        kw = dict(kw, **({"mask": None} if "mask" in base else {}), **({"hkv": 128} if "hkv" in base else {}))
    got = status(fn, base, **kw)
    assert got == want, bros.LIB.bros_last_error().decode()


@pytest.mark.parametrize("fn,base", ROWS_CALLS[:2])
@pytest.mark.parametrize("kw,want", MASKS)
def test_mask_refusals(fn, base, kw, want):
    assert status(fn, base, **kw) == want


def test_pools_and_heads():
    for kw, want in [(dict(k_pool=None), NULL), (dict(v_pool=None), NULL), (dict(k_pool=A + 8), SHAPE), (dict(hkv=3), SHAPE),
                     (dict(hkv=0), SHAPE), (dict(dim=64), UNSUPPORTED)]:
        assert status("bros_attn_tree", TREE, **kw) == want, kw
    for fn, base in ROWS_CALLS[1:]:
        for kw, want in [(dict(pool=None), NULL), (dict(pool=A + 8), SHAPE), (dict(row_dim=512), UNSUPPORTED)]:
            assert status(fn, base, **kw) == want, kw
    for kw, want in [(dict(w_kv=None), NULL), (dict(w_kv=A + 2), SHAPE), (dict(cu_q=None, rows=2), NULL), (dict(total=-1), SHAPE),
                     (dict(total=2 ** 31 - 1), SHAPE)]:
        assert status("bros_attn_latent_prefill", PREFILL, **kw) == want, kw


def test_calls_with_nothing_to_do():
    for fn, base in ROWS_CALLS:
        assert status(fn, base, seqs=0) == 0 and status(fn, base, rows=0, ws=None, out=None) == 0
    assert status("bros_tree_commit", COMMIT, seqs=0) == 0 and status("bros_tree_commit", COMMIT, max_path=0, path=None) == 0
    assert status("bros_latent_append", APPEND, tokens=0, kv=None) == 0


def test_commit_refusals():
    for kw, want in [(dict(dtype=3), DTYPE), (dict(block=8), UNSUPPORTED), (dict(hkv=0), SHAPE), (dict(row_dim=64), UNSUPPORTED),
                     (dict(row_dim=576), SHAPE), (dict(row_dim=576, hkv=1), SHAPE), (dict(row_dim=576, hkv=1, v_pool=None, dtype=0), UNSUPPORTED),
                     (dict(hkv=16385), UNSUPPORTED), (dict(seqs=-1), SHAPE), (dict(max_path=-1), SHAPE), (dict(max_path=257), UNSUPPORTED),
                     (dict(v_pool=None), NULL), (dict(k_pool=None), NULL), (dict(path=None), NULL), (dict(lens=None), NULL),
                     (dict(cu_q=None), NULL), (dict(ctx=None), NULL), (dict(tables=None), NULL), (dict(num_blocks=0), SHAPE),
                     (dict(k_pool=A + 8), SHAPE), (dict(path=A + 2), SHAPE), (dict(lens=A + 1), SHAPE)]:
        assert status("bros_tree_commit", COMMIT, **kw) == want, kw


def test_append_refusals():
    table = torch.zeros((9, 64))
    rope = bros.Rope(table)
    wide = bros.Rope(torch.zeros((9, 128)))
    for kw, want in [(dict(dtype=0), UNSUPPORTED), (dict(dtype=5), DTYPE), (dict(block=32), UNSUPPORTED), (dict(row_dim=512), UNSUPPORTED),
                     (dict(tokens=-1), SHAPE), (dict(seqs=-1), SHAPE), (dict(hq=-1), SHAPE), (dict(hq=16385), UNSUPPORTED),
                     (dict(q=None), NULL), (dict(q_out=None), NULL), (dict(hq=0), SHAPE), (dict(seqs=0), SHAPE), (dict(kv=None), NULL),
                     (dict(pool=None), NULL), (dict(pos0=None), NULL), (dict(cu_new=None), NULL), (dict(tables=None), NULL),
                     (dict(kv_stride=568), SHAPE), (dict(kv_stride=580), SHAPE), (dict(q_head=56), SHAPE), (dict(q_stride=7 * 192 + 56), SHAPE),
                     (dict(out_head=63), SHAPE), (dict(out_stride=64), SHAPE), (dict(kv=4 * A + 8), SHAPE), (dict(pool=A + 2), SHAPE),
                     (dict(norm=A + 4), SHAPE), (dict(q=2 * A + 2), SHAPE), (dict(pos0=A + 2), SHAPE),
                     (dict(rope=wide.ref, rope_pos=A), SHAPE)]:
        assert status("bros_latent_append", APPEND, **kw) == want, kw
    assert rope.axes == 1


def overlaps(**kw):
    """Whether the call is refused for its rows."""
    got = status("bros_latent_append", APPEND, **kw)
    assert got == SHAPE
    return "overlaps" in bros.LIB.bros_last_error().decode()


def test_append_overlaps():
    row = 192
    same = dict(q_out=2 * A, out_stride=8 * row, out_head=row)
    assert overlaps(q_out=2 * A + 16, out_stride=8 * row, out_head=row)         # q moved by eight values
    assert overlaps(q_out=2 * A, out_stride=8 * row + 8, out_head=row)          # q, other strides
    assert overlaps(q_out=2 * A, out_stride=16 * row, out_head=2 * row)
    assert overlaps(**dict(same, kv=2 * A + 2 * (4 * 8 * row) - 16))            # kv's first rows over q's last token
    assert overlaps(q_out=4 * A + 1024, out_stride=64 * 8, out_head=64)         # over kv's rotated dims
    assert overlaps(tokens=2 ** 31 - 1, q_stride=1 << 40, out_stride=1 << 40)   # no product of these goes around


@pytest.fixture(scope="module")
def ways(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("ways")
    (d / "ways.cpp").write_text("""
#include "plan.h"
extern "C" int way(int latent, long long columns, long long segments, long long keys, int cus) {
  return latent ? bros::pick_rows_way(bros::kLatentWays, columns, segments, keys, cus) : bros::pick_rows_way(bros::kTreeWays, columns, segments, keys, cus);
}
extern "C" long long planned(long long max_rows, long long rows, long long seqs) { return bros::planned_rows(max_rows, rows, seqs); }
extern "C" int team(long long tiles, long long rows, long long max_rows, long long seqs) { return bros::rows_team(tiles, rows, max_rows, seqs); }
""")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-ftrapv", "-shared", "-fPIC", "-I", CSRC, str(d / "ways.cpp"),
                    "-o", str(d / "ways.so")], check=True)
    lib = ctypes.CDLL(str(d / "ways.so"))
    L = ctypes.c_longlong
    lib.way.argtypes = [ctypes.c_int, L, L, L, ctypes.c_int]
    lib.team.argtypes = [L, L, L, L]
    lib.planned.argtypes, lib.planned.restype = [L, L, L], L
    return lib


def test_the_gpu_tests_shapes_take_every_way(ways):
    """Card of 256 compute units; a context counts by its last block."""
    blocks = lambda c0, n: 16 * max((c + m + 15) // 16 for c, m in zip(c0, n))  # noqa: E731
    got = [ways.way(0, ways.planned(max(n), sum(n), len(n)) * hq // hkv, len(n) * hkv, blocks(c0, n), 256) for _, n, c0, hq, hkv in WAYS_TREE]
    assert got == [w for w, *_ in WAYS_TREE] and set(got) == {0, 1, 2}
    got = [ways.way(1, ways.planned(max(n), sum(n), len(n)) * hq, len(n), blocks(c0, n), 256) for _, n, c0, hq in WAYS_LATENT]
    assert got == [w for w, *_ in WAYS_LATENT] and set(got) == {0, 1, 2, 3}


def test_the_gpu_tests_shapes_take_every_team(ways):
    blocks = lambda c0, n: 16 * max((c + m + 15) // 16 for c, m in zip(c0, n))  # noqa: E731
    for team, n, c0, hq, hkv in TEAMS_TREE:
        columns = ways.planned(max(n), sum(n), len(n)) * hq // hkv
        assert ways.way(0, columns, len(n) * hkv, blocks(c0, n), 256) == 2 and ways.team(-(-columns // 128), sum(n), ways.planned(max(n), sum(n), len(n)), len(n)) == team
    for team, n, c0, hq in TEAMS_CHUNKS:
        assert max(a + b for a, b in zip(n, c0)) > 1024 and ways.team(-(-ways.planned(max(n), sum(n), len(n)) // 128), sum(n), ways.planned(max(n), sum(n), len(n)), len(n)) == team
    assert ways.planned(256, 8 * 16, 16) == 16 and ways.planned(32, 400, 16) == 32 and ways.planned(1, 7, 9) == 1
    assert ways.planned(2 ** 31 - 1, 2 ** 31 - 1, 1) == 2 ** 31 - 1
    assert ways.team(16, 16 * 4, 256, 16) == 1      # a bound far above the rows there are
    assert ways.team(1, 5, 5, 1) == 1 and ways.team(3, 300, 300, 1) == 1 and ways.team(2, 300, 256, 2) == 1


def test_ways_hold_for_any_sizes(ways):
    rng = np.random.default_rng(0)
    for latent, widths in ((0, (32, 64, 128)), (1, (16, 32, 64, 128))):
        for _ in range(2000):
            columns, segments, keys = (int(2 ** rng.uniform(0, 31)) for _ in range(3))
            w = ways.way(latent, columns, segments, keys, int(rng.integers(1, 257)))
            assert 0 <= w < len(widths) and (w == 0 or widths[w - 1] < columns)
        assert ways.way(latent, 1, 1, 0, 256) == 0
        big = ways.way(latent, 2 ** 30, 2 ** 31 - 1, 2 ** 31 - 1, 1)
        assert widths[big] == 128


# --- the binding ---------------------------------------------------------------

def t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def ints(*values):
    return torch.tensor(values, dtype=torch.int32)


def py_call(fn, **kw):
    seq = dict(block_tables=torch.zeros((2, 4), dtype=torch.int32), dir=torch.ones(2, dtype=torch.int8), cls=None)
    base = {
        "bros_attn_tree": dict(out=t(5, 8, 128), q=t(5, 8, 128), cu_q=ints(0, 2, 5), max_q_len=3, k_pool=t(9, 2, 16, 128),
                               v_pool=t(9, 2, 16, 128), **seq, ctx_lens=ints(9, 9), max_ctx=9, mask=torch.zeros((5, 1), dtype=torch.int64)),
        "bros_attn_latent": dict(out=t(5, 8, 512), q=t(5, 8, 576), cu_q=ints(0, 2, 5), max_q_len=3, pool=t(9, 16, 576), **seq,
                                 ctx_lens=ints(9, 9), max_ctx=9, mask=torch.zeros((5, 1), dtype=torch.int64)),
        "bros_attn_latent_prefill": dict(out=t(5, 8, 128), q=t(5, 8, 192), cu_q=ints(0, 2, 5), max_q_len=3, w_kv=t(8, 256, 512),
                                         pool=t(9, 16, 576), **seq, ctx_lens=ints(9, 9), max_ctx=9, total_ctx=18),
        "bros_tree_commit": dict(k_pool=t(9, 2, 16, 128), v_pool=t(9, 2, 16, 128), **seq, ctx_lens=ints(9, 9), cu_q=ints(0, 2, 5),
                                 path=torch.zeros((2, 3), dtype=torch.int32), path_lens=ints(1, 1)),
        "bros_latent_append": dict(q_out=t(5, 8, 64), q=t(5, 8, 192)[..., 128:], kv=t(5, 576), pool=t(9, 16, 576), **seq,
                                   pos0=ints(3, 4), cu_new=ints(0, 2, 5)),
    }[fn]
    assert set(kw) <= set(base) | {"rope", "rope_pos", "norm", "eps", "workspace"}
    getattr(bros, fn)(**{**base, **kw})


CALLS = ["bros_attn_tree", "bros_attn_latent", "bros_attn_latent_prefill", "bros_tree_commit", "bros_latent_append"]


@pytest.mark.parametrize("fn", CALLS)
def test_binding_asks_for_the_device(fn):
    with pytest.raises(ValueError, match="current device"):
        py_call(fn)


@pytest.mark.parametrize("fn,kw,words", [
    ("bros_attn_tree", dict(q=t(5, 8, 64)), "q must be"), ("bros_attn_tree", dict(q=t(5, 8, 128, dtype=torch.float16)), "q must be"),
    ("bros_attn_tree", dict(v_pool=t(9, 1, 16, 128)), "q must be"), ("bros_attn_tree", dict(out=t(4, 8, 128)), "out must"),
    ("bros_attn_tree", dict(mask=torch.zeros((5, 1), dtype=torch.int32)), "mask"), ("bros_attn_tree", dict(mask=torch.zeros(5, dtype=torch.int64)), "mask"),
    ("bros_attn_tree", dict(mask=torch.zeros((4, 1), dtype=torch.int64)), "mask"), ("bros_attn_tree", dict(cu_q=None), "5"),
    ("bros_attn_tree", dict(cu_q=ints(0, 5)), "int32"), ("bros_attn_tree", dict(ctx_lens=torch.zeros(2, dtype=torch.int64)), "int32"),
    ("bros_attn_latent", dict(q=t(5, 8, 512)), "576"), ("bros_attn_latent", dict(out=t(5, 8, 576)), "out must"),
    ("bros_attn_latent", dict(pool=t(9, 1, 16, 576)), "latent pool"), ("bros_attn_latent", dict(pool=t(9, 16, 576, dtype=torch.float32)), "latent pool"),
    ("bros_attn_latent_prefill", dict(q=t(5, 8, 576)), "192"), ("bros_attn_latent_prefill", dict(w_kv=t(8, 256, 576)), "w_kv"),
    ("bros_attn_latent_prefill", dict(w_kv=t(4, 256, 512)), "w_kv"), ("bros_attn_latent_prefill", dict(out=t(5, 8, 192)), "out must"),
    ("bros_tree_commit", dict(v_pool=t(9, 2, 16, 128, dtype=torch.float32)), "one shape and type"), ("bros_tree_commit", dict(v_pool=None), "latent pool"),
    ("bros_tree_commit", dict(path=torch.zeros((3, 3), dtype=torch.int32)), "path"), ("bros_tree_commit", dict(path=torch.zeros((2, 3), dtype=torch.int64)), "path"),
    ("bros_tree_commit", dict(path_lens=ints(1)), "int32"),
    ("bros_latent_append", dict(kv=t(5, 512)), "kv must"), ("bros_latent_append", dict(kv=t(576, 5).t()), "kv must"),
    ("bros_latent_append", dict(q=None), "both q and q_out"), ("bros_latent_append", dict(q_out=None), "both q and q_out"),
    ("bros_latent_append", dict(q=t(5, 64, 8).transpose(1, 2)), "q must"), ("bros_latent_append", dict(q_out=t(5, 7, 64)), "q's shape"),
    ("bros_latent_append", dict(q_out=t(4, 8, 64)), "q_out must"), ("bros_latent_append", dict(norm=t(576)), "norm"),
    ("bros_latent_append", dict(norm=t(512, dtype=torch.float32)), "norm"), ("bros_latent_append", dict(rope_pos=torch.zeros((1, 5), dtype=torch.int32)), "rotation"),
])
def test_binding_refusals(fn, kw, words):
    with pytest.raises(ValueError, match=words):
        py_call(fn, **kw)


def test_workspace_sizes():
    for kind, dim in ((bros.BROS_WS_TREE, 128), (bros.BROS_WS_LATENT, 576)):
        one = bros.bros_attn_workspace_size(kind, bros.BROS_BF16, 1, 1, dim, 0)
        assert one > 0 and one == bros.bros_attn_workspace_size(kind, bros.BROS_BF16, 5000, 128, dim, 1 << 20)
        assert bros.bros_attn_workspace_size(kind, bros.BROS_F32, 1, 1, dim, 0) == 0
        assert bros.bros_attn_workspace_size(kind, bros.BROS_BF16, 1, 1, 64, 0) == 0
    size = bros.bros_latent_prefill_workspace_size
    assert size(0, 100, 4) == size(2, -1, 4) == size(2, 100, 0) == 0
    assert size(2, 100, 4) - size(2, 100, 3) == size(2, 100, 2) - size(2, 100, 1) > 100 * 512
