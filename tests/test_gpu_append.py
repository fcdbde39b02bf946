"""bros_qkv_append and bros_qkv_append_q8 against the fp64 oracle: q rows, the
written slots, and every other byte of the pools as it was."""

import dataclasses

import numpy as np
import pytest

import oracle
from paper_2504_09590_amd import workload as W
from tests import append_helpers as A
from tests.gpu_helpers import announce, require_gpu, with_direction_table

pytestmark = pytest.mark.gpu

MIXED = dict(ctx=[300, 40, 7, 90, 22, 58], cls=[W.RT, W.RT, W.BE, W.BE, W.RT, W.BE], num_prefill=2,
             new_counts=[130, 40, 1, 1, 1, 1])


def mixed(hkv, dtype="bf16", seed=0):
    return W.custom(MIXED["ctx"], MIXED["cls"], hkv, hkv, dtype=dtype, seed=seed, num_prefill=MIXED["num_prefill"],
                    new_counts=MIXED["new_counts"], spare_blocks=3)


def eight_bit_pool(batch, seed=0):
    """Random bytes everywhere: what no token owns may hold anything, NaN codes too."""
    rng = np.random.default_rng(seed)
    shape = (batch.num_blocks, batch.num_kv_heads, 16, batch.head_dim)
    return (rng.integers(0, 256, shape, dtype=np.uint8), rng.integers(0, 256, shape, dtype=np.uint8),
            rng.integers(0, 256, (batch.num_blocks, batch.num_kv_heads, 2, 16), dtype=np.uint8))


def run(r, eight=False, packed=True, pools=None, tables=None, use_cls=False, q_rows=True, in_place=False):
    """One call; returns host (q_out or None, k_pool, v_pool, scales or None) and the pools it started from."""
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    b = r.batch
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    q, k, v = A.device_rows(r, packed)
    q_out = q if in_place else torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    start = pools if pools is not None else (eight_bit_pool(b) if eight else (b.k_pool, b.v_pool))
    dev = [bros._tensor(x, None if eight else r.dtype, "cuda") for x in start]
    meta = (up(b.block_tables if tables is None else tables), None if use_cls else up(b.dir), up(b.cls), up(b.pos0), up(b.cu_new))
    call = bros.bros_qkv_append_q8 if eight else bros.bros_qkv_append
    call(q_out if q_rows else None, q if q_rows else None, k, v, *dev, *meta, **A.options(r))
    torch.cuda.synchronize()
    return (bros.to_host_bits(q_out) if q_rows else None, *(bros.to_host_bits(x) for x in dev)), start


def check(r, got, start, eight=False, stored=None):
    """Everything a call wrote. stored: tokens that have a slot (default all)."""
    b = r.batch
    q_out, k_pool, v_pool = got[:3]
    seq, pos = A.tokens(b)
    (q, q_reach), (k, k_reach) = A.expected(r, seq, pos)
    if q_out is not None:
        A.check_close(q_out, q, q_reach, r.dtype, "q")
    keep = np.arange(len(seq)) if stored is None else stored
    blk, slot = [], []
    for t in keep:
        x, y = oracle.physical_location(b.block_tables, b.dir, int(seq[t]), pos[t:t + 1])
        blk.append(int(x[0]))
        slot.append(int(y[0]))
    blk, slot = np.array(blk, dtype=np.int64), np.array(slot, dtype=np.int64)
    touched = np.zeros((b.num_blocks, 16), dtype=bool)
    touched[blk, slot] = True
    for name, was, now in zip(("k", "v"), start, (k_pool, v_pool)):
        same = was.view(np.uint8) == now.view(np.uint8)
        same = same.reshape(b.num_blocks, b.num_kv_heads, 16, -1).all(-1).transpose(0, 2, 1)
        assert same[~touched].all(), f"{name}_pool: a slot of no new token changed"
    if eight:
        scales = got[3]
        same = (start[2] == scales).transpose(0, 3, 1, 2)
        assert same[~touched].all(), "scales: a slot of no new token changed"
        A.check_codes(k_pool[blk, :, slot], scales[blk, :, 0, slot], k[keep], k_reach[keep], "k")
        # v takes no arithmetic: its codes and scales are the oracle's
        codes, bytes_ = oracle.encode(oracle.widen(r.v, r.dtype)[keep])
        assert (v_pool[blk, :, slot] == codes).all() and (scales[blk, :, 1, slot] == bytes_).all(), "v"
    else:
        A.check_close(k_pool[blk, :, slot], k[keep], k_reach[keep], r.dtype, "k")
        assert (v_pool[blk, :, slot] == r.v[keep]).all(), "v"


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", [(32, 8), (8, 1), (16, 8), (3, 1), (5, 5)])
def test_heads(hq, hkv, dtype, eight):
    r = A.make_rows(mixed(hkv, dtype), hq, dtype, True, True, rotary=128, seed=hq)
    announce(f"append {hq}/{hkv} {dtype} eight={eight}")
    check(r, *run(r, eight), eight)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("rotary,sections", [(0, None), (16, None), (64, None), (96, None), (112, None), (128, None),
                                             (128, (16, 24, 24)), (96, (5, 27, 16)), (64, (31, 1)), (32, (3, 0, 4, 9)),
                                             (128, (64,))])
def test_rotations(rotary, sections, adjacent, eight):
    r = A.make_rows(mixed(2), 4, "bf16", False, False, rotary, adjacent, sections, seed=rotary)
    announce(f"append rotary={rotary} sections={sections} adjacent={adjacent} eight={eight}")
    check(r, *run(r, eight), eight)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_norm,k_norm", [(False, False), (True, False), (False, True), (True, True)])
def test_norms(q_norm, k_norm, dtype, eight):
    r = A.make_rows(mixed(2, dtype), 8, dtype, q_norm, k_norm, rotary=64, adjacent=True, seed=3)
    announce(f"append norms {q_norm} {k_norm} {dtype} eight={eight}")
    check(r, *run(r, eight), eight)


@pytest.mark.parametrize("eight", [False, True])
def test_separate_tensors_classes_and_k_v_alone(eight):
    r = A.make_rows(mixed(2), 4, "bf16", True, True, rotary=128, seed=4)
    announce(f"append separate tensors, directions from classes, eight={eight}")
    check(r, *run(r, eight, packed=False, use_cls=True), eight)
    got, start = run(r, eight, q_rows=False)
    check(r, got, start, eight)


def test_q_in_place():
    r = A.make_rows(mixed(2), 4, "bf16", True, True, rotary=128, seed=5)
    announce("append with q_out = q")
    check(r, *run(r, packed=False, in_place=True))


@pytest.mark.parametrize("eight", [False, True])
def test_direction_table(eight):
    b = with_direction_table(mixed(2))
    r = A.make_rows(b, 4, "bf16", rotary=128, seed=6)
    announce(f"append with a direction table, eight={eight}")
    check(r, *run(r, eight), eight)


@pytest.mark.parametrize("eight", [False, True])
def test_many_sequences(eight):
    # more sequences than a workgroup's threads; single tokens, some at position 0
    rng = np.random.default_rng(7)
    ctx = [int(x) for x in rng.integers(1, 60, 700)]
    b = W.custom(ctx, [W.RT if i % 3 else W.BE for i in range(700)], 2, 2, seed=7)
    r = A.make_rows(b, 4, "bf16", True, True, rotary=128, seed=7)
    announce(f"append 700 sequences, eight={eight}")
    check(r, *run(r, eight), eight)


@pytest.mark.parametrize("eight", [False, True])
def test_rows_of_no_sequence_are_left_alone(eight):
    # the call's token count may exceed the sequences' (a padded batch)
    b = mixed(2)
    pad = 37
    grown = dataclasses.replace(b, cu_new=b.cu_new.copy())
    r = A.make_rows(b, 4, "bf16", True, True, rotary=128, seed=8)
    rng = np.random.default_rng(8)
    wide = dataclasses.replace(r, batch=grown, **{n: np.concatenate([getattr(r, n), rng.integers(0, 60000, (pad,) + getattr(r, n).shape[1:]).astype(np.uint16)])
                                                  for n in ("q", "k", "v")})
    announce(f"append with {pad} rows of padding, eight={eight}")
    got, start = run(wide, eight)
    tn = int(b.cu_new[-1])
    assert (oracle.widen(got[0][tn:], "bf16") == 7.0).all(), "a row of padding was written"
    check(r, (got[0][:tn], *got[1:]), start, eight)


@pytest.mark.parametrize("eight", [False, True])
def test_invalid_entries_and_empty_sequences(eight):
    # entries outside the pool, and positions past the table: q rows as ever, nothing stored
    b = W.custom([300, 40, 7, 90, 16, 16], MIXED["cls"], 2, 2, seed=9, num_prefill=2, new_counts=[130, 40, 0, 1, 0, 1],
                 spare_blocks=2)
    tables = b.block_tables.copy()
    tables[0, 15] = b.num_blocks
    tables[1, 0] = -1
    tables[3, 5] = -5
    r = A.make_rows(b, 4, "bf16", True, True, rotary=64, seed=9)
    seq, pos = A.tokens(b)
    entry = tables[seq, pos // 16]
    stored = np.nonzero((entry >= 0) & (entry < b.num_blocks))[0]
    assert 0 < len(stored) < len(seq)
    announce(f"append with invalid table entries, eight={eight}")
    got, start = run(r, eight, tables=tables)
    check(r, got, start, eight, stored)
    short = tables[:, :3].copy()           # tables too short for the first chunk and the decode row of sequence 3
    stored = np.nonzero((entry >= 0) & (entry < b.num_blocks) & (pos // 16 < 3))[0]
    got, start = run(r, eight, tables=short)
    check(r, got, start, eight, stored)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("axes", [1, 3])
def test_rotation_positions_outside_the_table(axes, eight):
    # such a token's q rows are zeros and it is not stored
    b = mixed(2)
    r = A.make_rows(b, 4, "bf16", True, False, rotary=128, sections=(16, 24, 24) if axes == 3 else None, seed=10)
    tn = int(b.cu_new[-1])
    if axes == 1:
        r.pos = A.tokens(b)[1][None].astype(np.int32)
    out = np.array([0, 31, tn - 1])
    bad = r.pos.copy()
    bad[-1, out] = [-1, r.table.shape[0], 2 ** 31 - 1]
    announce(f"append with rotation positions outside the table, axes={axes} eight={eight}")
    got, start = run(dataclasses.replace(r, pos=bad), eight)
    assert (got[0][out] == 0).all()
    live = np.setdiff1d(np.arange(tn), out)
    seq, pos = A.tokens(b)
    (q, reach), _ = A.expected(r, seq, pos)
    A.check_close(got[0], q, reach, "bf16", "q", live)
    check(r, (None, *got[1:]), start, eight, live)


def test_a_table_shorter_than_the_positions():
    b = mixed(2)
    r = A.make_rows(b, 4, "bf16", rotary=128, seed=11)
    seq, pos = A.tokens(b)
    r = dataclasses.replace(r, table=r.table[:100])
    live = np.nonzero(pos < 100)[0]
    announce("append with a table shorter than the positions")
    got, start = run(r)
    assert (got[0][pos >= 100] == 0).all()
    full = dataclasses.replace(r, table=A.make_table(int(b.ctx_lens.max()) + 3, 128, 11))
    (q, reach), _ = A.expected(full, seq, pos)
    A.check_close(got[0], q, reach, "bf16", "q", live)
    check(full, (None, *got[1:]), start, False, live)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_eight_bit_rows_of_all_sizes(dtype):
    # zeros, the least and the largest magnitudes, exact ties, infinities and NaNs: bit-exact without arithmetic
    b = W.custom([20, 33, 48, 5], [W.RT, W.BE, W.RT, W.BE], 2, 2, dtype=dtype, seed=12, new_counts=[20, 33, 48, 5],
                 num_prefill=4)
    r = A.make_rows(b, 4, dtype, seed=12)
    x = oracle.widen(r.k, dtype).astype(np.float32)
    x[0] = 0.0
    x[1, 0] = 1e-38
    x[2] *= np.float32(2.0 ** 120)
    x[3] *= np.float32(2.0 ** -110)
    x[4, 0, :16] = [1.0625, 1.1875, -1.0625, -1.1875, 448, -448, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 0.0, -0.0, 1.5, 17, 19, 240, 432]
    x[4, 0, 16:] = 0.25
    x[5, 1, 3], x[5, 1, 64], x[5, 1, 127] = np.inf, -np.inf, np.nan
    x[6, 0] = np.nan
    x[7, 0] = 448.0
    x[8, 0] = np.float32(448.0) * np.float32(1 + 2.0 ** -7)
    x[9, 0, :] = 0
    x[9, 0, 5] = np.float32(3.38e38)
    r.k = r.v = A._store(x, dtype)
    announce(f"append-q8 rows of all sizes {dtype}")
    got, start = run(r, True)
    seq, pos = A.tokens(b)
    locs = [oracle.physical_location(b.block_tables, b.dir, int(s), np.array([p])) for s, p in zip(seq, pos)]
    blk, slot = np.array([int(a[0]) for a, _ in locs]), np.array([int(c[0]) for _, c in locs])
    codes, bytes_ = oracle.encode(oracle.widen(r.k, dtype))
    for which, pool in ((0, got[1]), (1, got[2])):
        assert (got[3][blk, :, which, slot] == bytes_).all()
        now = pool[blk, :, slot]
        nan = codes == oracle.NAN_CODE
        assert ((now & 0x7F) == oracle.NAN_CODE)[nan].all()
        assert (now == codes)[~nan].all()


def test_v_rows_keep_their_bits():
    # NaN payloads and infinities of a 16-bit pool's v rows pass unchanged, as in bros_kv_write
    b = mixed(2)
    r = A.make_rows(b, 4, "bf16", True, True, rotary=128, seed=13)
    r.v = np.random.default_rng(13).integers(0, 1 << 16, r.v.shape).astype(np.uint16)
    announce("append of arbitrary v bits")
    check(r, *run(r))


def test_nothing_to_do_and_one_token():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    b = W.custom([1], [W.RT], 1, 1, seed=14)
    r = A.make_rows(b, 1, "bf16", True, True, rotary=128, seed=14)
    announce("append of one token, then of none")
    check(r, *run(r))
    empty = torch.empty((0, 1, 128), dtype=torch.bfloat16, device="cuda")
    pool = torch.zeros((2, 1, 16, 128), dtype=torch.bfloat16, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    bros.bros_qkv_append(empty, empty, empty, empty, pool, pool.clone(), i32(0)[None], None,
                         torch.zeros(1, dtype=torch.uint8, device="cuda"), i32(0), i32(0, 0))
    torch.cuda.synchronize()
    assert not pool.any()


@pytest.mark.parametrize("eight", [False, True])
def test_captured_and_replayed_on_another_stream(eight):
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    b = mixed(2)
    r = A.make_rows(b, 4, "bf16", True, True, rotary=128, seed=15)
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    q, k, v = A.device_rows(r)
    q_out = torch.zeros(q.shape, dtype=q.dtype, device="cuda")
    start = eight_bit_pool(b) if eight else (b.k_pool, b.v_pool)
    dev = [bros._tensor(x, None if eight else "bf16", "cuda") for x in start]
    fresh = [x.clone() for x in dev]
    args = (q_out, q, k, v, *dev, up(b.block_tables), up(b.dir), None, up(b.pos0), up(b.cu_new))
    kw = A.options(r)
    call = bros.bros_qkv_append_q8 if eight else bros.bros_qkv_append
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    announce(f"append captured, eight={eight}")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        call(*args, **kw)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            call(*args, **kw)
    for _ in range(3):
        q_out.zero_()
        for x, y in zip(dev, fresh):
            x.copy_(y)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(r, (bros.to_host_bits(q_out), *(bros.to_host_bits(x) for x in dev)), start, eight)
