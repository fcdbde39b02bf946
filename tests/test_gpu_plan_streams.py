"""PlanExecutor on streams that are not the current one and are held back by earlier work."""

import types

import numpy as np
import pytest

from tests.gpu_helpers import announce, require_gpu

pytestmark = pytest.mark.gpu

NB, HKV = 12, 3
HELD = 40_000_000      # cycles of earlier work: some 20 ms


def pools(eight):
    torch = require_gpu()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    if not eight:
        return [torch.randn((NB, HKV, 16, 128), generator=gen, device="cuda").bfloat16() for _ in range(2)]
    shapes = [(NB, HKV, 16, 128)] * 2 + [(NB, HKV, 2, 16)]
    return [torch.randint(0, 256, s, generator=gen, device="cuda", dtype=torch.uint8) for s in shapes]


def rows(pool, ids):
    """The slots' rows (codes and values [n][Hkv][128], scales [n][Hkv][2])."""
    blk, slot = np.asarray(ids) // 16, np.asarray(ids) % 16
    return pool[blk, :, :, slot] if pool.shape[2] == 2 else pool[blk, :, slot]


def put(pool, ids, x):
    blk, slot = np.asarray(ids) // 16, np.asarray(ids) % 16
    if pool.shape[2] == 2:
        pool[blk, :, :, slot] = x
    else:
        pool[blk, :, slot] = x


def plan(victims=(), move=((), ()), restore=((), ())):
    return types.SimpleNamespace(victims=np.array(victims, dtype=np.int64).reshape(-1, 4), move_src=np.array(move[0]), move_dst=np.array(move[1]),
                                 restore_pos=np.array(restore[0]), restore_dst=np.array(restore[1]))


def bits(ts):
    torch = require_gpu()
    return [t.view(torch.int16).cpu().numpy().copy() if t.dtype == torch.bfloat16 else t.cpu().numpy().copy() for t in ts]


def executor(ps):
    from paper_2504_09590_amd.swap import PlanExecutor
    return PlanExecutor(ps[0], ps[1], max_rows=8, kv_scales=ps[2] if len(ps) == 3 else None)


@pytest.mark.parametrize("eight", [False, True])
def test_on_a_held_stream(eight):
    torch = require_gpu()
    ps = pools(eight)
    ex = executor(ps)
    ids = np.random.default_rng(1).permutation(NB * 16)
    saved, src, dst, back = ids[:8], ids[8:28], ids[28:48], ids[48:56]
    side = torch.cuda.Stream()
    announce(f"a plan on a held stream, eight={eight}")
    torch.cuda.synchronize()
    host = bits(ps)
    ex.execute(7, plan(victims=[(7, p, i // 16, i % 16) for p, i in enumerate(saved)]), stream=side)
    with torch.cuda.stream(side):
        torch.cuda._sleep(HELD)
    ex.execute(7, plan(move=(src, dst), restore=(np.arange(8), back)), stream=side)
    # other tensors of the current stream, of the ids' size
    other = [torch.full((n,), 5, dtype=torch.int32, device="cuda") for n in (8, 8, 4, 8, 8, 4, 8, 8)]
    torch.cuda.synchronize()
    for h in host:
        was, moved = rows(h, saved).copy(), rows(h, src).copy()
        put(h, dst, moved)
        put(h, back, was)
    assert all(np.array_equal(a, b) for a, b in zip(bits(ps), host))
    assert all(int((t != 5).sum()) == 0 for t in other) and not ex.store


@pytest.mark.parametrize("eight", [False, True])
def test_plans_on_two_streams(eight):
    # the first waits behind earlier work; the second, on a free stream, takes the same staging buffers
    torch = require_gpu()
    ps = pools(eight)
    ex = executor(ps)
    ids = np.random.default_rng(2).permutation(NB * 16)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    announce(f"plans on two streams, eight={eight}")
    torch.cuda.synchronize()
    host = bits(ps)
    with torch.cuda.stream(a):
        torch.cuda._sleep(HELD)
    ex.execute(1, plan(move=(ids[:8], ids[8:16])), stream=a)
    ex.execute(2, plan(move=(ids[16:24], ids[24:32])), stream=b)
    torch.cuda.synchronize()
    for h in host:
        put(h, ids[8:16], rows(h, ids[:8]).copy())
        put(h, ids[24:32], rows(h, ids[16:24]).copy())
    assert all(np.array_equal(x, y) for x, y in zip(bits(ps), host))
