"""The append's q_out where it lies close to the rows, but on none of them: accepted, and right."""

import pytest

from paper_2504_09590_amd import workload as W
from tests import append_helpers as A
from tests.gpu_helpers import announce, require_gpu
from tests.test_gpu_append import check, eight_bit_pool

pytestmark = pytest.mark.gpu


def call(r, eight, q_out, q, k, v):
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    b = r.batch
    start = eight_bit_pool(b) if eight else (b.k_pool, b.v_pool)
    dev = [bros._tensor(x, None if eight else r.dtype, "cuda") for x in start]
    up = lambda x: bros._tensor(x, None, "cuda")  # noqa: E731
    fn = bros.bros_qkv_append_q8 if eight else bros.bros_qkv_append
    fn(q_out, q, k, v, *dev, up(b.block_tables), up(b.dir), up(b.cls), up(b.pos0), up(b.cu_new), **A.options(r))
    torch.cuda.synchronize()
    check(r, (bros.to_host_bits(q_out), *(bros.to_host_bits(x) for x in dev)), start, eight)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_neighbours(dtype, eight):
    torch = require_gpu()
    hq, hkv, n = 4, 2, 9
    b = W.custom([30, 5], [W.RT, W.BE], hq, hkv, dtype=dtype, seed=2, new_counts=[8, 1], num_prefill=1, spare_blocks=1)
    r = A.make_rows(b, hq, dtype, True, True, rotary=128, seed=4)
    q, k, v = A.device_rows(r, packed=False)
    announce(f"append, q_out beside the rows, {dtype}, eight={eight}")
    # one buffer: k rows | q_out | v rows
    buf = torch.cat([k.flatten(), torch.zeros_like(q).flatten(), v.flatten()])
    kn, qn = k.numel(), q.numel()
    call(r, eight, buf[kn:kn + qn].view(q.shape), q, buf[:kn].view(k.shape), buf[kn + qn:].view(v.shape))
    # q_out between the first two tokens' k rows
    wide = torch.zeros((n, k.shape[1] * 128 + qn + 16), dtype=q.dtype, device="cuda")
    kk = wide[:, :hkv * 128].unflatten(1, (hkv, 128))
    kk.copy_(k)
    call(r, eight, wide.flatten()[hkv * 128:hkv * 128 + qn].view(q.shape), q, kk, v)


def test_one_token_in_place():
    # a projection's only token: q_out is its q, k and v behind it
    torch = require_gpu()
    hq, hkv = 4, 2
    b = W.custom([30], [W.BE], hq, hkv, dtype="bf16", seed=3, new_counts=[1], num_prefill=0, spare_blocks=1)
    r = A.make_rows(b, hq, "bf16", True, True, rotary=128, seed=5)
    q, k, v = A.device_rows(r)
    announce("append of one token in place")
    assert q.untyped_storage().data_ptr() == k.untyped_storage().data_ptr()
    call(r, False, q, q, k, v)
    torch.cuda.synchronize()
