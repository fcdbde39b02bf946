"""Slots of an 8-bit pool: gather and scatter move bytes, read gives the values."""

import numpy as np
import pytest

import oracle
from tests.gpu_helpers import announce, require_gpu

pytestmark = pytest.mark.gpu


def pool(nb, hkv, seed):
    """Any codes, scales over the range an append writes."""
    rng = np.random.default_rng(seed)
    shape = (nb, hkv, 16, 128)
    return (rng.integers(0, 256, shape, dtype=np.uint8), rng.integers(0, 256, shape, dtype=np.uint8),
            rng.integers(27, 248, (nb, hkv, 2, 16), dtype=np.uint8))


def ids_of(nb, n, seed, outside=True):
    rng = np.random.default_rng(seed)
    ids = rng.permutation(nb * 16)[:n].astype(np.int32)
    if outside and n >= 4:
        ids[[0, n // 2, n - 1]] = [-1, nb * 16, -2 ** 31]
    return ids


def rows(pool_, ids):
    ok = (ids >= 0) & (ids < pool_.shape[0] * 16)
    at = np.where(ok, ids, 0)
    return pool_[at // 16, :, at % 16], ok


@pytest.mark.parametrize("hkv", [1, 3, 8, 40])
@pytest.mark.parametrize("n", [1, 4, 33, 700])
def test_gather_scatter_read(hkv, n):
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    nb = 64
    host = pool(nb, hkv, n)
    up = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    k, v, s = (up(x) for x in host)
    ids = ids_of(nb, n, n + hkv)
    announce(f"kv_q8 moves hkv={hkv} n={n}")
    ko, vo = (torch.full((n, hkv, 128), 9, dtype=torch.uint8, device="cuda") for _ in range(2))
    so = torch.full((n, hkv, 2), 9, dtype=torch.uint8, device="cuda")
    bros.bros_kv_gather_q8(k, v, s, up(ids), ko, vo, so)
    torch.cuda.synchronize()
    kw, ok = rows(host[0], ids)
    vw, _ = rows(host[1], ids)
    sw = host[2][np.where(ok, ids, 0) // 16, :, :, np.where(ok, ids, 0) % 16]
    kw, vw, sw = (np.where(ok[:, None, None], x, 0) for x in (kw, vw, sw))
    assert (ko.cpu().numpy() == kw).all() and (vo.cpu().numpy() == vw).all() and (so.cpu().numpy() == sw).all()

    for dt in (torch.bfloat16, torch.float32):
        kr, vr = (torch.full((n, hkv, 128), 9.0, dtype=dt, device="cuda") for _ in range(2))
        bros.bros_kv_read_q8(k, v, s, up(ids), kr, vr)
        torch.cuda.synchronize()
        for got, codes, which in ((kr, kw, 0), (vr, vw, 1)):
            want = np.where(ok[:, None, None], oracle.decode_rows(codes, np.where(ok[:, None], sw[:, :, which], 127)), 0.0)
            # Exact in both types, as far as they reach: 2^128 is the first power of two that
            # neither bf16 nor fp32 holds, and a value of at least that (codes of 256 and more at
            # e = 120, which no append of fp32 rows writes) is an infinity.
            want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
            back = got.double().cpu().numpy()
            same = (back == want) | (np.isnan(back) & np.isnan(want))
            assert same.all(), (back[~same][:4], want[~same][:4])

    other = ids_of(nb, n, n + hkv + 1)
    bros.bros_kv_scatter_q8(ko, vo, so, up(other), k, v, s)
    torch.cuda.synchronize()
    want = [x.copy() for x in host]
    okd = (other >= 0) & (other < nb * 16)
    want[0][other[okd] // 16, :, other[okd] % 16] = kw[okd]
    want[1][other[okd] // 16, :, other[okd] % 16] = vw[okd]
    want[2][other[okd] // 16, :, :, other[okd] % 16] = sw[okd]
    for got, w in zip((k, v, s), want):
        assert (got.cpu().numpy() == w).all()


def test_part_of_the_list_and_pinned_host_buffers():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    host = pool(8, 2, 3)
    k, v, s = (torch.from_numpy(x).cuda() for x in host)
    ids = np.arange(40, dtype=np.int32)
    announce("kv_q8 gather of 24 of 40 ids into pinned memory")
    ko, vo = (torch.full((40, 2, 128), 9, dtype=torch.uint8, pin_memory=True) for _ in range(2))
    so = torch.full((40, 2, 2), 9, dtype=torch.uint8, pin_memory=True)
    bros.bros_kv_gather_q8(k, v, s, torch.from_numpy(ids).cuda(), ko, vo, so, num_slots=24)
    torch.cuda.synchronize()
    assert (ko.numpy()[:24] == rows(host[0], ids)[0][:24]).all() and (ko.numpy()[24:] == 9).all()
    assert (vo.numpy()[:24] == rows(host[1], ids)[0][:24]).all() and (so.numpy()[24:] == 9).all()


def test_far_slots():
    # a pool beyond 4 GiB per tensor: byte offsets pass 32 bits
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    nb, hkv = 140000, 16
    k, v = (torch.zeros((nb, hkv, 16, 128), dtype=torch.uint8, device="cuda") for _ in range(2))
    s = torch.full((nb, hkv, 2, 16), 127, dtype=torch.uint8, device="cuda")
    ids = torch.tensor([nb * 16 - 1, 0, (1 << 31) // (hkv * 128) + 5, (1 << 32) // (hkv * 128) + 5], dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(5)
    src = [torch.from_numpy(rng.integers(0, 120, (4, hkv, w), dtype=np.uint8)).cuda() for w in (128, 128, 2)]
    announce("kv_q8 far slots")
    bros.bros_kv_scatter_q8(*src, ids, k, v, s)
    out = [torch.empty_like(x) for x in src]
    bros.bros_kv_gather_q8(k, v, s, ids, *out)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(src, out))
    assert int((k != 0).any(-1).sum()) <= 4 * hkv
    assert torch.equal(k[-1, :, 15], src[0][0]) and torch.equal(k[0, :, 0], src[0][1])
