"""What bros_kv_read_q8 gives for every code under every scale byte from the least an append writes on."""

import numpy as np
import pytest

import oracle
from tests.gpu_helpers import announce, require_gpu

pytestmark = pytest.mark.gpu


def test_every_code_under_every_scale():
    torch = require_gpu()
    from paper_2504_09590_amd import bros
    bytes_ = np.arange(27, 256)
    nb = (2 * len(bytes_) + 15) // 16
    codes = np.zeros((nb * 16, 128), dtype=np.uint8)
    scale = np.full(nb * 16, 127, dtype=np.uint8)
    for half in range(2):                                        # codes 0 .. 127, then 128 .. 255
        at = half * len(bytes_) + np.arange(len(bytes_))
        codes[at], scale[at] = np.arange(128) + 128 * half, bytes_
    k = torch.from_numpy(codes.reshape(nb, 1, 16, 128)).cuda()
    s = torch.from_numpy(np.stack([scale.reshape(nb, 1, 16)] * 2, axis=2)).cuda()
    ids = torch.arange(nb * 16, dtype=torch.int32, device="cuda")
    want = oracle.decode_rows(codes, scale)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    want[scale == 255] = np.nan                                  # the scale of no number
    announce("kv_q8 read of every code under every scale")
    for dt in (torch.bfloat16, torch.float32):
        out = [torch.zeros((nb * 16, 1, 128), dtype=dt, device="cuda") for _ in range(2)]
        bros.bros_kv_read_q8(k, k, s, ids, *out)
        torch.cuda.synchronize()
        for x in out:
            got = x.double().cpu().numpy()[:, 0]
            bad = ~((got == want) | (np.isnan(got) & np.isnan(want)))
            assert not bad.any(), (scale[np.nonzero(bad)[0][:3]], codes[bad][:3], got[bad][:3], want[bad][:3])
