"""A step over a latent cache whose prompts go on from chunk to chunk: the lengths move on the device, within its bounds."""

import numpy as np
import pytest

from tests.gpu_helpers import announce, require_gpu
from tests.rows_helpers import attention, bf16, visible
from tests.test_gpu_draft_steps import make
from tests.test_gpu_latent import LATENT, ROW

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bounded", [True, False])
def test_chunk_after_chunk(bounded):
    """Five chunks of each prompt, to contexts within the bounds of a long one and of narrow units. Without bounds a step
    takes the first chunk's alone, as its documentation says."""
    torch = require_gpu()
    from paper_2504_09590_amd.step import LatentStep
    rng = np.random.default_rng(4)
    hq, n, c0, most = 3, [300, 41], [0, 64], 5
    b, batch, dev = make(n, c0, 1300, hq, num_prefill=2)
    host = bf16(rng, (b.num_blocks, 16, ROW))
    pool, w = host.cuda(), bf16(rng, (hq, 256, LATENT), LATENT ** -0.5)
    last = [c + most * m for c, m in zip(c0, n)]
    step = LatentStep(batch, dev, pool, w.cuda(), **(dict(max_ctx_chunks=max(last), total_ctx=sum(last)) if bounded else {}))
    for i in range(most if bounded else 1):
        kv, q = bf16(rng, (b.rows, ROW)), bf16(rng, (b.rows, hq, 192))
        for s in range(b.S):
            host[b.places(s, b.c0[s] + np.arange(b.n[s]))] = kv[b.cu[s]:b.cu[s + 1]]
        announce(f"latent, chunk {i}")
        got = step.run(kv.cuda(), q_chunks=q.cuda())[0]
        torch.cuda.synchronize()
        assert torch.equal(pool.cpu(), host)
        for s in range(b.S):
            lo, hi = int(b.cu[s]), int(b.cu[s + 1])
            c, see = host[b.places(s, np.arange(b.ctx[s]))].double(), visible(b, s, None)
            for h in range(hq):
                k = torch.cat([c[:, :LATENT] @ w[h, :128].double().t(), c[:, LATENT:]], 1)
                y, _ = attention(q[lo:hi, h].double(), k, c[:, :LATENT] @ w[h, 128:].double().t(), see, 192 ** -0.5)
                # (bounds value by value are the expanded form's own tests'; here: the roundings together)
                assert float((got[lo:hi, h].cpu().double() - y).norm() / y.norm()) <= 2.0 ** -7, (i, s, h)
        b.c0, b.ctx = b.c0 + b.n, b.ctx + b.n
        dev.pos0 += torch.from_numpy(b.n.astype(np.int32)).cuda()
        dev.ctx_lens += torch.from_numpy(b.n.astype(np.int32)).cuda()
