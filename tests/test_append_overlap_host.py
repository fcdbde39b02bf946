"""The append refuses a q_out that overlaps rows it reads (no GPU): workgroups would overwrite
rows that others have yet to read. Every call here is refused, none is launched."""

import pytest

bros = pytest.importorskip("paper_2504_09590_amd.bros", reason="libbros_attn.so not built")

BASE = 1 << 24
SHAPE = -2
HQ, HKV, D = 8, 2, 128


def refused(eight, elem, tn, q_out, q, k, v, qs=None, ks=None, vs=None):
    """Addresses in elements from BASE, strides in elements (default: contiguous tokens)."""
    at = lambda x: BASE + elem * x  # noqa: E731
    far = 1 << 40
    args = [at(q_out), at(q), at(k), at(v), HQ * D if qs is None else qs, HKV * D if ks is None else ks, HKV * D if vs is None else vs,
            tn, HQ, None, None, None, far, 2 * far] + ([3 * far] if eight else [])
    args += [10, 4 * far, 4, 4 * far, None, 0, 4 * far, 4 * far, 2, HKV, D, 16, 0 if elem == 4 else 1, None]
    status = (bros.LIB.bros_qkv_append_q8 if eight else bros.LIB.bros_qkv_append)(*args)
    assert status == SHAPE
    return "overlaps" in bros.LIB.bros_last_error().decode()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("elem", [2, 4])
def test_overlaps_are_refused(eight, elem):
    heads = HQ + 2 * HKV
    row = heads * D                                    # a projection's rows: q | k | v of each token
    packed = dict(qs=row, ks=row, vs=row)
    q, k, v = 0, HQ * D, (HQ + HKV) * D
    call = lambda tn, out, **kw: refused(eight, elem, tn, out, **dict(dict(q=q, k=k, v=v, **packed), **kw))  # noqa: E731
    assert call(5, 0)                                  # in place, but q's tokens are not contiguous
    assert call(2, 0)
    assert call(5, 5 * row - 8)                        # the last eight values of the last v row
    assert call(5, 4 * row)                            # the last token
    assert call(5, row - HQ * D)                       # from the first token's k on
    apart = dict(q=0, k=1 << 20, v=1 << 21, qs=HQ * D, ks=HKV * D, vs=HKV * D)
    n = 5 * HQ * D
    assert call(5, 8, **apart) and call(5, n - 8, **apart)                          # q, moved by eight values
    assert call(5, (1 << 20) - n + 8, **apart) and call(5, (1 << 20) + 5 * HKV * D - 8, **apart)
    assert call(5, (1 << 21) - n + 8, **apart) and call(5, (1 << 21) + 5 * HKV * D - 8, **apart)
    assert call(5, 0, **dict(apart, qs=HQ * D + 8))    # in place, rows eight values apart
    assert call(1, HQ * D, q=0, k=HQ * D, v=v)         # one token, but its k row
