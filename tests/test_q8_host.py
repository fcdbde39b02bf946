"""Refusals of the append and the 8-bit cache's calls (no GPU): every bad argument
is turned down before anything is launched. And the oracle's 8-bit rows against
torch's conversion."""

import ctypes

import numpy as np
import pytest
import torch

import oracle

bros = pytest.importorskip("paper_2504_09590_amd.bros", reason="libbros_attn.so not built")

FAKE = 1 << 20   # a 16-byte aligned non-NULL address; only used on paths rejected before launch


def rope(**kw):
    a = dict(table=FAKE, rows=64, dim=128, pairs=0, axes=1, sections=(0, 0, 0, 0))
    a.update(kw)
    return bros._Rope(a["table"], a["rows"], a["dim"], a["pairs"], a["axes"], (ctypes.c_int32 * 4)(*a["sections"]))


def append(eight, **kw):
    a = dict(q_out=FAKE, q=FAKE, k=FAKE, v=FAKE, qs=1024, ks=256, vs=256, tn=5, hq=8, norm=None, rope=None, rope_pos=None,
             kp=FAKE, vp=FAKE, scales=FAKE, nb=10, bt=FAKE, maxb=4, dir=FAKE, cls=None, dpe=0, pos0=FAKE, cu=FAKE, S=2, hkv=2,
             d=128, bs=16, dtype=1)
    a.update(kw)
    ref = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    args = [a["q_out"], a["q"], a["k"], a["v"], a["qs"], a["ks"], a["vs"], a["tn"], a["hq"], ref(a["norm"]), ref(a["rope"]),
            a["rope_pos"], a["kp"], a["vp"]] + ([a["scales"]] if eight else [])
    args += [a["nb"], a["bt"], a["maxb"], a["dir"], a["cls"], a["dpe"], a["pos0"], a["cu"], a["S"], a["hkv"], a["d"], a["bs"],
             a["dtype"], None]
    return (bros.LIB.bros_qkv_append_q8 if eight else bros.LIB.bros_qkv_append)(*args)


NULL, SHAPE, DTYPE, UNSUPPORTED = -1, -2, -3, -4


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), DTYPE), (dict(d=64), UNSUPPORTED), (dict(bs=32), UNSUPPORTED), (dict(hkv=0), SHAPE),
    (dict(hkv=20000), UNSUPPORTED), (dict(hq=20000), UNSUPPORTED), (dict(tn=-1), SHAPE), (dict(S=-1), SHAPE), (dict(S=0), SHAPE),
    (dict(q=None), NULL), (dict(q_out=None), NULL), (dict(hq=0), SHAPE), (dict(hq=-1), SHAPE), (dict(k=None), NULL),
    (dict(v=None), NULL), (dict(kp=None), NULL), (dict(vp=None), NULL), (dict(bt=None), NULL), (dict(dir=None), NULL),
    (dict(pos0=None), NULL), (dict(cu=None), NULL), (dict(nb=0), SHAPE), (dict(maxb=0), SHAPE), (dict(dpe=2), SHAPE),
    (dict(qs=1023), SHAPE), (dict(qs=1028), SHAPE), (dict(ks=255), SHAPE), (dict(ks=0), SHAPE), (dict(vs=-256), SHAPE),
    (dict(vs=2 ** 62), SHAPE), (dict(q=FAKE + 4), SHAPE), (dict(q_out=FAKE + 8), SHAPE), (dict(kp=FAKE + 2), SHAPE),
    (dict(tn=2 ** 31 - 1), SHAPE), (dict(tn=(2 ** 29 - 32) // 12 + 1), SHAPE),   # 12 head rows a token
    (dict(rope=rope(dim=0)), SHAPE), (dict(rope=rope(dim=144)), SHAPE), (dict(rope=rope(dim=24)), SHAPE),
    (dict(rope=rope(pairs=2)), SHAPE), (dict(rope=rope(axes=0)), SHAPE), (dict(rope=rope(axes=5)), SHAPE),
    (dict(rope=rope(rows=0)), SHAPE), (dict(rope=rope(table=None)), NULL), (dict(rope=rope(table=FAKE + 4)), SHAPE),
    (dict(rope=rope(axes=3, sections=(16, 24, 24, 0))), SHAPE),                    # no rope_pos
    (dict(rope=rope(axes=3, sections=(16, 24, 23, 0)), rope_pos=FAKE), SHAPE),
    (dict(rope=rope(axes=3, sections=(2 ** 31 - 1, 2 ** 31 - 1, 66, 0)), rope_pos=FAKE), SHAPE),
    (dict(rope=rope(axes=3, sections=(70, -6, 0, 0)), rope_pos=FAKE), SHAPE),
    (dict(rope=rope(), rope_pos=FAKE + 2), SHAPE),
    (dict(norm=bros._QkNorm(FAKE + 4, None, 1e-6)), SHAPE),
])
def test_append_rejects(eight, kw, code):
    assert append(eight, **kw) == code
    assert bros.LIB.bros_last_error().decode() != ""


def test_append_q8_needs_scales():
    assert append(True, scales=None) == NULL
    assert append(True, scales=FAKE + 1) == SHAPE


@pytest.mark.parametrize("eight", [False, True])
def test_append_of_no_tokens(eight):
    assert append(eight, tn=0, k=None, v=None, S=0) == 0


@pytest.mark.parametrize("fn", ["gather", "scatter", "read"])
def test_moves_reject(fn):
    L = getattr(bros.LIB, f"bros_kv_{fn}_q8")
    names = {"gather": ["k", "v", "s", "nb", "ids", "n", "ko", "vo", "so", "hkv", "d", "bs"],
             "scatter": ["ko", "vo", "so", "ids", "n", "k", "v", "s", "nb", "hkv", "d", "bs"],
             "read": ["k", "v", "s", "nb", "ids", "n", "ko", "vo", "hkv", "d", "bs", "dtype"]}[fn]
    good = dict(k=FAKE, v=FAKE, s=FAKE, nb=10, ids=FAKE, n=5, ko=FAKE, vo=FAKE, so=FAKE, hkv=8, d=128, bs=16, dtype=1)

    def call(**kw):
        a = dict(good, **kw)
        return L(*[a[n] for n in names], None)

    for kw, code in ((dict(d=64), UNSUPPORTED), (dict(bs=8), UNSUPPORTED), (dict(hkv=0), SHAPE), (dict(hkv=20000), UNSUPPORTED),
                     (dict(n=-1), SHAPE), (dict(nb=0), SHAPE), (dict(k=None), NULL), (dict(v=None), NULL), (dict(s=None), NULL),
                     (dict(ids=None), NULL), (dict(ko=None), NULL), (dict(vo=None), NULL), (dict(k=FAKE + 8), SHAPE),
                     (dict(ko=FAKE + 4), SHAPE), (dict(ids=FAKE + 2), SHAPE), (dict(s=FAKE + 1), SHAPE)):
        assert call(**kw) == code, kw
    if "so" in names:
        assert call(so=None) == NULL
    if "dtype" in names:
        assert call(dtype=3) == DTYPE
    assert call(n=0, ids=None, k=None) == 0


def rows(t, h, dtype=torch.bfloat16):
    return torch.zeros((t, h, 128), dtype=dtype)


def py_call(**kw):
    """bros_qkv_append with host tensors: whatever passes the shape checks fails the device check, never a launch."""
    a = dict(q_out=rows(5, 8), q=rows(5, 8), k=rows(5, 2), v=rows(5, 2), k_pool=torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16),
             v_pool=torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16), block_tables=torch.zeros((2, 3), dtype=torch.int32),
             dir=torch.ones(2, dtype=torch.int8), cls=None, pos0=torch.zeros(2, dtype=torch.int32),
             cu_new=torch.tensor([0, 3, 5], dtype=torch.int32))
    a.update(kw)
    bros.bros_qkv_append(**a)


@pytest.mark.parametrize("kw,says", [
    ({}, "current device"),
    (dict(k=rows(5, 2, torch.float32)), "pool"),
    (dict(k=rows(4, 2)), "must be"),
    (dict(v=rows(5, 3)), "heads"),
    (dict(q_out=rows(5, 4)), "q_out"),
    (dict(q=torch.zeros((5, 128, 8), dtype=torch.bfloat16).transpose(1, 2)), "contiguous within"),
    (dict(q=rows(5, 16)[:, ::2]), "contiguous within"),
    (dict(block_tables=torch.zeros((2, 3), dtype=torch.int64)), "block_tables"),
    (dict(block_tables=torch.zeros((1, 3), dtype=torch.int32)), "block_tables"),
    (dict(dir=torch.ones(3, dtype=torch.int8)), "dir"),
    (dict(dir=torch.ones((2, 4), dtype=torch.int8)), "direction table"),
    (dict(pos0=torch.zeros(3, dtype=torch.int32)), "offset"),
    (dict(rope_pos=torch.zeros((1, 5), dtype=torch.int32)), "without a rotation"),
    (dict(rope=bros.Rope(torch.zeros((9, 128))), rope_pos=torch.zeros((2, 5), dtype=torch.int32)), "rope_pos"),
    (dict(rope=bros.Rope(torch.zeros((9, 128)), sections=(16, 24, 24)), rope_pos=torch.zeros((5, 3), dtype=torch.int32)), "rope_pos"),
    (dict(norm=bros.QkNorm(torch.ones(64, dtype=torch.bfloat16), None)), "norm weights"),
    (dict(norm=bros.QkNorm(torch.ones(128), None)), "norm weights"),
])
def test_binding_refuses(kw, says):
    with pytest.raises(ValueError, match=says):
        py_call(**kw)


def test_binding_refuses_eight_bit_shapes():
    pool = torch.zeros((4, 2, 16, 128), dtype=torch.uint8)
    scales = torch.zeros((4, 2, 2, 16), dtype=torch.uint8)
    ids = torch.zeros(3, dtype=torch.int32)
    out, so = torch.zeros((3, 2, 128), dtype=torch.uint8), torch.zeros((3, 2, 2), dtype=torch.uint8)
    for args, says in (((pool.to(torch.int16), pool, scales, ids, out, out, so), "one byte"),
                       ((pool, pool, scales[:3], ids, out, out, so), "kv_scales"),
                       ((pool, pool, scales, ids.long(), out, out, so), "slot_ids"),
                       ((pool, pool, scales, ids, out[:2], out, so), "dense"),
                       ((pool, pool, scales, ids, out, out.float(), so), "dense"),
                       ((pool, pool, scales, ids, out, out, so[:, :1]), "scales"),
                       ((pool, pool, scales, ids, out, out, so), "current device")):
        with pytest.raises(ValueError, match=says):
            bros.bros_kv_gather_q8(*args)
    with pytest.raises(ValueError, match="one type"):
        bros.bros_kv_read_q8(pool, pool, scales, None, torch.zeros((0, 2, 128)), torch.zeros((0, 2, 128), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="float32"):
        bros.Rope(torch.zeros((9, 128), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="sections"):
        bros.Rope(torch.zeros((9, 128)), sections=(1, 2, 3, 4, 5))


def test_oracle_rows_match_the_type():
    # the oracle's nearest values against torch's conversion, over all sizes and ties
    rng = np.random.default_rng(1)
    x = rng.standard_normal((300, 128)) * np.exp2(rng.uniform(-20, 20, (300, 1)))
    x[0] = 0
    x[1] = np.arange(128) * 3.5
    x = x.astype(np.float32).astype(np.float64)
    codes, scales = oracle.encode(x)
    e = scales.astype(int) - 127
    amax = np.abs(x).max(-1)
    assert ((amax <= 448 * 2.0 ** e) & ((amax > 224 * 2.0 ** e) | (e == -100))).all()
    z = torch.from_numpy((x / 2.0 ** e[:, None]).astype(np.float32)).to(torch.float8_e4m3fn)
    assert (z.view(torch.uint8).numpy() == codes).all()
    assert np.array_equal(oracle.E4M3, torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)


def test_rope_table():
    from paper_2504_09590_amd.rope import rope_table
    t = rope_table(200001, 64, 10000.0, device="cpu")
    for p, i in ((0, 0), (1, 0), (131072, 0), (200000, 3), (777, 31)):
        a = p * 10000.0 ** (-2 * i / 64)
        assert abs(float(t[p, i]) - np.cos(a)) <= 2.0 ** -24 and abs(float(t[p, 32 + i]) - np.sin(a)) <= 2.0 ** -24
    with pytest.raises(ValueError):
        rope_table(4, 33, device="cpu")
    with pytest.raises(ValueError):
        rope_table(4, 32, inv_freq=[1.0, 2.0], device="cpu")


def decode(**kw):
    a = dict(out=FAKE, q=FAKE, k=FAKE, v=FAKE, s=FAKE, nb=10, bt=FAKE, maxb=4, dir=FAKE, cls=None, dpe=0, ctx=FAKE, max_ctx=64,
             S=2, hq=8, hkv=2, d=128, bs=16, scale=0.0, dtype=1, ws=FAKE, wsb=1 << 40)
    a.update(kw)
    return bros.LIB.bros_attn_decode_q8(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=0), UNSUPPORTED), (dict(dtype=7), DTYPE), (dict(d=64), UNSUPPORTED), (dict(bs=32), UNSUPPORTED),
    (dict(hq=6, hkv=4), SHAPE), (dict(hq=48), UNSUPPORTED), (dict(out=None), NULL), (dict(q=None), NULL), (dict(k=None), NULL),
    (dict(v=None), NULL), (dict(s=None), NULL), (dict(ctx=None), NULL), (dict(bt=None), NULL), (dict(dir=None), NULL),
    (dict(dpe=2), SHAPE), (dict(S=-1), SHAPE), (dict(max_ctx=-1), SHAPE), (dict(nb=0), SHAPE), (dict(maxb=0), SHAPE),
    (dict(out=FAKE + 4), SHAPE), (dict(s=FAKE + 4), SHAPE), (dict(S=2 ** 20, max_ctx=2 ** 31 - 1), SHAPE), (dict(ws=None), -5),
    (dict(wsb=16), -5), (dict(ws=FAKE + 4), -5),
])
def test_decode_rejects(kw, code):
    assert decode(**kw) == code
    assert bros.LIB.bros_last_error().decode() != ""


def test_decode_of_no_sequences():
    assert decode(S=0, out=None, q=None, ws=None) == 0


def test_decode_binding_refuses():
    q, pool = rows(2, 8), torch.zeros((4, 2, 16, 128), dtype=torch.uint8)
    scales, bt = torch.zeros((4, 2, 2, 16), dtype=torch.uint8), torch.zeros((2, 3), dtype=torch.int32)
    d, ctx = torch.ones(2, dtype=torch.int8), torch.ones(2, dtype=torch.int32)
    for args, says in (((q, q, pool, pool, scales, bt, d, None, ctx, 16), "current device"),
                       ((q, q[:1], pool, pool, scales, bt, d, None, ctx, 16), "of one type"),
                       ((q.float(), q, pool, pool, scales, bt, d, None, ctx, 16), "of one type"),
                       ((q, q, pool.bfloat16(), pool, scales, bt, d, None, ctx, 16), "one byte"),
                       ((q, q, pool, pool, scales[:, :1], bt, d, None, ctx, 16), "kv_scales"),
                       ((q, q, pool, pool, scales, bt[:1], d, None, ctx, 16), "block_tables"),
                       ((q, q, pool, pool, scales, bt, d, None, ctx.long(), 16), "length")):
        with pytest.raises(ValueError, match=says):
            bros.bros_attn_decode_q8(*args)


def prefill(**kw):
    a = dict(out=FAKE, q=FAKE, cu_q=FAKE, n=64, max_q=32, k=FAKE, v=FAKE, s=FAKE, nb=10, bt=FAKE, maxb=4, dir=FAKE, cls=None, dpe=0,
             ctx=FAKE, max_ctx=64, S=2, hq=8, hkv=2, d=128, bs=16, scale=0.0, dtype=1, ws=None, wsb=0)
    a.update(kw)
    return bros.LIB.bros_attn_prefill_chunk_q8(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=0), UNSUPPORTED), (dict(dtype=7), DTYPE), (dict(d=64), UNSUPPORTED), (dict(bs=32), UNSUPPORTED),
    (dict(hq=6, hkv=4), SHAPE), (dict(hq=48), UNSUPPORTED), (dict(out=None), NULL), (dict(q=None), NULL), (dict(cu_q=None), NULL),
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(s=None), NULL), (dict(ctx=None), NULL), (dict(bt=None), NULL),
    (dict(dir=None), NULL), (dict(dpe=2), SHAPE), (dict(S=-1), SHAPE), (dict(n=-1), SHAPE), (dict(max_q=0), SHAPE),
    (dict(max_ctx=-1), SHAPE), (dict(nb=0), SHAPE), (dict(maxb=0), SHAPE), (dict(out=FAKE + 4), SHAPE), (dict(s=FAKE + 4), SHAPE),
    (dict(max_ctx=40000), -5), (dict(max_ctx=40000, ws=FAKE, wsb=100), -5), (dict(n=2 ** 30, max_ctx=2 ** 31 - 1), SHAPE),
    (dict(n=2 ** 31 - 1, max_q=2 ** 31 - 1, S=2 ** 20), SHAPE),
])
def test_prefill_rejects(kw, code):
    assert prefill(**kw) == code
    assert bros.LIB.bros_last_error().decode() != ""


def test_prefill_of_nothing():
    assert prefill(S=0, out=None) == 0 and prefill(n=0, q=None) == 0


def test_prefill_binding_refuses():
    q, pool = rows(5, 8), torch.zeros((4, 2, 16, 128), dtype=torch.uint8)
    scales, bt = torch.zeros((4, 2, 2, 16), dtype=torch.uint8), torch.zeros((2, 3), dtype=torch.int32)
    d, ctx, cu = torch.ones(2, dtype=torch.int8), torch.ones(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for args, says in (((q, q, cu, 5, pool, pool, scales, bt, d, None, ctx, 16), "current device"),
                       ((q, q, cu[:2], 5, pool, pool, scales, bt, d, None, ctx, 16), "offset"),
                       ((q[:4], q, cu, 5, pool, pool, scales, bt, d, None, ctx, 16), "of one type"),
                       ((q, q, cu, 5, pool, pool, scales.int(), bt, d, None, ctx, 16), "kv_scales")):
        with pytest.raises(ValueError, match=says):
            bros.bros_attn_prefill_chunk_q8(*args)
