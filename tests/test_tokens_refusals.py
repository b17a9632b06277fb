"""What the operators on token rows have to refuse, without a GPU."""
import math

import pytest
import torch

from paper_2604_22808_amd import binding as B
from tests.test_operators_refusals import BIG, dev

F, I8, U8, I32 = torch.float32, torch.int8, torch.uint8, torch.int32
R, H = B.Rows(16, 64, 64), B.Heads(16, 64, 64, 64)     # addresses that no refused call may reach
TOP = 2 ** 31 - 1


def refused(match, fn, *args, **kw):
    with pytest.raises((ValueError, TypeError), match=match):
        fn(*args, **kw)


def test_library_refuses_norms():
    L = B.lib()
    shape = lambda **kw: B.NormShape(**{**dict(batch=1, rows=2, channels=8, dtype=1, weights_per_batch=0, eps=1e-6), **kw})   # noqa: E731
    fwd = lambda s, x=R, out=R: L.freqattn_layer_norm(s, x, None, None, out, None)   # noqa: E731
    bwd = lambda s, x=R, dx=R, dw=None, ws=None, size=0: L.freqattn_layer_norm_backward(s, x, None, R, dx, dw, None, ws, size, None)   # noqa: E731
    for call in (fwd, bwd):
        assert call(None) == B.EINVAL and call(shape(), x=None) == B.EINVAL
        for kw in (dict(batch=-1), dict(rows=-1), dict(channels=0), dict(channels=-5), dict(dtype=2), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf)):
            assert call(shape(**kw)) == B.EINVAL, kw
        for kw in (dict(channels=16385), dict(batch=TOP, rows=TOP), dict(batch=1 << 16, rows=1 << 15), dict(batch=65536, rows=1, weights_per_batch=1)):
            assert call(shape(**kw)) == B.EUNSUPPORTED, kw
        assert call(shape(rows=0), x=None) == B.OK and call(shape(batch=0), x=None) == B.OK      # nothing to do: no launch
    assert fwd(shape(), out=B.Rows(None, 0, 0)) == B.EINVAL and bwd(shape(), dx=None) == B.EINVAL
    many = shape(rows=100000)
    need = L.freqattn_layer_norm_workspace(many)
    assert need > 0 and L.freqattn_layer_norm_workspace(shape()) == 0 and L.freqattn_layer_norm_workspace(None) == 0
    assert bwd(many, dw=16) == B.EINVAL and bwd(many, dw=16, ws=16, size=need - 1) == B.EINVAL and bwd(many, dw=16, ws=24, size=need) == B.EINVAL
    assert b"workspace" in L.freqattn_last_error(None)


def test_library_refuses_codes_and_products():
    L = B.lib()
    code = lambda dtype=1, b=1, n=1, c=8, x=R, q=R, s=16: L.freqattn_quantize_rows(dtype, b, n, c, x, q, s, None)   # noqa: E731
    assert code(dtype=5) == B.EINVAL and code(b=-1) == B.EINVAL and code(n=-1) == B.EINVAL and code(c=0) == B.EINVAL
    assert code(x=None) == B.EINVAL and code(q=B.Rows(None, 0, 0)) == B.EINVAL and code(s=None) == B.EINVAL
    assert code(c=131072) == B.EUNSUPPORTED and code(b=TOP, n=TOP) == B.EUNSUPPORTED
    assert code(n=0, x=None) == B.OK
    shape = lambda **kw: B.ProductShape(**{**dict(rows=3, channels=32, outputs=5, dtype=1), **kw})   # noqa: E731
    mul = lambda s, a=16, sa=16, w=16, sw=16, out=16: L.freqattn_product_i8(s, a, 32, sa, w, 32, sw, None, out, 5, None)   # noqa: E731
    assert mul(None) == B.EINVAL
    for kw in (dict(rows=-1), dict(outputs=-1), dict(channels=0), dict(dtype=-1)):
        assert mul(shape(**kw)) == B.EINVAL, kw
    for kw in (dict(a=None), dict(sa=None), dict(w=None), dict(sw=None), dict(out=None)):
        assert mul(shape(), **kw) == B.EINVAL, kw
    assert mul(shape(channels=131072)) == B.EUNSUPPORTED
    assert mul(shape(rows=TOP, outputs=TOP)) == B.EUNSUPPORTED and mul(shape(rows=TOP, outputs=TOP), a=17) == B.EUNSUPPORTED
    assert mul(shape(rows=0), a=None) == B.OK and mul(shape(outputs=0)) == B.OK


def test_library_refuses_caches():
    L = B.lib()
    shape = lambda **kw: B.SequenceShape(**{**dict(sequences=2, q_heads=4, kv_heads=2, head_dim=64, q_rows=3, k_rows=100, dtype=1, causal=1), **kw})   # noqa: E731
    cache = lambda **kw: B.Cache8(**{**dict(k_data=16, v_data=16, k_row_stride=128, v_row_stride=128, k_scales=16, v_scales=16, block_rows=64), **kw})   # noqa: E731
    app = lambda s, c, rows=None, k=H: L.freqattn_cache8_append(s, rows, k, H, c, None)   # noqa: E731
    read = lambda s, c, rows=None, k=H: L.freqattn_cache8_read(s, rows, c, k, H, None)   # noqa: E731
    att = lambda s, c, rows=None, k=H: L.freqattn_cache8_attention(s, rows, k, c, H, None, None, 0, None)   # noqa: E731
    off = B.SequenceRows(None, 16, None, None)
    for call in (app, read, att):
        assert call(None, cache()) == B.EINVAL and call(shape(), None) == B.EINVAL and call(shape(), cache(), k=None) == B.EINVAL
        for n in (0, 8, 24, 512, -16):
            assert call(shape(), cache(block_rows=n)) == B.EINVAL
        for kw in (dict(sequences=-1), dict(q_rows=-1), dict(k_rows=-1), dict(kv_heads=0), dict(head_dim=0), dict(dtype=7)):
            assert call(shape(**kw), cache()) == B.EINVAL, kw
        assert call(shape(), cache(), rows=off) == B.EINVAL
        for kw in (dict(k_data=None), dict(v_data=None), dict(k_scales=None), dict(v_scales=None)):
            assert call(shape(), cache(**kw)) == B.EINVAL, kw
        for kw in (dict(head_dim=129), dict(k_rows=1 << 30), dict(sequences=TOP, k_rows=1 << 20, q_rows=1 << 20)):
            assert call(shape(**kw), cache()) == B.EUNSUPPORTED, kw
        assert call(shape(sequences=0), cache()) == B.OK
    assert app(shape(q_rows=0), cache()) == B.OK and read(shape(k_rows=0), cache()) == B.OK and att(shape(q_rows=0), cache()) == B.OK
    assert att(shape(q_heads=3), cache()) == B.EINVAL and att(shape(softmax_scale=math.inf), cache()) == B.EINVAL
    assert L.freqattn_cache8_attention_workspace(None, None) == 0


def test_binding_refuses_norms():
    x, w = dev(2, 5, 64), dev(64)
    refused("torch tensor", B.layer_norm, [1], None, None, x)
    refused("device tensor", B.layer_norm, torch.zeros(5, 64), None, None, torch.zeros(5, 64))
    refused("dtype", B.layer_norm, dev(5, 64, dtype=torch.float16), None, None, x)
    refused("rows, channels", B.layer_norm, dev(64), None, None, dev(64))
    refused("shape", B.layer_norm, x, None, None, dev(2, 5, 65))
    refused("dtype", B.layer_norm, x, None, None, dev(2, 5, 64, dtype=F))
    refused("contiguous", B.layer_norm, x, dev(65), None, x)
    refused("contiguous", B.layer_norm, x, dev(64, dtype=F), None, x)
    refused("contiguous", B.layer_norm, x, dev(3, 64), None, x)
    refused("all", B.layer_norm, x, dev(64), dev(2, 64), x)
    refused("contiguous", B.layer_norm, dev(5, 64), dev(5, 64), None, dev(5, 64))       # without a batch there is one set of weights
    refused("adjacent", B.layer_norm, dev(5, 64, 2)[..., 0], None, None, dev(5, 64))
    refused("expanded", B.layer_norm, x, None, None, dev(1, 5, 64).expand(2, 5, 64))
    refused("2\\^31", B.layer_norm, dev(BIG, 8), None, None, dev(BIG, 8))
    refused("contiguous", B.layer_norm_backward, x, w, x, x, dev(64))
    refused("all", B.layer_norm_backward, x, w, x, x, dev(2, 64, dtype=F))
    refused("shape", B.layer_norm_backward, x, w, dev(2, 4, 64), x)
    refused("expanded", B.layer_norm_backward, x, w, x, dev(2, 1, 64).expand(2, 5, 64))


def test_binding_refuses_codes_and_products():
    x, q, s = dev(5, 64), dev(5, 64, dtype=I8), dev(5, dtype=F)
    refused("dtype", B.quantize_rows, x, dev(5, 64, dtype=U8), s)
    refused("shape", B.quantize_rows, x, dev(5, 63, dtype=I8), s)
    refused("contiguous", B.quantize_rows, x, q, dev(6, dtype=F))
    refused("scales", B.quantize_rows, x, q, None)
    refused("expanded", B.quantize_rows, x, dev(1, 64, dtype=I8).expand(5, 64), s)
    w, ws, out = dev(7, 64, dtype=I8), dev(7, dtype=F), dev(5, 7)
    refused("dtype", B.product_i8, x, s, w, ws, out)
    refused("w must be", B.product_i8, q, s, dev(7, 65, dtype=I8), ws, out)
    refused("w must be", B.product_i8, q, s, dev(1, 7, 64, dtype=I8), ws, out)
    refused("shape", B.product_i8, q, s, w, ws, dev(5, 8))
    refused("dtype", B.product_i8, q, s, w, ws, dev(5, 7, dtype=I8))
    refused("contiguous", B.product_i8, q, dev(7, dtype=F), w, ws, out)
    refused("must be tensors", B.product_i8, q, None, w, ws, out)
    refused("contiguous", B.product_i8, q, s, w, ws, out, bias=dev(7, dtype=F))
    refused("one stride", B.product_i8, dev(2, 9, 64, dtype=I8)[:, :5], dev(2, 5, dtype=F), w, ws, dev(2, 5, 7))
    refused("one stride", B.product_i8, dev(2, 5, 64, dtype=I8), dev(2, 5, dtype=F), w, ws, dev(2, 9, 7)[:, :5])
    refused("2\\^31", B.product_i8, dev(BIG, 64, dtype=I8), dev(BIG, dtype=F), w, ws, dev(BIG, 7))
    refused("2\\^31", B.product_i8, dev(2 ** 16, 2 ** 15, 64, dtype=I8), dev(2 ** 16, 2 ** 15, dtype=F), w, ws, dev(2 ** 16, 2 ** 15, 7))


def test_binding_refuses_caches():
    c = lambda *s: dev(*s, dtype=U8)   # noqa: E731
    ck, sc, k, q = c(3, 100, 2, 64), c(3, 7, 2), dev(3, 4, 2, 64), dev(3, 4, 8, 64)
    cache = (ck, ck, sc, sc, 16)
    for fn, args in ((B.cache8_append, lambda *t: (k, k, *t)), (B.cache8_read, lambda *t: (*t, dev(3, 100, 2, 64), dev(3, 100, 2, 64))), (B.cache8_attention, lambda *t: (q, *t, q))):
        refused("torch tensor", fn, *args(None, ck, sc, sc, 16))
        refused("device tensor", fn, *args(torch.zeros(3, 100, 2, 64, dtype=U8), ck, sc, sc, 16))
        refused("float8_e4m3fn", fn, *args(dev(3, 100, 2, 64), ck, sc, sc, 16))
        refused("one shape", fn, *args(ck, c(3, 100, 2, 65), sc, sc, 16))
        refused("adjacent", fn, *args(c(3, 100, 2, 64, 2)[..., 0], ck, sc, sc, 16))
        refused("block", fn, *args(ck, ck, sc, sc, 24))
        refused("contiguous", fn, *args(ck, ck, c(3, 6, 2), sc, 16))
        refused("contiguous", fn, *args(ck, ck, sc, dev(3, 7, 2), 16))
        refused("must be tensors", fn, *args(ck, ck, sc, None, 16))
        refused("k_lengths", fn, *args(*cache), k_lengths=dev(4, dtype=I32))
    refused("expanded", B.cache8_append, k, k, c(1, 100, 2, 64).expand(3, 100, 2, 64), ck, sc, sc, 16)
    refused("shape", B.cache8_append, k, dev(3, 4, 2, 65), *cache)
    refused("shape", B.cache8_append, dev(3, 4, 3, 64), dev(3, 4, 3, 64), *cache)
    refused("shape", B.cache8_append, dev(2, 4, 2, 64), dev(2, 4, 2, 64), *cache)
    refused("q_offsets", B.cache8_append, dev(4, 2, 64), dev(4, 2, 64), *cache)
    refused("q_offsets", B.cache8_append, k, k, *cache, q_offsets=dev(4, dtype=I32))
    refused("q_offsets", B.cache8_append, dev(9, 2, 64), dev(9, 2, 64), *cache, q_offsets=dev(3, dtype=I32))
    refused("q_lengths", B.cache8_append, k, k, *cache, q_lengths=dev(2, dtype=I32))
    refused("shape", B.cache8_read, *cache, k, k)
    refused("shape", B.cache8_attention, dev(3, 4, 8, 32), *cache, dev(3, 4, 8, 32))
    refused("lse", B.cache8_attention, q, *cache, q, lse=dev(8, 11, dtype=F))
    refused("2\\^31", B.cache8_attention, q, c(3, BIG, 2, 64), c(3, BIG, 2, 64), sc, sc, 16, q)
