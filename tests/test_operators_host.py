"""Host side of the operators around the layer, without a GPU: frequencies, refusals of the library and of the binding."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2604_22808_amd import binding as B
from tests import heads_util as U


@pytest.mark.parametrize("dims,base,scaling,factor,context", [([64], 10000.0, 0, 1.0, 0), ([16, 24, 24], 10000.0, 1, 4.0, 0), ([128], 500000.0, 2, 8.0, 0),
                                                              ([2, 30], 10000.0, 2, 3.0, 0), ([128], 10000.0, 3, 16.0, 4096), ([0, 6, 4, 2], 100.0, 0, 1.0, 0)])
def test_frequencies_and_amplitude(dims, base, scaling, factor, context):
    r = B.Rotary(sum(dims) + 6, dims, base=base, scaling=scaling, factor=factor, context=context)
    got, amp = r.frequencies()
    want, _, want_amp = U.frequencies(dims, base, scaling, factor, context)
    assert got.shape == (sum(dims) // 2,)
    assert np.abs(got / want.numpy() - 1).max() < 1e-13 and abs(amp - want_amp) < 1e-15
    assert B.Rotary(64, [64], scaling=3, factor=4.0, context=100, amplitude=1.5).frequencies()[1] == 1.5


@pytest.mark.parametrize("kw", [dict(head_dim=63), dict(head_dim=0), dict(head_dim=514), dict(axis_dims=[66]), dict(axis_dims=[3]), dict(axis_dims=[0]),
                                dict(axis_dims=[-2, 4]), dict(layout=2), dict(scaling=4), dict(base=1.0), dict(base=math.nan), dict(base=math.inf),
                                dict(scaling=1, factor=0.0), dict(scaling=2, factor=math.inf), dict(scaling=3, factor=0.5, context=10),
                                dict(scaling=3, factor=2.0, context=0), dict(scaling=3, factor=2.0, context=10, beta_fast=1.0), dict(amplitude=-1.0),
                                dict(grid=(-4,)), dict(axis_dims=[2, 2], grid=(4, 0))])
def test_rotary_refuses(kw):
    with pytest.raises(B.FreqAttnError) as e:
        B.Rotary(**{**dict(head_dim=64, axis_dims=[64]), **kw})
    assert e.value.status == B.EINVAL


def test_rotary_handles():
    L = B.lib()
    assert L.freqattn_rotary_create(None, None) == B.EINVAL
    L.freqattn_rotary_destroy(None)
    assert L.freqattn_rotary_frequencies(None, None, None) == B.EINVAL
    with pytest.raises(ValueError):
        B.Rotary(64, [2] * 5)
    with pytest.raises(ValueError):
        B.Rotary(64, [2, 2], grid=(4,))


H = B.Heads(16, 0, 64, 64)     # an address that no refused call may reach


def test_library_refuses_rotations_and_norms():
    L = B.lib()
    r, r2 = B.Rotary(64, [64]), B.Rotary(64, [32, 32])
    grid = B.Rotary(64, [32, 32], grid=(4, 5))
    ap = lambda rot, dtype=1, b=1, n=1, h=1, x=H, out=H: L.freqattn_rotary_apply(rot, dtype, b, n, h, x, None, 0, 0, out, None)   # noqa: E731
    assert ap(None) == B.EINVAL
    assert ap(r._h, dtype=2) == B.EINVAL
    assert ap(r._h, b=-1) == B.EINVAL and ap(r._h, n=-1) == B.EINVAL and ap(r._h, h=-1) == B.EINVAL
    assert ap(r._h, x=None) == B.EINVAL and ap(r._h, out=B.Heads(None, 0, 0, 0)) == B.EINVAL
    assert ap(r2._h) == B.EINVAL and b"positions" in L.freqattn_last_error(None)
    assert ap(grid._h, n=19) == B.EINVAL
    assert ap(r._h, b=0) == B.OK and ap(r._h, h=0, x=None) == B.OK      # nothing to do: no launch
    shape = lambda **kw: B.QkShape(**{**dict(batch=1, tokens=1, q_heads=1, k_heads=1, head_dim=64, dtype=1, eps=1e-6), **kw})   # noqa: E731

    def norm(s, q=H, k=H, oq=H, ok=H, rot=None):
        return L.freqattn_qk_norm(s, rot, None, 0, q, k, None, None, oq, ok, None)

    assert norm(None) == B.EINVAL
    for kw in (dict(batch=-1), dict(tokens=-1), dict(q_heads=-1), dict(k_heads=-1), dict(head_dim=63), dict(head_dim=514), dict(head_dim=0), dict(dtype=9),
               dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf)):
        assert norm(shape(**kw)) == B.EINVAL, kw
    for kw in (dict(q=None), dict(k=None), dict(oq=None), dict(ok=B.Heads(None, 0, 0, 0)), dict(rot=B.Rotary(32, [32])._h)):
        assert norm(shape(), **kw) == B.EINVAL, kw
    assert norm(shape(tokens=0)) == B.OK

    def back(s, q=H, dq=H, dw=None, ws=None, size=0):
        return L.freqattn_qk_norm_backward(s, None, None, 0, q, H, None, None, H, H, dq, H, dw, None, ws, size, None)

    assert back(None) == B.EINVAL and back(shape(), q=None) == B.EINVAL and back(shape(), dq=None) == B.EINVAL and back(shape(q_heads=0)) == B.EINVAL
    need = L.freqattn_qk_norm_workspace(64)
    assert need > 0 and L.freqattn_qk_norm_workspace(0) == 0
    assert back(shape(), dw=16) == B.EINVAL and back(shape(), dw=16, ws=16, size=need - 1) == B.EINVAL and back(shape(), dw=16, ws=24, size=need) == B.EINVAL
    assert back(shape(tokens=0)) == B.OK


def test_library_refuses_sequences():
    L = B.lib()
    shape = lambda **kw: B.SequenceShape(**{**dict(sequences=1, q_heads=4, kv_heads=2, head_dim=64, q_rows=8, k_rows=8, dtype=1, causal=1,   # noqa: E731
                                                   softmax_scale=0.0), **kw})

    def fwd(s, q=H, k=H, v=H, out=H, ws=16, size=1 << 40):
        return L.freqattn_sequence_attention(s, None, q, k, v, out, None, ws, size, None)

    def bwd(s, dout=H, lse=16, dq=H, dk=H, dv=H, ws=16, size=1 << 40):
        return L.freqattn_sequence_attention_backward(s, None, dout, H, H, H, H, lse, dq, dk, dv, ws, size, None)

    assert fwd(None) == B.EINVAL and bwd(None) == B.EINVAL
    for kw in (dict(sequences=-1), dict(q_heads=0), dict(q_heads=3), dict(kv_heads=0), dict(kv_heads=-2), dict(head_dim=0), dict(q_rows=-1), dict(k_rows=-1), dict(dtype=2),
               dict(softmax_scale=math.nan), dict(softmax_scale=math.inf)):
        assert fwd(shape(**kw)) == B.EINVAL and bwd(shape(**kw)) == B.EINVAL, kw
        assert L.freqattn_sequence_attention_workspace(shape(**kw), None) == 0
    for kw in (dict(head_dim=129), dict(q_rows=2 ** 30), dict(k_rows=2 ** 30), dict(sequences=2 ** 20, q_rows=2 ** 12), dict(sequences=2 ** 23)):
        assert fwd(shape(**kw)) == B.EUNSUPPORTED and bwd(shape(**kw)) == B.EUNSUPPORTED, kw
    none = B.Heads(None, 0, 0, 0)
    for kw in (dict(q=None), dict(k=none), dict(v=None), dict(out=none)):
        assert fwd(shape(), **kw) == B.EINVAL, kw
    for kw in (dict(dout=None), dict(lse=None), dict(dq=none), dict(dk=None), dict(dv=None), dict(ws=None), dict(size=4), dict(ws=20)):
        assert bwd(shape(), **kw) == B.EINVAL, kw
    need = L.freqattn_sequence_attention_workspace(shape(k_rows=100000), None)   # (one short row of queries: split along the keys)
    if need:
        assert fwd(shape(k_rows=100000), ws=None) == B.EINVAL and fwd(shape(k_rows=100000), size=need - 1) == B.EINVAL
        assert fwd(shape(k_rows=100000), ws=24) == B.EINVAL
    assert fwd(shape(sequences=0)) == B.OK and bwd(shape(sequences=0)) == B.OK and fwd(shape(q_rows=0), q=None) == B.OK
    assert L.freqattn_last_error(None)


class FakeDevice(torch.Tensor):      # a host tensor that claims to live on the device: reaches the later checks
    is_cuda = True


def dev(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(FakeDevice)


def test_binding_refuses_tensors():
    rot = B.Rotary(64, [64])
    x = dev(2, 5, 3, 64)
    host = torch.zeros(2, 5, 3, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        B.rotary_apply(rot, host, host)
    with pytest.raises(TypeError):
        B.rotary_apply(rot, np.zeros((2, 5, 3, 64)), x)
    with pytest.raises(TypeError):
        B.rotary_apply(None, x, x)
    for bad, match in ((dev(2, 5, 3, 64, dtype=torch.float32), "dtype"), (dev(2, 5, 4, 64), "shape"), (dev(2, 5, 64, 3).transpose(2, 3), "adjacent"),
                       (dev(2, 5, 1, 64).expand(2, 5, 3, 64), "expanded")):
        with pytest.raises(ValueError, match=match):
            B.rotary_apply(rot, x, bad)
    with pytest.raises(ValueError, match="dtype"):
        B.rotary_apply(rot, dev(2, 5, 3, 64, dtype=torch.float64), x)
    with pytest.raises(ValueError, match="made for"):
        B.rotary_apply(rot, dev(2, 5, 3, 32), dev(2, 5, 3, 32))
    with pytest.raises(ValueError):
        B.rotary_apply(rot, dev(5, 3, 64), dev(5, 3, 64))
    for pos in (dev(2, 5, 1, dtype=torch.int64), dev(2, 6, dtype=torch.int32), dev(5, 2, dtype=torch.int32).transpose(0, 1), torch.zeros(5, 2, dtype=torch.int32)):
        with pytest.raises(ValueError, match="positions"):
            B.rotary_apply(rot, x, x, positions=pos)
    with pytest.raises(ValueError, match="without a rotary"):
        B.qk_norm(x, x, None, None, x, x, positions=dev(5, dtype=torch.int32))
    with pytest.raises(ValueError, match="wq"):
        B.qk_norm(x, x, dev(32), None, x, x)
    with pytest.raises(ValueError, match="wk"):
        B.qk_norm(x, x, None, dev(64, dtype=torch.float32), x, x)
    with pytest.raises(ValueError, match="shape"):
        B.qk_norm(x, dev(2, 4, 3, 64), None, None, x, x)
    with pytest.raises(ValueError, match="k must"):
        B.qk_norm(x, dev(5, 3, 64), None, None, x, x)
    with pytest.raises(ValueError, match="dwq"):
        B.qk_norm_backward(x, None, None, None, x, None, x, None, dwq=dev(64))


def test_binding_refuses_sequences():
    q, k = dev(10, 4, 64), dev(10, 2, 64)
    off = dev(3, dtype=torch.int32)
    go = lambda q=q, k=k, v=k, out=q, **kw: B.sequence_attention(q, k, v, out, **{**dict(q_offsets=off, k_offsets=off), **kw})   # noqa: E731
    for kw, match in ((dict(q_offsets=None), "q must be"), (dict(k_offsets=None), "k must be"), (dict(v=dev(9, 2, 64)), "shape"), (dict(out=dev(10, 2, 64)), "shape"),
                      (dict(k_offsets=dev(4, dtype=torch.int32)), "number of sequences"), (dict(q_offsets=dev(3, dtype=torch.int64)), "q_offsets"),
                      (dict(k_lengths=dev(3, dtype=torch.int32)), "k_lengths"), (dict(q_lengths=torch.zeros(2, dtype=torch.int64)), "q_lengths"),
                      (dict(k=dev(10, 2, 32), v=dev(10, 2, 32)), "head_dim"), (dict(lse=dev(4, 9, dtype=torch.float32)), "lse"),
                      (dict(q_offsets=[0, 5, 10]), "q_offsets")):
        with pytest.raises(ValueError, match=match):
            go(**kw)
    with pytest.raises(ValueError, match="lse"):
        B.sequence_attention_backward(q, q, k, k, q, None, q, k, k, q_offsets=off, k_offsets=off)


def test_forward_tokens_refuses():
    ctx = B.Context(1, 2, 64, (4, 8, 8), B.BF16, B.make_cfg(mid_block=16, mid_stride=4, high_window=32, n_summary=4), path=B.PATH_TABLES_ONLY)
    L, cfg = B.lib(), C.byref(ctx.cfg)
    ha = (C.c_int32 * 2)(1, 4)
    go = lambda c=ctx._h, q=H, v=H, alloc=ha, out=32: L.freqattn_forward_tokens(c, q, H, v, None, None, 1e-6, None, None, 0, cfg, alloc, out, None)   # noqa: E731
    assert go(c=None) == B.EINVAL and go(q=None) == B.EINVAL and go(v=B.Heads(None, 0, 0, 0)) == B.EINVAL and go(alloc=None) == B.EINVAL and go(out=None) == B.EINVAL
    assert go() == B.EUNSUPPORTED and b"tables-only" in L.freqattn_last_error(ctx._h)
    q, out = dev(1, 256, 2, 64), dev(1, 2, 256, 64)
    for kw, match in ((dict(q=dev(1, 2, 256, 64)), "shape"), (dict(out=dev(1, 256, 2, 64)), "shape"), (dict(head_alloc=[1]), "head_alloc"), (dict(wq=dev(32)), "wq"),
                      (dict(rotary=B.Rotary(32, [32])), "made for"), (dict(positions=dev(256, dtype=torch.int32)), "without a rotary"),
                      (dict(v=dev(1, 256, 2, 64, dtype=torch.float32)), "dtype")):
        with pytest.raises(ValueError, match=match):
            ctx.forward_tokens(**{**dict(q=q, k=q, v=q, head_alloc=[1, 4], out=out), **kw})
