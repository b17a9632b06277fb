"""Sizes and numbers that the operators around the layer have to refuse, without a GPU."""
import pytest
import torch

from paper_2604_22808_amd import binding as B


class FakeDevice(torch.Tensor):      # a tensor without memory that claims to live on the device: reaches the checks of sizes
    is_cuda = True


def dev(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta").as_subclass(FakeDevice)


BIG = 2 ** 32 + 5      # 5 in 32 bits


def test_axes_beyond_32_bits():
    """The library counts in int32: a longer axis would be cut to its low bits."""
    rot, x, one = B.Rotary(8, [8]), dev(1, BIG, 1, 8), dev(1, 5, 1, 8)
    with pytest.raises(ValueError, match="2\\^31"):
        B.rotary_apply(rot, x, x)
    with pytest.raises(ValueError, match="2\\^31"):
        B.qk_norm(x, None, None, None, x, None)
    with pytest.raises(ValueError, match="2\\^31"):
        B.qk_norm_backward(x, None, None, None, x, None, x, None)
    with pytest.raises(ValueError, match="2\\^31"):
        B.qk_norm(one, dev(1, 5, BIG, 8), None, None, one, dev(1, 5, BIG, 8))
    q, k, off = dev(BIG, 1, 8), dev(5, 1, 8), dev(2, dtype=torch.int32)
    for a, b in ((q, k), (k, q)):
        with pytest.raises(ValueError, match="2\\^31"):
            B.sequence_attention(a, b, b, a, q_offsets=off, k_offsets=off)
    many = dev(BIG, dtype=torch.int32)
    with pytest.raises(ValueError, match="2\\^31"):
        B.sequence_attention(k, k, k, k, q_offsets=many, k_offsets=many)


def test_counts_whose_products_pass_64_bits():
    """Products of three sizes near 2^31 wrap around in 64 bits; they are too many all the same."""
    L, h, top = B.lib(), B.Heads(16, 0, 64, 64), 2 ** 31 - 1
    rot = B.Rotary(64, [64])
    assert L.freqattn_rotary_apply(rot._h, B.BF16, top, top, top, h, None, 0, 0, h, None) == B.EUNSUPPORTED
    s = B.QkShape(batch=top, tokens=top, q_heads=top, k_heads=top, head_dim=64, dtype=B.BF16, eps=1e-6)
    assert L.freqattn_qk_norm(s, None, None, 0, h, h, None, None, h, h, None) == B.EUNSUPPORTED
    assert L.freqattn_qk_norm_backward(s, None, None, 0, h, h, None, None, h, h, h, h, None, None, None, 0, None) == B.EUNSUPPORTED
    q = B.SequenceShape(sequences=top, q_heads=256, kv_heads=256, head_dim=64, q_rows=2 ** 29, k_rows=2 ** 29, dtype=B.BF16, causal=1)
    size = 1 << 62
    assert L.freqattn_sequence_attention(q, None, h, h, h, h, None, 16, size, None) == B.EUNSUPPORTED
    assert L.freqattn_sequence_attention_backward(q, None, h, h, h, h, h, 16, h, h, h, 16, size, None) == B.EUNSUPPORTED
    assert L.freqattn_sequence_attention_workspace(q, None) == 0 and L.freqattn_sequence_attention_backward_workspace(q, None) == 0


def test_an_amplitude_beyond_fp32():
    """The kernels scale in fp32: a larger amplitude would be infinite there, and NaN beside zeros."""
    assert B.Rotary(64, [64], amplitude=3e38).frequencies()[1] == 3e38
    with pytest.raises(B.FreqAttnError) as e:
        B.Rotary(64, [64], amplitude=1e39)
    assert e.value.status == B.EINVAL
