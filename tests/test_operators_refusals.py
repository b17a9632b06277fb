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
