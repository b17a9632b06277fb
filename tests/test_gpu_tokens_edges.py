"""Operators on token rows at the ends of their ranges, against the plain 64-bit forms."""
import math

import pytest
import torch

from paper_2604_22808_amd import binding as B
from tests import tokens_util as U
from tests.test_gpu_layer_norm import expect, make

pytestmark = pytest.mark.gpu


def both_passes(x, w, bias, dout, eps):
    x, w, bias, dout = (t.cuda() for t in (x, w, bias, dout))
    out, dx = torch.empty_like(x), torch.empty_like(x)
    dw, db = (torch.empty(w.shape, device="cuda") for _ in range(2))
    B.layer_norm(x, w, bias, out, eps=eps)
    B.layer_norm_backward(x, w, dout, dx, dw, db, eps=eps)
    return dict(out=out, dx=dx, dw=dw, db=db)


def in_fp32(eps):
    return float(torch.tensor(eps))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("c,size", [(64, 1e37), (130, 8e36), (700, 2e36), (2048, 3e35), (5000, 1e35), (9000, 2e35)])
def test_norm_of_rows_whose_sum_leaves_fp32(c, size, dtype):
    """Rows of one sign, finite, whose sum is not, beside ordinary ones."""
    io, x, w, bias, dout = make(c, dtype, 1, 11, c, False)
    x = x.double()
    x[0, 2], x[0, 9] = size * (1 + 0.1 * x[0, 2]), -size * (1 + 0.1 * x[0, 9])
    x = x.to(io)
    assert not bool(torch.isfinite(x[0, 2].float().sum())) and bool(torch.isfinite(x.float()).all())
    big = dout.clone()
    big[0, 2], big[0, 9] = dout[0, 2] * 2.0 ** 40, dout[0, 9] * 2.0 ** 40      # gradients of dx that the bound's own 1e-30 does not hide
    for eps in (0.0, 1e-6):
        for do in (dout, big):
            got, want = both_passes(x, w, bias, do, eps), expect(x, w, bias, in_fp32(eps), io, False, do)
            for name in got:
                U.check((name, eps), got[name], *want[name])
