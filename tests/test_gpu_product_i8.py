"""Rows in 8-bit integers and their products on the GPU, against whole numbers on the host."""
import math

import pytest
import torch

from paper_2604_22808_amd import binding as B
from tests import tokens_util as U

pytestmark = pytest.mark.gpu


def codes_of(x):
    codes, scales = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(x.shape[:-1], device="cuda")
    B.quantize_rows(x, codes, scales)
    return codes, scales


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,c", [(1, 1), (3, 7), (70, 16), (33, 65), (5, 250), (21, 150), (11, 350), (9, 601), (64, 512), (9, 1000), (40, 1536), (6, 2048), (4, 2500), (3, 3333), (5, 4096), (4, 5001), (3, 7001), (3, 16384), (2, 20001), (2, 131071)])
def test_codes_are_exact(n, c, dtype):
    io, gen = U.TYPES[dtype], torch.Generator().manual_seed(n * c)
    x = torch.randn(n, c, generator=gen, dtype=torch.float64).to(io)
    x *= torch.exp2(torch.randint(-30, 30, (n, 1), generator=gen).double()).to(io)
    x[0, c // 2:] = x[0].abs().max() / 2        # on the border between two codes
    if n > 2:
        x[1] = 0.0
        x[2] = torch.round(x[2].double() / x[2].double().abs().max() * 254).to(io)     # many borders: half codes of a = 254
    want, scales = U.code_rows(x)
    for pad in (0, 5):
        at = torch.zeros(n, c + pad, dtype=io, device="cuda")[:, :c]
        at.copy_(x)
        out = torch.full((n, c + pad), 99, dtype=torch.int8, device="cuda")
        s = torch.empty(n, device="cuda")
        B.quantize_rows(at, out[:, :c], s)
        assert torch.equal(out[:, :c].cpu(), want) and torch.equal(s.cpu(), scales)
        assert bool((out[:, c:] == 99).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_codes_of_rows_of_any_size_and_not_finite(dtype):
    io = U.TYPES[dtype]
    gen = torch.Generator().manual_seed(2)
    x = torch.randn(12, 300, generator=gen, dtype=torch.float64)
    for i, e in enumerate((-140, -126, -118, -60, 0, 60, 120)):
        x[i] = x[i] / x[i].abs().max() * 2.0 ** e
    x = x.to(io)
    x[8, 17], x[9, 18], x[10, 299] = math.inf, math.nan, -math.inf
    codes, scales = codes_of(x.cuda())
    want, ws = U.code_rows(x)
    assert torch.equal(codes.cpu(), want)
    U.check("scales", scales, ws.double(), torch.zeros(12))


def test_codes_of_a_batch_of_any_strides():
    x = torch.randn(3, 10, 96, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    want, scales = U.code_rows(x.reshape(30, 96))
    at = x.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    codes = torch.empty(10, 3, 96, dtype=torch.int8, device="cuda").transpose(0, 1)
    s = torch.empty(3, 10, device="cuda")
    B.quantize_rows(at, codes, s)
    assert torch.equal(codes.cpu().reshape(30, 96), want) and torch.equal(s.cpu().reshape(30), scales)
    B.quantize_rows(at[:0], codes[:0], s[:0])


def case(seed, m, k, n, top=127):
    gen = torch.Generator().manual_seed(seed)
    a, w = (torch.randint(-top, top + 1, (r, k), generator=gen).to(torch.int8) for r in (m, n))
    return a, w, torch.rand(m, generator=gen) + 0.01, torch.rand(n, generator=gen) * 0.02 + 1e-4, torch.randn(n, generator=gen)


def expect(a, w, sa, sw, bias, io):
    acc = (a.double() @ w.double().T)           # whole numbers below 2^53
    y = acc * sa.double()[:, None] * sw.double()[None]
    bound = 4 * U.F32 * y.abs()
    if bias is not None:
        y = y + bias.double()
        bound = bound + U.F32 * y.abs()
    return y, bound + U.STEP[io] * y.abs() * (1 + 2.0 ** -6) + 1e-37


SIZES = [(1, 1, 1), (1, 16, 16), (2, 15, 3), (1, 2048, 48), (16, 2048, 6144), (5, 1040, 250), (17, 512, 100), (33, 4096, 40), (64, 144, 1000), (65, 128, 64), (100, 96, 130),
         (333, 1000, 1100), (200, 1008, 129), (257, 2048, 512), (128, 256, 128), (1000, 384, 700), (513, 1536, 4608), (2100, 160, 2304), (70000, 64, 48), (70001, 48, 100), (66000, 80, 200), (32, 304, 4000), (3, 8192, 1024), (70, 131056, 65),
         (1000, 2064, 2048), (300, 4112, 608), (64, 656, 1000), (40, 128, 64),
         (2000, 400, 4600), (2001, 640, 4603), (1990, 128, 4604), (2048, 16, 4608), (2047, 1280, 4601), (2100, 161, 2304), (1900, 33, 2301), (2050, 129, 2400)]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_products(m, k, n, io):
    t = U.TYPES[io]
    a, w, sa, sw, bias = case(m + k + n, m, k, n)
    for b in (None, bias.to(t)):
        out = torch.full((m, n + 3), U.MARK, dtype=t, device="cuda")
        B.product_i8(a.cuda(), sa.cuda(), w.cuda(), sw.cuda(), out[:, :n], bias=None if b is None else b.cuda())
        U.check((m, k, n, io), out[:, :n], *expect(a, w, sa, sw, b, t))
        assert bool((out[:, n:] == U.MARK).all())


@pytest.mark.parametrize("m", [5, 60, 200, 900, 2000])
def test_rows_of_any_stride_and_address(m):
    k, n = 272, 4700 if m == 2000 else 96
    a, w, sa, sw, _ = case(m, m, k, n)
    want = expect(a, w, sa, sw, None, torch.float32)
    for pad, lead in ((16, 0), (16, 16), (1, 0), (0, 1), (7, 3)):
        def place(x):
            at = torch.full((lead + x.shape[0] * (k + pad),), 77, dtype=torch.int8, device="cuda")[lead:].view(-1, k + pad)[:, :k]
            at.copy_(x)
            return at
        rows = torch.full((m, n + pad), U.MARK, device="cuda")
        out = rows[:, :n]
        B.product_i8(place(a), sa.cuda(), place(w), sw.cuda(), out)
        U.check((m, pad, lead), out, *want)
        assert bool((rows[:, n:] == U.MARK).all())


def test_sums_that_need_all_32_bits():
    """Codes of -128 and 127 over the most channels: 131071 * 2^14 is just below 2^31; sums are exact."""
    for m, k in ((2, 131071), (80, 131056)):
        a = torch.full((m, k), -128, dtype=torch.int8)
        w = torch.full((40, k), -128, dtype=torch.int8)
        w[1], w[2, 5:] = 127, 127
        out = torch.empty(m, 40, device="cuda")
        one = torch.ones(m, device="cuda"), torch.ones(40, device="cuda")
        B.product_i8(a.cuda(), one[0], w.cuda(), one[1], out)
        want = (a.double() @ w.double().T)
        U.check((m, k), out, want, U.F32 * want.abs())


def test_scales_that_are_not_finite_or_far_apart():
    a, w, sa, sw, bias = case(9, 70, 64, 40)
    sa[3], sa[5], sa[7], sw[2] = math.nan, 0.0, 1e38, 1e-38
    for rows in (8, 70):
        out = torch.empty(rows, 40, device="cuda")
        B.product_i8(a[:rows].cuda(), sa[:rows].cuda(), w.cuda(), sw.cuda(), out)
        got = out.cpu()
        assert bool(torch.isnan(got[3]).all()) and bool((got[5] == 0).all())
        want = (a[7].double() @ w.double().T) * sa[7].double() * sw.double()     # some are finite, though the sum times the larger scale is not
        assert torch.equal(torch.isfinite(got[7]), want.abs() <= 3.4028235e38) and bool(torch.isfinite(got[7, 2]))


@pytest.mark.parametrize("m,k", [(5, 32), (5, 33), (70, 32), (1500, 32), (2000, 32)])
def test_sums_of_zero_between_scales_whose_product_leaves_fp32(m, k):
    n = 4600 if m == 2000 else 1500
    a, w = torch.ones(m, k, dtype=torch.int8), torch.ones(n, k, dtype=torch.int8)
    a[:, k - 1] = 1 - k      # sums of zero
    a[1] = 1
    out = torch.full((m, n), U.MARK, device="cuda")
    big = 2.0 ** 100
    B.product_i8(a.cuda(), torch.full((m,), big, device="cuda"), w.cuda(), torch.full((n,), big, device="cuda"), out, torch.ones(n, device="cuda"))
    got = out.cpu()
    assert bool((got[1] == math.inf).all())
    got[1] = 1.0
    assert bool((got == 1.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_linear_layer_in_8_bits(dtype):
    """Rows coded on the device times weights coded by the same call: the product of the coded values, and near the product of the values."""
    io, gen = U.TYPES[dtype], torch.Generator().manual_seed(11)
    x, wt = torch.randn(2, 75, 320, generator=gen).to(io), torch.randn(200, 320, generator=gen).to(io)
    codes, scales = codes_of(x.cuda())
    wc, ws = codes_of(wt.cuda())
    out = torch.empty(2, 75, 200, dtype=io, device="cuda")
    B.product_i8(codes, scales, wc, ws, out)
    want, bound = expect(codes.cpu().reshape(150, 320), wc.cpu(), scales.cpu().reshape(150), ws.cpu(), None, io)
    U.check("out", out.reshape(150, 200), want, bound)
    true = x.double().reshape(150, 320) @ wt.double().T
    # half a code of either side in every term, and both
    sa, sw = scales.cpu().double().reshape(150, 1), ws.cpu().double()[:, None]
    off = 0.5001 * sa * wt.double().abs().sum(1) + (x.double().abs().reshape(150, 320).sum(1, keepdim=True) * 0.5001 + 0.26 * 320 * sa) * sw.T
    U.check("true", out.reshape(150, 200), true, off + bound + 1e-5)


def test_no_rows_no_outputs():
    a, w, sa, sw, _ = case(1, 4, 32, 5)
    B.product_i8(a[:0].cuda(), sa[:0].cuda(), w.cuda(), sw.cuda(), torch.empty(0, 5, device="cuda"))
    B.product_i8(a.cuda(), sa.cuda(), w[:0].cuda(), sw[:0].cuda(), torch.empty(4, 0, device="cuda"))


def test_codes_behind_2_31_bytes():
    base = torch.zeros(2100, 1 << 21, dtype=torch.int8, device="cuda")
    a, w, sa, sw, _ = case(12, 2100, 64, 40)
    base[:, :64] = a.cuda()
    out = torch.empty(2100, 40, device="cuda")
    B.product_i8(base[:, :64], sa.cuda(), w.cuda(), sw.cuda(), out)
    U.check("far", out, *expect(a, w, sa, sw, None, torch.float32))
    out = torch.empty(40, 2100, device="cuda")
    B.product_i8(w.cuda(), sw.cuda(), base[:, :64], sa.cuda(), out)
    U.check("far weights", out.T, *expect(a, w, sa, sw, None, torch.float32))
