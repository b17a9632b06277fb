"""Operators on token rows at the ends of their ranges, against the plain 64-bit forms."""
import math

import pytest
import torch

from paper_2604_22808_amd import binding as B
from paper_2604_22808_amd import workloads as WL
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


SIZES_FAR = [1.5e-45, 3e-44, 1e-42, 1e-40, 1e-38, 1e-30, 1.0, 1e18, 1e30, 3e36, 3e38]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("c", [8, 64, 150, 700, 1900, 5000, 16384])
def test_norm_of_rows_of_any_size_fp32_holds(c, dtype):
    """Rows from the smallest numbers to the largest, each normalised as if it were alone, and beside them the same rows around a large mean of their own."""
    io, x, w, bias, dout = make(c, dtype, 1, 2 * len(SIZES_FAR) + 1, c, False)
    x = x.double().clamp(-4, 4) / 4.1
    for i, s in enumerate(SIZES_FAR):
        x[0, i] *= s
        x[0, len(SIZES_FAR) + i] = 0.75 * s + 0.25 * s * x[0, len(SIZES_FAR) + i]
    x = x.to(io)
    x[0, -1] = torch.where(torch.arange(c) % 3 == 0, -1.0, 1.0) * 3.3e38       # centred values beyond fp32
    assert bool(torch.isfinite(x.float()).all())
    near, far = dout.double(), dout.double()
    for i, s in enumerate(SIZES_FAR + SIZES_FAR + [3e38]):
        far[0, i] = far[0, i] * (1e-25 if s < 1e-20 else 1e20 if s > 1e20 else 1.0)    # dx of 1e-19 to 1e20: neither hidden by the bound's 1e-30 nor infinite
    flat = (x[0].double().var(1, correction=0) == 0)          # (what the type rounds to one value: 0 / 0 with eps 0)
    far, near = far.to(io), near.to(io)
    keep = ~flat
    for eps in (0.0, 1e-6, 1e-31, 1e38):
        rows = keep if eps == 0.0 else torch.ones_like(keep)
        xs, ds = x[:, rows], (near[:, rows], far[:, rows])
        for do, names in zip(ds, (("out", "dw", "db"), ("out", "dx"))):
            got, want = both_passes(xs, w, bias, do, eps), expect(xs, w, bias, in_fp32(eps), io, False, do)
            for name in names:
                U.check((name, eps), got[name], *want[name])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("c", [64, 100, 700, 1999, 5000, 9001])
def test_norm_of_constant_rows_of_any_size(c, dtype):
    """A row of one value gives b, and a gradient of eps^-1/2 (g - mean g), however large the value and however small eps."""
    io, x, w, bias, dout = make(c, dtype, 1, 7, c, False)
    x[0, 0], x[0, 2], x[0, 3], x[0, 5] = 2.0 ** 66, -1e37, 3e38, 2.0 ** 70
    g = dout.double() * w.double()
    for eps in (1e-31, 1e-6):
        got = both_passes(x, w, bias, dout, eps)
        r = 1 / math.sqrt(in_fp32(eps))
        dx = r * (g - g.mean(2, keepdim=True))
        for i in (0, 2, 3, 5) if c == 64 else (2, 3):     # (powers of two: where 1 / channels is none either, their mean is off by a rounding)
            assert torch.equal(got["out"][0, i].cpu(), bias), (eps, i)
            # the mean of g, the root, its product, the store
            bound = r * (U.CHAIN + 4) * U.F32 * (g[0, i].abs().mean() + g[0, i].abs()) + (8 * U.F32 + U.STEP[io] * (1 + 2.0 ** -6)) * dx[0, i].abs()
            U.check(("dx", eps, i), got["dx"][0, i], dx[0, i], bound)
        assert bool(torch.isfinite(got["dw"]).all()), eps
        U.check(("db", eps), got["db"], *expect(x, w, bias, in_fp32(eps), io, False, dout)["db"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", [(2048, 16, 4608), (1990, 130, 4604), (1000, 2064, 2048), (1001, 400, 1999), (2100, 161, 2304), (1900, 33, 2301)])
def test_results_that_pass_through_lds_land_in_their_places(m, k, n, dtype):
    """256 x 256 and 128 x 128 tiles, copied and of any alignment: a wave's lanes store what others computed, one 32-row strip after another.  Sums below 2^24 are exact in
    fp32, and in bf16 rounded once."""
    gen = torch.Generator().manual_seed(m + n)
    a, w = (torch.randint(-40, 41, (r, k), generator=gen).to(torch.int8) for r in (m, n))
    out = torch.full((m, n), U.MARK, dtype=U.TYPES[dtype], device="cuda")
    one = torch.ones(max(m, n), device="cuda")
    for _ in range(3):
        B.product_i8(a.cuda(), one[:m], w.cuda(), one[:n], out)
        assert torch.equal(out.cpu(), (a.double() @ w.double().T).to(U.TYPES[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", [(1, 1024, 8192), (1, 1040, 8208), (16, 528, 8193), (16, 512, 16400), (17, 2048, 4096), (17, 512, 4097), (32, 1040, 4112), (2, 528, 70000), (13, 528, 140001),
                                   (1, 544, 262144)])
def test_few_rows_on_either_side_of_the_choice_of_their_kernel(m, k, n, dtype):
    t, gen = U.TYPES[dtype], torch.Generator().manual_seed(m + n)
    a, w = (torch.randint(-127, 128, (r, k), generator=gen).to(torch.int8) for r in (m, n))
    sa, sw, bias = torch.rand(m, generator=gen) + 0.01, torch.rand(n, generator=gen) * 0.02 + 1e-4, torch.randn(n, generator=gen).to(t)
    rows = torch.full((m, n + 3), U.MARK, dtype=t, device="cuda")
    B.product_i8(a.cuda(), sa.cuda(), w.cuda(), sw.cuda(), rows[:, :n], bias=bias.cuda())
    y = (a.double() @ w.double().T) * sa.double()[:, None] * sw.double()[None]
    want = y + bias.double()
    U.check((m, k, n), rows[:, :n], want, 4 * U.F32 * y.abs() + (U.F32 + U.STEP[t] * (1 + 2.0 ** -6)) * want.abs() + 1e-37)
    assert bool((rows[:, n:] == U.MARK).all())


def definition(q, k, v, causal, scale):
    """Attention of one sequence and head in 64 bits, q [rows, d], keys and values that may be infinite; masked pairs do not count."""
    nq, nk = q.shape[0], k.shape[0]
    seen = torch.arange(nk)[None] <= torch.arange(nq)[:, None] + nk - nq if causal else torch.ones(nq, nk, dtype=torch.bool)
    s = ((q[:, None] * k[None]).sum(2) * scale).masked_fill(~seen, -math.inf)
    p = torch.exp(s - s.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    return torch.where(seen[:, :, None], p[:, :, None] * v[None], 0.0).sum(1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bits", [8, 16, 24])
@pytest.mark.parametrize("rows,cap,d,q_pad", [(1, 200, 64, 0), (20, 200, 128, 0), (150, 300, 64, 0), (150, 300, 72, 0), (3, 5000, 128, 0), (40, 200, 64, 3)])
def test_values_that_read_back_infinite(rows, cap, d, q_pad, bits, dtype):
    """Code 256 at the largest byte that append writes is 2^128: attention takes it as an infinite value, and as an infinite key, whatever bits the queries have."""
    io, heads, block, at = U.TYPES[dtype], 3, 16, 100
    gen = torch.Generator().manual_seed(rows + d)
    codes = [torch.randint(0, 0x7f, (1, cap, heads, d), generator=gen).to(torch.uint8) for _ in range(2)]
    scales = [torch.full((1, -(-cap // block), heads), 117, dtype=torch.uint8) for _ in range(2)]
    hot = at // block
    lo, hi = hot * block, hot * block + block
    # head 0: an infinite value and a negative one; head 1: an infinite key; head 2: neither
    codes[1][0, lo:hi, 0], codes[0][0, lo:hi, 1] = 0, 0
    scales[1][0, hot, 0], scales[0][0, hot, 1] = 247, 247
    codes[1][0, at, 0, 3], codes[1][0, at + 1, 0, 9], codes[0][0, at, 1, 5] = 0x78, 0xf8, 0x78
    q = torch.randn(1, rows, heads, d, generator=gen)
    q = (q.view(torch.int32) & -(1 << (24 - bits))).view(torch.float32).to(io)      # `bits` significant bits
    q[0, :, 1, 5] = torch.where(torch.arange(rows) % 2 == 0, -q[0, :, 1, 5].abs(), q[0, :, 1, 5].abs())
    kv = [U.cache_values(codes[w], scales[w], block).float() for w in range(2)]
    assert bool(torch.isinf(kv[1][0, at, 0, 3])) and bool(torch.isinf(kv[0][0, at, 1, 5]))
    for causal in (False, True):
        for last in (cap, at + 3):      # the row of the infinities in the middle, and among the keys that not every query sees
            dev = torch.empty(1, rows, heads, d + q_pad, dtype=io, device="cuda")[..., q_pad:]
            dev.copy_(q)
            out = torch.empty(1, rows, heads, d + q_pad, dtype=io, device="cuda")[..., q_pad:]
            B.cache8_attention(dev, *(c.cuda() for c in codes), *(s.cuda() for s in scales), block, out, causal=causal, k_lengths=torch.tensor([last], dtype=torch.int32).cuda())
            for h in range(heads):
                first = max(0, rows - last) if causal else 0       # (queries before the first key see nothing)
                want = definition(q[0, :, h].double(), kv[0][0, :last, h].double(), kv[1][0, :last, h].double(), causal, 1 / math.sqrt(d))[first:]
                # scores of up to 8 d^1/2: fp32 sums of three terms a product and probabilities (bf16: one more rounding), as tests of finite caches count them
                size = kv[1][0, :last, h][torch.isfinite(kv[1][0, :last, h])].abs().max().double()
                step = 3 * (2 * U.F32 * (d + 8) * 16 * math.sqrt(d) + 2 * (last + 16) * U.F32) + (2 * U.STEP[io] if io is torch.bfloat16 else 0.0)
                U.check((h, causal, last), out[0, first:, h], want, step * size + U.STEP[io] * want.abs().nan_to_num(0.0, 0.0, 0.0))


@pytest.mark.parametrize("name,heads", [("tiny_f32", 2), ("16k", 8)])
def test_projections_in_8_bits_into_the_frequency_domain_forward(name, heads):
    """Norm, codes and the fused product into a part of wider rows, which forward_tokens takes as they lie: the bits of the same call on copies of their own, eager and captured,
    and every stage before it against its plain form."""
    wl = WL.WORKLOADS[name]
    io, d, n, model = U.TYPES["bf16" if wl.dtype == "bf16" else "f32"], wl.head_dim, wl.n_tokens, 192
    ctx = B.Context(1, heads, d, wl.grid, B.BF16 if wl.dtype == "bf16" else B.F32, B.make_cfg(**wl.band))
    alloc = [1, 4] if heads == 2 else [1, 1, 2, 2, 2, 4, 4, 7]
    gen = torch.Generator().manual_seed(5)
    outs = 3 * heads * d
    w, b = (1 + 0.2 * torch.randn(model, generator=gen)).to(io), (0.2 * torch.randn(model, generator=gen)).to(io)
    wqk = [(1 + 0.2 * torch.randn(d, generator=gen)).to(io).cuda() for _ in range(2)]
    wt = (torch.randn(outs, model, generator=gen) / 14).cuda()
    wc, ws = B.quantize_rows(wt, torch.empty(outs, model, dtype=torch.int8, device="cuda"), torch.empty(outs, device="cuda"))
    rot = B.Rotary(d, [16, 24, 24], layout=B.ROTARY_INTERLEAVED, grid=wl.grid)
    e = lambda *s, dtype=io: torch.empty(s, dtype=dtype, device="cuda")   # noqa: E731
    x, h, hc, hs, out = e(1, n, model), e(1, n, model), e(1, n, model, dtype=torch.int8), e(1, n, dtype=torch.float32), e(1, heads, n, d)
    rows = torch.full((1, n, outs + 24), U.MARK, dtype=io, device="cuda")
    qkv = rows[..., 8:8 + outs]

    def step():
        B.layer_norm(x, w_, b_, h)
        B.quantize_rows(h, hc, hs)
        B.product_i8(hc, hs, wc, ws, qkv)
        q, k, v = (t.unflatten(2, (heads, d)) for t in qkv.split(heads * d, 2))
        return ctx.forward_tokens(q, k, v, alloc, out, *wqk, rotary=rot)

    w_, b_ = w.cuda(), b.cuda()
    fill = lambda: x.copy_(torch.randn(1, n, model, generator=gen).to(io))   # noqa: E731
    fill()
    step()
    torch.cuda.synchronize()
    some = torch.arange(0, n, 37)
    U.check("norm", h[0, some], *U.norm(x[0, some].cpu().double(), w.double(), b.double(), 1e-6, io)["out"])
    codes, scales = U.code_rows(h[0, some].cpu())
    assert torch.equal(hc[0, some].cpu(), codes) and torch.equal(hs[0, some].cpu(), scales)
    y = (codes.double() @ wc.cpu().double().T) * scales.double()[:, None] * ws.cpu().double()
    U.check("product", qkv[0, some], y, (4 * U.F32 + U.STEP[io] * (1 + 2.0 ** -6)) * y.abs() + 1e-37)
    assert bool((rows[..., :8] == U.MARK).all()) and bool((rows[..., 8 + outs:] == U.MARK).all())

    def copies():
        q, k, v = (t.unflatten(2, (heads, d)).contiguous() for t in qkv.split(heads * d, 2))
        return ctx.forward_tokens(q, k, v, alloc, torch.empty_like(out), *wqk, rotary=rot)

    got = out.clone()
    assert torch.equal(got, copies()) and bool(torch.isfinite(got.float()).all())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        fill()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, copies()), i
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out), i
    ctx.destroy()
