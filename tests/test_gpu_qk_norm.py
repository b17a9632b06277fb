"""Rotary positions and per-head norms of queries and keys on the GPU against their plain 64-bit forms."""
import pytest
import torch

from paper_2604_22808_amd import binding as B
from tests import heads_util as U

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def randn(gen, *shape):
    return torch.randn(shape, generator=gen, dtype=torch.float64)


def rotary_of(d, dims, layout, scaling=0, grid=None, base=10000.0):
    factor, context = (8.0, 4096) if scaling else (1.0, 0)
    r = B.Rotary(d, dims, layout=layout, base=base, scaling=scaling, factor=factor, context=context, grid=grid)
    return r, U.frequencies(dims, base, scaling, factor, context)


def grid_positions(grid, batch):
    n = torch.cartesian_prod(*(torch.arange(g) for g in grid)).reshape(-1, len(grid))
    return n[None].expand(batch, -1, -1)


def rotated_bound(want, size, io):
    # angle 2^-31 turns and conversions, Taylor sums and amplitude within 8 fp32 steps of the pair's size, then the store's own step
    return U.STEP[io] * want.abs() * (1 + 2.0 ** -6) + (16 + 8) * U.F32 * size + 1e-30


ROTARY = [  # batch, tokens, heads, head_dim, axis dims, layout, scaling, grid
    (1, 1, 1, 2, [2], 0, 0, None),
    (3, 1, 16, 64, [64], 0, 3, None),
    (2, 37, 5, 128, [128], 0, 2, None),
    (2, 37, 5, 128, [128], 1, 1, None),
    (1, 60, 3, 64, [16, 24, 24], 1, 0, (3, 4, 5)),
    (2, 60, 40, 128, [44, 42, 42], 0, 0, (3, 4, 5)),
    (1, 12, 2, 96, [32], 0, 0, None),
    (1, 12, 2, 80, [20], 0, 0, None),        # half a rotation of 10 pairs: no aligned pieces
    (1, 12, 2, 80, [20], 1, 0, None),
    (1, 7, 3, 18, [6, 4], 0, 0, None),
    (1, 7, 3, 34, [2, 2, 2, 2], 1, 0, (7, 1, 1, 1)),
    (1, 9, 2, 512, [512], 0, 0, None),
    (1, 9, 2, 256, [0, 100], 1, 0, None),
    (1, 700, 20, 64, [32, 32], 0, 0, (28, 25)),
    (2, 513, 70, 128, [64], 1, 3, None),     # enough rows for four steps a wave
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", ROTARY, ids=str)
def test_rotary_and_its_inverse(case, dtype):
    batch, tokens, heads, d, dims, layout, scaling, grid = case
    io, gen = TYPES[dtype], torch.Generator().manual_seed(sum(map(ord, str(case))))
    rot, (theta, axis, amp) = rotary_of(d, dims, layout, scaling, grid)
    x = randn(gen, batch, tokens, heads, d).to(io)
    if grid:
        pos, given = grid_positions(grid, batch), None
    else:
        pos = torch.randint(-2 ** 31, 2 ** 31, (batch, tokens, len(dims)), generator=gen)
        given = pos.to(torch.int32).cuda()
    dx = x.cuda()
    for inverse in (False, True):
        out = torch.empty_like(dx)
        assert B.rotary_apply(rot, dx, out, positions=given, inverse=inverse) is out
        want = U.rotate(x.double(), pos, theta, axis, amp, layout, inverse)
        # (theta in double precision: at positions of 2^31 its own rounding is 2^31 * 2^-53 radians of the reference)
        bound = rotated_bound(want, U.rotate_size(x.double(), len(theta), amp, layout), io) + 2.0 ** 31 * 2.0 ** -51 * U.rotate_size(x.double(), len(theta), amp, layout)
        U.check((case, dtype, inverse), out, want, bound)
    same = dx.clone()
    B.rotary_apply(rot, same, same, positions=given, inverse=True)     # in place
    assert torch.equal(same, out)
    rest = 2 * len(theta)
    assert torch.equal(out[..., rest:], dx[..., rest:])


def test_positions_forms_and_orders_of_axes():
    """No positions (token index), one list for all entries, and one per entry agree; so do token-major, head-major, sliced and misaligned tensors."""
    gen = torch.Generator().manual_seed(5)
    b, n, h, d = 2, 33, 6, 64
    rot, _ = rotary_of(d, [d], 0)
    x = randn(gen, b, n, h, d).to(torch.bfloat16).cuda()
    want = torch.empty_like(x)
    B.rotary_apply(rot, x, want)
    p = torch.arange(n, dtype=torch.int32).cuda()
    for pos in (p, p[:, None].contiguous(), p[None].repeat(b, 1), p[None, :, None].repeat(b, 1, 1)):
        got = torch.empty_like(x)
        B.rotary_apply(rot, x, got, positions=pos)
        assert torch.equal(got, want)
    hm = x.transpose(1, 2).contiguous().transpose(1, 2)
    out = torch.zeros(b, h, n, d, dtype=x.dtype, device="cuda").transpose(1, 2)
    B.rotary_apply(rot, hm, out)
    assert torch.equal(out, want)
    wide = torch.zeros(b, n, h + 3, d + 5, dtype=x.dtype, device="cuda")
    for off in (0, 1, 5):
        part = wide[:, :, 2:2 + h, off:off + d]
        part.copy_(x)
        B.rotary_apply(rot, part, part)
        assert torch.equal(part, want)
    assert float(wide[:, :, :2].abs().max()) == 0 and float(wide[:, :, 2 + h:].abs().max()) == 0


QK = [  # batch, tokens, q heads, k heads, head_dim, axis dims or None, layout, grid
    (1, 1, 1, 1, 64, [64], 0, None),
    (64, 1, 32, 8, 128, [128], 0, None),
    (2, 60, 5, 5, 64, [16, 24, 24], 1, (3, 4, 5)),
    (1, 131, 12, 4, 128, None, 0, None),
    (2, 9, 3, 1, 80, [32], 0, None),
    (1, 11, 3, 2, 50, [20], 0, None),
    (1, 11, 3, 2, 50, [20], 1, None),
    (1, 5, 2, 1, 512, [256], 1, None),
    (1, 5, 2, 2, 32, [32], 0, None),
    (2, 600, 24, 24, 128, [44, 42, 42], 0, (6, 10, 10)),
    (3, 400, 1, 1, 64, [64], 1, None),
    (1, 17, 4, 0, 64, [64], 0, None),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", QK, ids=str)
def test_norm_and_rotation_forward_and_backward(case, dtype):
    batch, tokens, hq, hk, d, dims, layout, grid = case
    io, gen, eps = TYPES[dtype], torch.Generator().manual_seed(sum(map(ord, str(case)))), 1e-5
    rot, spec = (None, None) if dims is None else rotary_of(d, dims, layout, 0, grid)
    pos = given = None
    if dims is not None:
        pos = grid_positions(grid, batch) if grid else torch.randint(0, 100000, (batch, tokens, len(dims)), generator=gen)
        given = None if grid else pos.to(torch.int32).cuda()
    fused = (randn(gen, batch, tokens, hq + 2 * hk, d) * torch.exp(randn(gen, d))).to(io)
    part = {"q": slice(0, hq), "k": slice(hq, hq + hk)}
    dev = fused.cuda()
    w = {n: (1 + 0.3 * randn(gen, d)).to(io) for n in "qk"}
    dy = {n: randn(gen, batch, h, tokens, d).to(io).transpose(1, 2) for n, h in (("q", hq), ("k", hk))}
    ddy = {n: dy[n].transpose(1, 2).contiguous().cuda().transpose(1, 2) for n in "qk"}
    dw = {n: w[n].cuda() for n in "qk"}
    y = {n: torch.full((batch, h, tokens, d), 7.0, dtype=io, device="cuda").transpose(1, 2) for n, h in (("q", hq), ("k", hk))}
    B.qk_norm(dev[:, :, part["q"]], dev[:, :, part["k"]] if hk else None, dw["q"], dw["k"] if hk else None, y["q"], y["k"] if hk else None,
              eps=eps, rotary=rot, positions=given)
    grad = torch.full_like(dev, 7.0)
    gw = {n: torch.full((d,), 7.0, device="cuda") for n in "qk"}
    args = (dev[:, :, part["q"]], dev[:, :, part["k"]] if hk else None, dw["q"], dw["k"] if hk else None, ddy["q"], ddy["k"] if hk else None,
            grad[:, :, part["q"]], grad[:, :, part["k"]] if hk else None)
    B.qk_norm_backward(*args, gw["q"], gw["k"] if hk else None, eps=eps, rotary=rot, positions=given)
    for n in ("q", "k") if hk else ("q",):
        x, wt = fused[:, :, part[n]].double(), w[n].double()
        r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
        norm_e = (d / 2 + 16) * U.F32       # the sum of squares (half of its relative error reaches r), square root, division, products
        u = x * r * wt
        want = u if rot is None else U.rotate(u, pos, *spec, layout)
        size = u.abs() if rot is None else U.rotate_size(u, len(spec[0]), spec[2], layout)
        U.check((case, dtype, n, "y"), y[n], want, rotated_bound(want, size, io) + norm_e * size)
        g = dy[n].double()
        g_size = g.abs()
        if rot is not None:
            g_size = U.rotate_size(g, len(spec[0]), spec[2], layout)
            g = U.rotate(g, pos, *spec, layout, inverse=True)
        terms = g * x * r
        term_size = g_size * (x * r).abs()
        want_w = terms.sum((0, 1, 2))
        rows = x.shape[0] * x.shape[1] * x.shape[2]
        U.check((case, dtype, n, "dw"), gw[n], want_w, ((24 + norm_e / U.F32) + rows) * U.F32 * term_size.sum((0, 1, 2)) + 1e-30)
        m = (g * wt * x).mean(-1, keepdim=True)
        m_size = (g_size * wt.abs() * x.abs()).mean(-1, keepdim=True)
        want_x = r * (g * wt - x * r * r * m)
        size_x = r * (g_size * wt.abs() + x.abs() * r * r * m_size)
        bound = U.STEP[io] * want_x.abs() * (1 + 2.0 ** -6) + (d + 64) * U.F32 * size_x + 1e-30
        U.check((case, dtype, n, "dx"), grad[:, :, part[n]], want_x, bound)
    # the values of a fused tensor are left alone, and equal calls give equal bits
    assert float((grad[:, :, hq + hk:] - 7.0).abs().sum()) == 0
    again = [t.clone() for t in gw.values()] + [grad.clone()]
    B.qk_norm_backward(*args, gw["q"], gw["k"] if hk else None, eps=eps, rotary=rot, positions=given)
    assert all(torch.equal(a, b) for a, b in zip(again, list(gw.values()) + [grad]))


def test_backward_against_differences():
    """The fp32 gradient against central differences of the fp32 forward pass: step h leaves h^2 of curvature and fp32 steps / h."""
    gen = torch.Generator().manual_seed(3)
    d, n, h = 16, 5, 2
    rot, _ = rotary_of(d, [8], 1)
    x = (randn(gen, 1, n, h, d)).float().cuda()
    w, g = (1 + 0.2 * randn(gen, d)).float().cuda(), randn(gen, 1, n, h, d).float().cuda()

    def loss(x, w):
        y = torch.empty_like(x)
        B.qk_norm(x, None, w, None, y, None, rotary=rot)
        return float((y.double() * g.double()).sum())

    dx, dw = torch.empty_like(x), torch.empty(d, device="cuda")
    B.qk_norm_backward(x, None, w, None, g, None, dx, None, dw, rotary=rot)
    e = 2.0 ** -7
    for target, grad, at in [(x, dx, (0, i % n, i % h, i)) for i in range(d)] + [(w, dw, (i,)) for i in range(d)]:
        hi, lo = target.clone(), target.clone()
        hi[at] += e
        lo[at] -= e
        num = (loss(hi if target is x else x, hi if target is w else w) - loss(lo if target is x else x, lo if target is w else w)) / (2 * e)
        # third derivative of x / |x| at |x| ~ 4 stays below 16 |g|_1 per unit^3: e^2 / 6 of it; fp32 steps of ~160 outputs of size ~3 over 2 e
        assert abs(num - float(grad[at])) < e * e / 6 * 16 * float(g.abs().sum()) / 16 + 160 * 3 * 16 * U.F32 / (2 * e), (at, num, float(grad[at]))


def test_nothing_to_do_and_empty_sums():
    rot, _ = rotary_of(64, [64], 0)
    x = torch.empty(2, 0, 4, 64, device="cuda")
    B.rotary_apply(rot, x, x)
    dw = torch.full((64,), 7.0, device="cuda")
    dk = torch.full((64,), 7.0, device="cuda")
    B.qk_norm(x, x, None, None, x, x)
    B.qk_norm_backward(x, x, None, None, x, x, x, x, dw, dk)
    assert float(dw.abs().sum()) == 0 and float(dk.abs().sum()) == 0


def test_far_strides_pass_32_bits():
    """A view whose rows lie more than 2^32 bytes apart."""
    rot, (theta, axis, amp) = rotary_of(64, [64], 0)
    big = torch.empty(3 * (2 ** 30 + 8), dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((1, 3, 2, 64), (0, 2 ** 30 + 8, 64, 1))
    gen = torch.Generator().manual_seed(9)
    v = randn(gen, 1, 3, 2, 64).to(torch.bfloat16)
    x.copy_(v)
    pos = torch.tensor([[[7], [8], [2 ** 31 - 1]]])
    B.rotary_apply(rot, x, x, positions=pos.to(torch.int32).cuda())
    want = U.rotate(v.double(), pos, theta, axis, amp, 0)
    size = U.rotate_size(v.double(), 32, 1.0, 0)
    U.check("far", x, want, rotated_bound(want, size, torch.bfloat16) + 2.0 ** -20 * size)


def test_captured_and_replayed_on_another_stream():
    """One graph of forward and backward, replayed with eager calls on other streams in between: every replay gives the eager bits."""
    gen = torch.Generator().manual_seed(11)
    b, n, h, d = 1, 300, 8, 64
    rot, _ = rotary_of(d, [d], 0)
    x, g = (randn(gen, b, n, h, d).to(torch.bfloat16).cuda() for _ in range(2))
    w = (1 + 0.3 * randn(gen, d)).to(torch.bfloat16).cuda()
    out = [torch.empty_like(x), torch.empty_like(x), torch.empty(d, device="cuda")]

    def step():
        B.qk_norm(x, None, w, None, out[0], None, rotary=rot)
        B.qk_norm_backward(x, None, w, None, g, None, out[1], None, out[2], rotary=rot)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    del rot     # the launches carry their table
    for i in range(4):
        x.copy_(randn(gen, b, n, h, d).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        rot, _ = rotary_of(d, [d], 0)
        with torch.cuda.stream(side if i % 2 else torch.cuda.current_stream()):
            step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, out)), i
