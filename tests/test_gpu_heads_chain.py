"""The operators around the layer together, as a model uses them: projections to norms, rotation, attention and back, and into the frequency-domain forward."""
import math

import pytest
import torch

from paper_2604_22808_amd import binding as B
from paper_2604_22808_amd import workloads as WL
from tests import heads_util as U

pytestmark = pytest.mark.gpu


def test_projection_to_attention_and_back():
    """Packed sequences, grouped heads, fp32: out and the gradients of the fused projection and of the norms' weights against autograd in 64 bits.
    With norms, |q| = |k| = sqrt(d) w: scores stay below sqrt(d) max w^2 < 12, and relative errors of q and k of (d / 2 + 48) steps move them by less than
    2 * 12 * 80 steps, probabilities by twice that relative to themselves; the gradients are sums of products of four such factors."""
    gen = torch.Generator().manual_seed(7)
    h, hk, d, lengths = 4, 2, 64, (70, 1, 45)
    n, eps = sum(lengths), 1e-5
    rot = B.Rotary(d, [32], scaling=B.ROTARY_BY_PARTS, factor=4.0, context=64)
    theta, axis, amp = U.frequencies([32], 10000.0, 3, 4.0, 64)
    pos = torch.cat([torch.arange(m) for m in lengths])
    qkv = torch.randn(1, n, h + 2 * hk, d, generator=gen, dtype=torch.float64).float()
    wq, wk = (1 + 0.1 * torch.randn(d, generator=gen, dtype=torch.float64).float() for _ in range(2))
    dout = torch.randn(n, h, d, generator=gen, dtype=torch.float64).float()
    off = torch.tensor([0, 70, 71, 116], dtype=torch.int32).cuda()

    x, g = qkv.cuda(), dout.cuda()
    w = [wq.cuda(), wk.cuda()]
    q, k, v = x[:, :, :h], x[:, :, h:h + hk], x[:, :, h + hk:]
    e = lambda *s: torch.empty(s, device="cuda")   # noqa: E731
    qn, kn, out, lse = e(1, n, h, d), e(1, n, hk, d), e(n, h, d), e(h, n)
    how = dict(causal=True, q_offsets=off, k_offsets=off)
    at = dict(eps=eps, rotary=rot, positions=pos.to(torch.int32).cuda())
    B.qk_norm(q, k, *w, qn, kn, **at)
    B.sequence_attention(qn[0], kn[0], v[0], out, lse=lse, **how)
    dqn, dkn, dx = torch.empty_like(qn), torch.empty_like(kn), torch.empty_like(x)
    B.sequence_attention_backward(g, qn[0], kn[0], v[0], out, lse, dqn[0], dkn[0], dx[0, :, h + hk:], **how)
    dw = [e(d), e(d)]
    B.qk_norm_backward(q, k, *w, dqn, dkn, dx[:, :, :h], dx[:, :, h:h + hk], *dw, **at)

    X, W = qkv.double().requires_grad_(), [t.double().requires_grad_() for t in (wq, wk)]

    def normed(t, wt):
        u = t * (t.square().mean(-1, keepdim=True) + eps).rsqrt() * wt
        return U.rotate(u, pos[None, :, None], theta, axis, amp, 0)

    Q, K, V = normed(X[:, :, :h], W[0])[0], normed(X[:, :, h:h + hk], W[1])[0], X[0, :, h + hk:]
    want = []
    for a, b in zip(off.tolist(), off.tolist()[1:]):
        m = b - a
        s = torch.einsum("ihd,jhd->hij", Q[a:b], K[a:b].repeat_interleave(h // hk, 1)) / math.sqrt(d)
        s = s.masked_fill(torch.ones(m, m).triu(1).bool(), -math.inf)
        want.append(torch.einsum("hij,jhd->ihd", s.softmax(-1), V[a:b].repeat_interleave(h // hk, 1)))
    want = torch.cat(want)
    gx, gq, gk = torch.autograd.grad(want, [X, *W], dout.double())
    step = 2 * 2 * 12 * 80 * U.F32       # relative error of a probability
    one = torch.ones
    U.check("out", out, want, step * V.abs().max() * one(want.shape))
    # scale |q| |k| dS: |dS| <= P |dout| |v| 2, over at most 70 keys and 2 heads of a group; weights' gradients sum over the rows
    size = float(gx.abs().max())
    U.check("d qkv", dx, gx, 8 * step * size * one(gx.shape))
    for name, got, ref in (("dwq", dw[0], gq), ("dwk", dw[1], gk)):
        U.check(name, got, ref, 8 * step * size * n * one(ref.shape))


@pytest.mark.parametrize("name,heads", [("tiny_f32", 2), ("16k", 8)])
def test_forward_from_token_major_projections(name, heads):
    """forward_tokens is the norms, the rotation and the forward one after the other, bit for bit; also without norms, without rotation, from tensors whose rows
    are not aligned, and captured into a graph."""
    wl = WL.WORKLOADS[name]
    io = torch.bfloat16 if wl.dtype == "bf16" else torch.float32
    d, grid = wl.head_dim, wl.grid
    n = wl.n_tokens
    ctx = B.Context(1, heads, d, grid, B.BF16 if wl.dtype == "bf16" else B.F32, B.make_cfg(**wl.band))
    alloc = [1, 4] if heads == 2 else [1, 1, 2, 2, 2, 4, 4, 7]
    gen = torch.Generator().manual_seed(3)
    fused = torch.randn(1, n, 3 * heads, d, generator=gen).to(io).cuda()
    odd = torch.zeros(1, n, 3 * heads, d + 1, dtype=io, device="cuda")[..., 1:]
    odd.copy_(fused)
    w = [(1 + 0.2 * torch.randn(d, generator=gen)).to(io).cuda() for _ in range(2)]
    rot = B.Rotary(d, [16, 24, 24], layout=B.ROTARY_INTERLEAVED, grid=grid)
    out, want = (torch.empty(1, heads, n, d, dtype=io, device="cuda") for _ in range(2))
    for x in (fused, odd):
        q, k, v = x[:, :, :heads], x[:, :, heads:2 * heads], x[:, :, 2 * heads:]
        for eps, r in ((1e-6, rot), (1e-6, None), (None, rot), (None, None)):
            hq, hk, hv = (t.transpose(1, 2).contiguous() for t in (q, k, v))
            if eps is not None:
                B.qk_norm(q, k, *w, hq.transpose(1, 2), hk.transpose(1, 2), eps=eps, rotary=r)
            elif r is not None:
                for s, t in ((q, hq), (k, hk)):
                    B.rotary_apply(r, s, t.transpose(1, 2))
            ctx.forward(hq, hk, hv, alloc, want)
            out.fill_(7.0)
            ctx.forward_tokens(q, k, v, alloc, out, *w, eps=eps, rotary=r)
            torch.cuda.synchronize()
            assert torch.equal(out, want), (name, eps, r is not None)
    q, k, v = (fused[:, :, i * heads:(i + 1) * heads] for i in range(3))
    graph = torch.cuda.CUDAGraph()
    ctx.forward_tokens(q, k, v, alloc, out, *w, rotary=rot)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ctx.forward_tokens(q, k, v, alloc, out, *w, rotary=rot)
    for i in range(3):
        fused.copy_(torch.randn(1, n, 3 * heads, d, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        ctx.forward_tokens(q, k, v, alloc, out, *w, rotary=rot)
        torch.cuda.synchronize()
        assert torch.equal(got, out), i
    with pytest.raises(B.FreqAttnError) as e:
        ctx.forward_tokens(q, k, v, alloc, out, rotary=B.Rotary(d, [32, 32], grid=(3, 5)))
    assert e.value.status == B.EINVAL and "grid" in str(e.value)
    ctx.destroy()
