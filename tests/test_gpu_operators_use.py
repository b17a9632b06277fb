"""The operators around the layer as programs call them: batches, positions of their own, workspaces of their own."""
import math

import pytest
import torch

from paper_2604_22808_amd import binding as B
from paper_2604_22808_amd import workloads as WL

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,heads,alloc", [("tiny_f32", 2, [1, 4]), ("16k", 3, [1, 2, 4])])
def test_forward_tokens_of_a_batch_with_positions(name, heads, alloc):
    """Two entries, positions one list for all or one each, on one axis and on three: the norms, the rotation and the forward one after the other, bit for bit."""
    wl = WL.WORKLOADS[name]
    io = torch.bfloat16 if wl.dtype == "bf16" else torch.float32
    b, n, d = 2, wl.n_tokens, wl.head_dim
    ctx = B.Context(b, heads, d, wl.grid, B.BF16 if wl.dtype == "bf16" else B.F32, B.make_cfg(**wl.band))
    gen = torch.Generator().manual_seed(5)
    fused = torch.randn(b, n, 3 * heads, d, generator=gen).to(io).cuda()
    q, k, v = (fused[:, :, i * heads:(i + 1) * heads] for i in range(3))
    w = [(1 + 0.2 * torch.randn(d, generator=gen)).to(io).cuda() for _ in range(2)]
    out, want = (torch.empty(b, heads, n, d, dtype=io, device="cuda") for _ in range(2))
    for dims in ([d], [d // 2, d // 4, d // 4]):
        rot = B.Rotary(d, dims)
        each = torch.randint(-1000, 100000, (b, n, len(dims)), generator=gen, dtype=torch.int32).cuda()
        for pos in (each, each[0].contiguous()):
            for eps in (1e-6, None):
                hq, hk, hv = (t.transpose(1, 2).contiguous() for t in (q, k, v))
                if eps is None:
                    for s, t in ((q, hq), (k, hk)):
                        B.rotary_apply(rot, s, t.transpose(1, 2), positions=pos)
                else:
                    B.qk_norm(q, k, *w, hq.transpose(1, 2), hk.transpose(1, 2), eps=eps, rotary=rot, positions=pos)
                ctx.forward(hq, hk, hv, alloc, want)
                out.fill_(7.0)
                ctx.forward_tokens(q, k, v, alloc, out, *w, eps=eps, rotary=rot, positions=pos)
                torch.cuda.synchronize()
                assert torch.equal(out, want), (name, dims, tuple(pos.shape), eps)
    ctx.destroy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,heads", [(1, 4), (700, 12)])
def test_what_the_workspace_of_the_norms_holds_does_not_matter(tokens, heads, dtype):
    io, d = torch.bfloat16 if dtype == "bf16" else torch.float32, 64
    gen = torch.Generator().manual_seed(6)
    x, g = (torch.randn(2, tokens, heads, d, generator=gen).to(io).cuda() for _ in range(2))
    w = (1 + 0.3 * torch.randn(d, generator=gen)).to(io).cuda()
    rot = B.Rotary(d, [d])
    need = B.lib().freqattn_qk_norm_workspace(d)
    res = []
    for fill in (0.0, math.nan, math.inf):
        ws = torch.full((need // 4 + 64,), fill, device="cuda")
        dx, dw = torch.empty_like(x), torch.empty(d, device="cuda")
        B.qk_norm_backward(x, None, w, None, g, None, dx, None, dw, rotary=rot, workspace=ws[:need // 4])
        assert torch.equal(ws[need // 4:].nan_to_num(1.0), torch.full((64,), fill, device="cuda").nan_to_num(1.0))
        res.append((dx, dw))
    for dx, dw in res[1:]:
        assert torch.equal(dx, res[0][0]) and torch.equal(dw, res[0][1])
