"""The operators on token rows one after the other, as a layer with 8-bit projections and an 8-bit cache calls them: prompts, single tokens, graphs, streams."""
import math

import pytest
import torch

from paper_2604_22808_amd import binding as B
from tests import heads_util as H
from tests import tokens_util as U

pytestmark = pytest.mark.gpu

MODEL, HEADS, KV, D, BLOCK, CAP, SEQ = 256, 4, 2, 64, 16, 80, 3


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


class Layer:
    def __init__(self, dtype, seed=1):
        self.io, gen = U.TYPES[dtype], torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=gen)   # noqa: E731
        self.w, self.b = (1 + 0.2 * r(MODEL)).to(self.io).cuda(), (0.2 * r(MODEL)).to(self.io).cuda()
        self.wq, self.wk = (1 + 0.2 * r(D)).to(self.io).cuda(), (1 + 0.2 * r(D)).to(self.io).cuda()
        self.proj = self.coded(r((HEADS + 2 * KV) * D, MODEL).cuda() / 16)
        self.back = self.coded(r(MODEL, HEADS * D).cuda() / 16)
        self.rotary = B.Rotary(D, [D])
        self.cache = [torch.zeros(SEQ, CAP, KV, D, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
        self.scales = [torch.zeros(SEQ, -(-CAP // BLOCK), KV, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def coded(self, w):
        codes, scales = torch.empty(w.shape, dtype=torch.int8, device="cuda"), torch.empty(w.shape[0], device="cuda")
        return B.quantize_rows(w, codes, scales)

    def buffers(self, n):
        e = lambda *s, dtype=self.io: torch.empty(SEQ, n, *s, dtype=dtype, device="cuda")   # noqa: E731
        return dict(x=e(MODEL), pos=e(dtype=torch.int32), filled=torch.empty(SEQ, dtype=torch.int32, device="cuda"), h=e(MODEL), hc=e(MODEL, dtype=torch.int8),
                    hs=e(dtype=torch.float32), qkv=e((HEADS + 2 * KV) * D), q=e(HEADS, D), k=e(KV, D), o=e(HEADS, D), oc=e(HEADS * D, dtype=torch.int8),
                    os=e(dtype=torch.float32), y=e(MODEL))

    def step(self, t):
        n = t["x"].shape[1]
        B.layer_norm(t["x"], self.w, self.b, t["h"])
        B.quantize_rows(t["h"], t["hc"], t["hs"])
        B.product_i8(t["hc"], t["hs"], *self.proj, t["qkv"])
        qkv = t["qkv"].view(SEQ, n, HEADS + 2 * KV, D)
        B.qk_norm(qkv[:, :, :HEADS], qkv[:, :, HEADS:HEADS + KV], self.wq, self.wk, t["q"], t["k"], rotary=self.rotary, positions=t["pos"])
        cache = (*self.cache, *self.scales, BLOCK)
        B.cache8_append(t["k"], qkv[:, :, HEADS + KV:], *cache, k_lengths=t["filled"])
        B.cache8_attention(t["q"], *cache, t["o"], causal=True, k_lengths=t["filled"])
        B.quantize_rows(t["o"].view(SEQ, n, HEADS * D), t["oc"], t["os"])
        B.product_i8(t["oc"], t["os"], *self.back, t["y"])
        return t["y"]

    def fill(self, t, seed, filled):
        n = t["x"].shape[1]
        t["x"].copy_(torch.randn(SEQ, n, MODEL, generator=torch.Generator().manual_seed(seed)).to(self.io))
        t["filled"].copy_(ints(filled))
        t["pos"].copy_(torch.arange(n, dtype=torch.int32)[None] + torch.tensor(filled, dtype=torch.int32)[:, None] - n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_layer_on_prompts_and_tokens(dtype):
    """Every stage against its plain form on what the stage before it gave."""
    layer = Layer(dtype)
    io = layer.io
    want = [(torch.zeros(SEQ, CAP, KV, D, dtype=torch.uint8), torch.zeros(SEQ, -(-CAP // BLOCK), KV, dtype=torch.uint8)) for _ in range(2)]
    for n, filled, seed in ((40, [40, 40, 40], 1), (1, [41, 41, 41], 2), (1, [42, 42, 42], 3), (17, [59, 59, 59], 4), (1, [60, 60, 60], 5)):
        t = layer.buffers(n)
        layer.fill(t, seed, filled)
        layer.step(t)
        torch.cuda.synchronize()
        flat = lambda name: t[name].cpu().reshape(SEQ * n, -1)   # noqa: E731
        U.check("norm", flat("h"), *U.norm(flat("x").double(), layer.w.cpu().double(), layer.b.cpu().double(), 1e-6, io)["out"])
        for codes, scales, src in (("hc", "hs", "h"), ("oc", "os", "o")):
            c, s = U.code_rows(flat(src))
            assert torch.equal(flat(codes), c) and torch.equal(flat(scales)[:, 0], s)
        for codes, scales, (w, ws), out in (("hc", "hs", layer.proj, "qkv"), ("oc", "os", layer.back, "y")):
            y = (flat(codes).double() @ w.cpu().double().T) * flat(scales).double() * ws.cpu().double()
            U.check(out, flat(out), y, (4 * U.F32 + U.STEP[io] * (1 + 2.0 ** -6)) * y.abs() + 1e-37)
        new = (t["k"].cpu(), t["qkv"].cpu().view(SEQ, n, -1, D)[:, :, HEADS + KV:])
        for w in range(2):
            codes, scales = want[w]
            for i in range(SEQ):
                for h in range(KV):
                    c, s = codes[i, :, h].tolist(), scales[i, :, h].tolist()
                    U.append(c, s, BLOCK, new[w][i, :, h].double().tolist(), filled[i])
                    codes[i, :, h], scales[i, :, h] = torch.tensor(c, dtype=torch.uint8), torch.tensor(s, dtype=torch.uint8)
            assert torch.equal(layer.cache[w].view(torch.uint8).cpu(), codes) and torch.equal(layer.scales[w].cpu(), scales)
        kv = [U.cache_values(*want[w], BLOCK).to(io) for w in range(2)]
        value, bound, _ = H.attend_all(t["q"].cpu(), *kv, True, 1 / math.sqrt(D), H.spans(None, None, n, SEQ), H.spans(None, filled, CAP, SEQ))["out"]
        U.check("attention", t["o"], value, 3 * bound if dtype == "f32" else bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_token_captured_and_replayed(dtype):
    """A step captured once and replayed for every token, with eager work of the same kind between the replays, gives the bits of the eager steps."""
    eager, graphed = Layer(dtype), Layer(dtype)
    prompts = []
    for layer in (eager, graphed):
        t = layer.buffers(30)
        layer.fill(t, 1, [30] * SEQ)
        prompts.append(layer.step(t).clone())
    assert torch.equal(*prompts)
    t, g = eager.buffers(1), graphed.buffers(1)
    keep = [[x.clone() for x in (*graphed.cache, *graphed.scales)]]
    graphed.fill(g, 2, [31] * SEQ)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.step(g)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step(g)
    for a, b in zip((*graphed.cache, *graphed.scales), keep[0]):
        a.copy_(b)
    for i in range(12):
        filled = [31 + i, 31 + i, 31 + i]
        eager.fill(t, 10 + i, filled)
        graphed.fill(g, 10 + i, filled)
        want = eager.step(t).clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(g["y"], want), i
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((*eager.cache, *eager.scales), (*graphed.cache, *graphed.scales)))


def test_a_training_step_captured_and_replayed():
    """Norm and its gradients in a graph while the eager calls run on the same tensors between the replays."""
    gen = torch.Generator().manual_seed(3)
    x, dout = (torch.randn(2, 900, 512, generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    w, b = torch.randn(2, 512, generator=gen).to(torch.bfloat16).cuda(), torch.randn(2, 512, generator=gen).to(torch.bfloat16).cuda()

    def step():
        out, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty(2, 512, device="cuda"), torch.empty(2, 512, device="cuda")
        B.layer_norm(x, w, b, out)
        B.layer_norm_backward(x, w, dout, dx, dw, db)
        return out, dx, dw, db

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        x.copy_(torch.randn(2, 900, 512, generator=gen).to(torch.bfloat16))
        want = step()
        graph.replay()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), i


def test_two_streams_at_once():
    """Calls on two streams with tensors and workspaces of their own do not disturb each other."""
    layers, streams = [Layer("bf16", s) for s in (1, 2)], [torch.cuda.Stream() for _ in range(2)]
    alone = []
    for i, layer in enumerate(layers):
        t = layer.buffers(20)
        layer.fill(t, i, [20] * SEQ)
        alone.append(layer.step(t).clone())
    torch.cuda.synchronize()
    ts = []
    for i, layer in enumerate(layers):
        t = layer.buffers(20)
        layer.fill(t, i, [20] * SEQ)
        ts.append(t)
    torch.cuda.synchronize()
    for _ in range(5):
        for layer, t, s in zip(layers, ts, streams):
            with torch.cuda.stream(s):
                layer.step(t)
    torch.cuda.synchronize()
    for t, want in zip(ts, alone):
        assert torch.equal(t["y"], want)
