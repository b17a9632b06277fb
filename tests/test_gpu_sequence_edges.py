"""Attention over sequences where values are not finite, very large, or cancel: what a pair that is seen, or not seen, gives."""
import math

import pytest
import torch

from paper_2604_22808_amd import binding as B
from tests import heads_util as U
from tests.test_gpu_sequence_attention import MARK, Call, ints, offsets

pytestmark = pytest.mark.gpu
N, AT = 300, 150


def pair_of_calls(seed, dtype, n=N, heads=2, kv_heads=1, d=64, causal=True, **change):
    """Two calls of the same inputs; `change` [name: function of the tensor] is made in both, so that it can make scores one-sided."""
    out = []
    for _ in range(2):
        c = Call(seed, dtype, heads, kv_heads, d, n, n, q_offsets=[0, n], k_offsets=[0, n], causal=causal)
        for name, f in change.items():
            c.dev[name].copy_(f(c.dev[name]))
        out.append(c)
    return out


def positive(channel):
    def f(t):
        t = t.clone()
        t[..., channel] = t[..., channel].abs() + 0.5
        return t
    return f


def run(*calls):
    for c in calls:
        c.forward()
        c.backward()


def same(a, b, what):
    assert torch.equal(a, b), (what, float((a.float() - b.float()).abs().nan_to_num(1e30).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_key_without_probability_gets_no_gradient(dtype):
    """Channel 5 of one key is -inf and of all queries positive: its scores are -inf, its probabilities zero, as they are exactly where that channel is -1e5
    (scores thousands below the row's others).  Out, lse, dk and dv keep their bits, also where the queries do not fill their last tile."""
    clean, bad = pair_of_calls(200, dtype, causal=False, q=positive(5))
    clean.dev["k"][AT, :, 5] = -1e5
    bad.dev["k"][AT, :, 5] = -math.inf
    run(clean, bad)
    for n in ("out", "dk", "dv"):
        same(bad.out[n], clean.out[n], n)
    same(bad.lse, clean.lse, "lse")
    assert float(bad.out["dk"][AT].abs().sum()) == 0 and float(bad.out["dv"][AT].abs().sum()) == 0


@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_seen_key_with_an_infinite_channel(dtype, causal):
    """As above: everything keeps its bits but channel 5 of dq, which is not finite for the rows that see the key."""
    clean, bad = pair_of_calls(201, dtype, causal=causal, q=positive(5))
    clean.dev["k"][AT, :, 5] = -1e5
    bad.dev["k"][AT, :, 5] = -math.inf
    run(clean, bad)
    first = AT if causal else 0
    dq, want = bad.out["dq"].clone(), clean.out["dq"].clone()
    assert not bool(torch.isfinite(dq[first:, :, 5]).any())
    dq[first:, :, 5] = want[first:, :, 5] = 0
    same(dq, want, "dq")
    for n in ("out", "dk", "dv"):
        same(bad.out[n], clean.out[n], n)
    same(bad.lse, clean.lse, "lse")
    assert bool(torch.isfinite(want.float()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_infinite_gradient_of_a_row(dtype):
    """Channel 3 of one row of dout is +inf and that channel of v positive: the row's dP and delta are +inf, its dS is NaN.  dv gets +inf in that channel from every key that
    the row sees, dk is NaN there, and keys that it does not see keep their bits."""
    clean, bad = pair_of_calls(202, dtype, v=positive(3))
    bad.dev["dout"][AT, 1, 3] = math.inf
    run(clean, bad)
    seen = AT + 1
    assert bool(torch.isnan(bad.out["dk"][:seen]).all())
    dv, want = bad.out["dv"].clone(), clean.out["dv"].clone()
    assert bool((dv[:seen, :, 3] == math.inf).all())
    dv[:seen, :, 3] = want[:seen, :, 3] = 0
    same(dv, want, "dv")
    same(bad.out["dk"][seen:], clean.out["dk"][seen:], "dk")
    assert bool(torch.isnan(bad.out["dq"][AT, 1]).all())
    rest = torch.ones(N, 2, dtype=torch.bool)
    rest[AT, 1] = False
    same(bad.out["dq"][rest], clean.out["dq"][rest], "dq")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_infinite_value_of_a_key_without_probability(dtype):
    """The scores of one key are -inf and a channel of its value +inf: zero times infinity is NaN in that channel of the rows that see it, on the diagonal as elsewhere."""
    clean, bad = pair_of_calls(203, dtype, q=positive(5))
    clean.dev["k"][AT, :, 5] = -1e5
    bad.dev["k"][AT, :, 5] = -math.inf
    bad.dev["v"][AT, :, 3] = math.inf
    clean.forward()
    bad.forward()
    out, want = bad.out["out"].clone(), clean.out["out"].clone()
    assert bool(torch.isnan(out[AT:, :, 3]).all())
    out[AT:, :, 3] = want[AT:, :, 3] = 0
    same(out, want, "out")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_channel_of_an_infinite_key_that_is_seen(dtype):
    """Its probabilities are zero, and zero times infinity is NaN in that channel of dq: of the rows that see the key, in and behind the tile on the diagonal, and of no others."""
    clean, bad = pair_of_calls(208, dtype, q=positive(5))
    bad.dev["k"][AT, :, 5] = -math.inf
    run(clean, bad)
    assert bool(torch.isnan(bad.out["dq"][AT:, :, 5]).all())
    same(bad.out["dq"][:AT], clean.out["dq"][:AT], "dq")
    assert bool(torch.isfinite(bad.out["dq"][..., :5].float()).all())


@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_row_whose_scores_are_all_minus_infinity(dtype, causal):
    """It sees keys, so its softmax is not that of a row that sees none: out and its gradients are NaN, lse -inf; other rows, and keys that it does not see, keep their bits."""
    clean, bad = pair_of_calls(204, dtype, causal=causal, k=positive(5))
    bad.dev["q"][AT, 0, 5] = -math.inf
    run(clean, bad)
    assert bool(torch.isnan(bad.out["out"][AT, 0]).all()) and float(bad.lse[0, AT]) == -math.inf
    assert bool(torch.isnan(bad.out["dq"][AT, 0]).all())
    seen = AT + 1 if causal else N
    rest = torch.ones(N, 2, dtype=torch.bool)
    rest[AT, 0] = False
    for n in ("out", "dq"):
        same(bad.out[n][rest], clean.out[n][rest], n)
    for n in ("dk", "dv"):
        assert bool(torch.isnan(bad.out[n][:seen]).all()), n
        same(bad.out[n][seen:], clean.out[n][seen:], n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_token_whose_scores_are_minus_infinity_over_a_long_cache(dtype):
    """All of them: NaN and lse -inf, from pieces of the keys too.  Those of the first 1500 keys alone: as without these keys.  A cache that holds none: zeros."""
    calls = []
    for _ in range(2):
        c = Call(205, dtype, 4, 2, 64, 1, 5000, batch=3, k_lengths=[5000, 4000, 0], causal=True)
        c.dev["q"].copy_(positive(5)(c.dev["q"]))
        calls.append(c)
    clean, bad = calls
    clean.dev["k"][1, :1500, :, 5] = -1e5
    bad.dev["k"][1, :1500, :, 5] = -math.inf
    bad.dev["k"][0, :, :, 5] = -math.inf
    for c in calls:
        c.forward()
    assert bool(torch.isnan(bad.out["out"][0]).all()) and bool((bad.lse[:, 0] == -math.inf).all())
    same(bad.out["out"][1:], clean.out["out"][1:], "out")
    same(bad.lse[:, 1:], clean.lse[:, 1:], "lse")
    assert float(bad.out["out"][2].abs().sum()) == 0 and bool((bad.lse[:, 2] == -math.inf).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("rows,keys,batch,heads", [(200, 700, 1, 2), (130, 200, 64, 4), (1, 200, 256, 8)])
def test_values_of_1e30_under_growing_scores(rows, keys, batch, heads, causal, dtype):
    """Scores that grow by some 24 along the keys, and values whose weighted sum is far below the type's largest while e^24 times one of them is above it."""
    d = 64
    c = Call(206, dtype, heads, heads, d, rows, keys, batch=batch, causal=causal, scale=1.0, spread=0.05)
    c.host["q"][..., 0] = 1.0
    c.host["k"][..., 0] = torch.linspace(0.0, 24.0, keys)[None, :, None].to(c.io)
    c.host["v"] = (c.host["v"].double() * 1e30).to(c.io)
    for n in "qkv":
        c.dev[n].copy_(c.host[n])
    c.forward()
    c.check(train=False)


def gradients_of_short_rows(q, k, v, dout, causal, scale, few=128):
    """One sequence and head in 64 bits: dq and dk with bounds for a kernel that sums delta from the probabilities in rows of up to `few` keys, and takes it from the stored bf16 out in others."""
    step, d = U.STEP[torch.bfloat16], q.shape[1]
    nq, nk = q.shape[0], k.shape[0]
    q, k, v, do = (t.double() for t in (q, k, v, dout))
    seen = torch.ones(nq, nk, dtype=torch.bool)
    if causal:
        seen = torch.arange(nk)[None] <= torch.arange(nq)[:, None] + nk - nq
    some = seen.any(1, keepdim=True)
    s = (q @ k.T * scale).masked_fill(~seen, -math.inf)
    lse = torch.where(some, torch.logsumexp(s, 1, keepdim=True), 0.0)
    p = torch.where(seen, torch.exp(s - lse), 0.0)
    out, dp = p @ v, do @ v.T
    # as in heads_util.attend: errors of scores, of probabilities relative to themselves, of dO V^T
    se = U.F32 * (d + 8) * torch.where(seen, q.abs() @ k.abs().T * scale + torch.where(seen, s, 0.0).abs(), 0.0).amax(1, keepdim=True)
    pe = 2 * se + (nk + 16) * U.F32
    dp_e = U.F32 * (d + 4) * (do.abs() @ v.abs().T)
    delta = (p * dp).sum(1, keepdim=True)
    exact = (p * dp_e).sum(1, keepdim=True) + (p * dp.abs()).sum(1, keepdim=True) * (pe + (nk + 4) * U.F32)
    stored = (do.abs() * ((p @ v.abs()) * (pe + step + nk * U.F32) + step * out.abs())).sum(1, keepdim=True) + d * U.F32 * (do * out).abs().sum(1, keepdim=True)
    delta_e = torch.where(seen.sum(1, keepdim=True) <= few, exact, stored)
    ds = p * (dp - delta)
    ds_e = p * (dp_e + delta_e) + ds.abs() * (pe + step + (nq + nk + 8) * U.F32)
    dq, dk = scale * ds @ k, scale * ds.T @ q
    return (dq, scale * ds_e @ k.abs() + step * dq.abs() * (1 + 2.0 ** -6) + 1e-30), (dk, scale * ds_e.T @ q.abs()), seen.sum(1)


@pytest.mark.parametrize("heads,kv_heads,d,nq,nk,causal,pad", [
    (1, 1, 64, 300, 200, True, 0), (4, 1, 64, 300, 340, True, 0), (2, 2, 128, 1, 128, False, 0), (2, 1, 128, 260, 270, True, 0),
    (2, 1, 64, 100, 100, True, 1), (2, 2, 64, 70, 128, False, 1), (1, 1, 64, 300, 200, True, 1), (2, 1, 44, 130, 120, True, 0), (3, 1, 128, 90, 100, True, 1)])
def test_gradients_of_rows_that_see_few_keys(heads, kv_heads, d, nq, nk, causal, pad):
    """bf16, values far from zero: dS is what is left of dO V^T - delta, and half a step of out would be several times the bound.  Whatever other rows a workgroup holds, and whatever
    the rows' alignment."""
    c = Call(207, "bf16", heads, kv_heads, d, nq, nk, q_offsets=[0, nq], k_offsets=[0, nk], causal=causal, pad=pad)
    c.host["v"] = (c.host["v"].double() + 64.0).to(c.io)
    c.host["k"] = (c.host["k"].double() + 1.0).to(c.io)
    for n in "kv":
        c.dev[n].copy_(c.host[n][0])
    run(c)
    group = heads // kv_heads
    dk, dk_b = torch.zeros(nk, kv_heads, d).double(), torch.zeros(nk, kv_heads, d).double()
    for h in range(heads):
        (dq, dq_b), (k1, k1_b), count = gradients_of_short_rows(*(c.host[n][0][:, h if n in ("q", "dout") else h // group] for n in ("q", "k", "v", "dout")), causal, c.scale)
        few = count <= 128
        U.check(("dq", h), c.out["dq"][:, h].cpu()[few], dq[few], dq_b[few])
        dk[:, h // group] += k1
        dk_b[:, h // group] += k1_b
    U.check("dk", c.out["dk"], dk, dk_b + (U.STEP[torch.bfloat16] * (1 + 2.0 ** -6) + group * U.F32) * dk.abs() + 1e-30)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("keys,far", [(200, (32, 64)), (5000, (0, 100)), (5000, (3000, 4000))])
def test_an_infinite_value_far_below_the_others(keys, far, dtype):
    """Scores thousands below the row's largest: probabilities of zero, times an infinity NaN, also where the key is in a piece of the keys of which nothing else counts."""
    c = Call(209, dtype, 4, 2, 64, 1, keys, batch=2, causal=True)
    c.dev["q"].copy_(positive(5)(c.dev["q"]))
    c.dev["k"][0, far[0]:far[1], :, 5] = -1e5
    c.dev["v"][0, far[0] + 20, :, 3] = math.inf
    c.forward()
    assert bool(torch.isnan(c.out["out"][0, :, :, 3]).all())
    c.out["out"][0, :, :, 3] = 0
    assert bool(torch.isfinite(c.out["out"].float()).all())


# ---- the second pass in the other cuts of a call: one-wave tiles, pieces of the keys, pieces of the query rows

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_last_key_that_only_the_last_token_sees(dtype):
    """Four tokens against a long cache: the last row of keys and values is NaN."""
    calls = [Call(210, dtype, 4, 2, 64, 4, 5000, batch=2, causal=True) for _ in range(2)]
    clean, bad = calls
    for n in "kv":
        bad.dev[n][:, -1] = math.nan
    run(*calls)
    for n in ("out", "dq"):
        same(bad.out[n][:, :3], clean.out[n][:, :3], n)
        assert bool(torch.isnan(bad.out[n][:, 3]).all()), n
    same(bad.lse.view(4, 2, 4)[..., :3], clean.lse.view(4, 2, 4)[..., :3], "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_late_key_under_pieces_of_the_keys(dtype):
    n, nk, at = 300, 4096, 4000
    calls = [Call(211, dtype, 2, 1, 64, n, nk, q_offsets=[0, n], k_offsets=[0, nk], causal=True) for _ in range(2)]
    clean, bad = calls
    bad.dev["v"][at, :, 7] = math.inf
    bad.dev["k"][at + 20] = math.nan
    for c in calls:
        c.forward()
    first = at - (nk - n)
    same(bad.out["out"][:first], clean.out["out"][:first], "out")
    assert bool((bad.out["out"][first:first + 20, :, 7] == math.inf).all()) and bool(torch.isnan(bad.out["out"][first + 20:]).all())
    same(bad.lse[:, :first + 20], clean.lse[:, :first + 20], "lse")
    rest = [i for i in range(64) if i != 7]
    same(bad.out["out"][first:first + 20][..., rest], clean.out["out"][first:first + 20][..., rest], "other channels")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_early_queries_under_pieces_of_the_query_rows(dtype):
    n = 1200
    clean, bad = pair_of_calls(212, dtype, n=n)
    bad.dev["q"][499] = math.nan
    bad.dev["dout"][500, 0, 9] = math.inf
    run(clean, bad)
    for name in ("dk", "dv"):
        same(bad.out[name][501:], clean.out[name][501:], name)
        assert not bool(torch.isfinite(bad.out[name][:500].float()).all(-1).any()), name


# ---- offsets and workspaces

def wrong_offsets(n, rows, seed):
    gen = torch.Generator().manual_seed(seed)
    top = 2 ** 31 - 1
    yield torch.randint(-2 ** 31, top, (n + 1,), generator=gen).tolist()
    yield torch.randint(-rows, 2 * rows, (n + 1,), generator=gen).tolist()
    yield torch.randint(0, rows + 1, (n + 1,), generator=gen).sort(descending=True).values.tolist()
    yield [-2 ** 31, top] * ((n + 2) // 2) if n % 2 else [0] + [top] * n


class Guarded:
    """A tensor inside a larger one whose other elements hold `guard`."""
    def __init__(self, shape, dtype, fill, guard, edge=8192):
        n = math.prod(shape)
        self.all, self.edge, self.n = torch.full((n + 2 * edge,), guard, dtype=dtype, device="cuda"), edge, n
        self.x = self.all[edge:edge + n].view(shape)
        self.x.copy_(fill) if isinstance(fill, torch.Tensor) else self.x.fill_(fill)
        self.guard = self.all[:edge].clone()

    def untouched(self):
        return torch.equal(self.all[:self.edge], self.guard) and torch.equal(self.all[self.edge + self.n:], self.guard)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 70])
def test_wrong_offsets_read_and_write_inside_alone(n, dtype):
    """Offsets that point outside, descend or overlap: outputs and workspaces keep the marks around them, and the NaN around the inputs reaches no result.  (Which results they are is open;
    workspaces of zeros and marks of small numbers make them finite.)"""
    rows, h, hk, d = 200, 4, 2, 64
    io = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator().manual_seed(213)
    for i, off in enumerate(wrong_offsets(n, rows, 214)):
        src = {m: Guarded((rows, x, d), io, torch.randn(rows, x, d, generator=gen).to(io).cuda(), math.nan) for m, x in (("q", h), ("k", hk), ("v", hk), ("dout", h))}
        dst = {m: Guarded((rows, x, d), io, 0.5, MARK) for m, x in (("out", h), ("dq", h), ("dk", hk), ("dv", hk))}
        lse = Guarded((h, rows), torch.float32, 1.0, MARK)
        how = dict(causal=i % 2 == 0, q_offsets=ints(off), k_offsets=ints(off if i == 1 else off[::-1]), q_lengths=ints([rows // 2] * n) if i == 2 else None)
        shape = B.SequenceShape(n, h, hk, d, rows, rows, B.BF16 if dtype == "bf16" else B.F32, 0, 0.0)
        which = B.SequenceRows(16, 16, None, None)
        ws = [Guarded((max(16, f(shape, which)),), torch.uint8, 0, 90) for f in (B.lib().freqattn_sequence_attention_workspace, B.lib().freqattn_sequence_attention_backward_workspace)]
        B.sequence_attention(*(src[m].x for m in "qkv"), dst["out"].x, lse=lse.x, workspace=ws[0].x, **how)
        # a row that two sequences own may be left with the lse of the one in which it sees no key (-inf): the other's exp(score - lse) is not finite, so lse is given here
        lse.x.fill_(1.0)
        B.sequence_attention_backward(*(src[m].x for m in ("dout", "q", "k", "v")), dst["out"].x, lse.x, *(dst[m].x for m in ("dq", "dk", "dv")), workspace=ws[1].x, **how)
        torch.cuda.synchronize()
        for m, t in {**dst, "lse": lse, "workspace": ws[0], "backward workspace": ws[1]}.items():
            assert t.untouched(), (n, i, m)
        for m, t in dst.items():
            assert bool(torch.isfinite(t.x.float()).all()), (n, i, m)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_rows,k_rows,causal", [(1, 5000, True), (300, 4096, True), (1500, 1500, False)])
def test_what_a_workspace_holds_does_not_matter(q_rows, k_rows, causal, dtype):
    c = Call(215, dtype, 4, 2, 64, q_rows, k_rows, batch=2, causal=causal, k_lengths=[k_rows, k_rows - 77])
    run(c)
    want = [t.clone() for t in (*c.out.values(), c.lse)]
    lens = c.how["k_lengths"]
    shape = B.SequenceShape(2, 4, 2, 64, q_rows, k_rows, B.BF16 if dtype == "bf16" else B.F32, int(causal), 0.0)
    which = B.SequenceRows(None, None, None, lens.data_ptr())
    need = max(f(shape, which) for f in (B.lib().freqattn_sequence_attention_workspace, B.lib().freqattn_sequence_attention_backward_workspace))
    d, o = c.dev, c.out
    for fill in (math.nan, math.inf):
        ws = torch.full((need // 4 + 4,), fill, device="cuda")
        B.sequence_attention(d["q"], d["k"], d["v"], o["out"], lse=c.lse, workspace=ws, **c.how)
        ws.fill_(fill)
        B.sequence_attention_backward(d["dout"], d["q"], d["k"], d["v"], o["out"], c.lse, o["dq"], o["dk"], o["dv"], workspace=ws, **c.how)
        for got, w in zip((*o.values(), c.lse), want):
            same(got, w, fill)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_tokens_against_packed_keys(dtype):
    """One query row, or some, of each of 24 sequences whose keys lie behind each other: the keys are split by all rows there are, and sequences end inside pieces."""
    kl = [(37 * i) % 700 + 1 for i in range(24)]
    for ql in ([1] * 24, [(i * 5) % 3 for i in range(24)]):
        c = Call(216, dtype, 4, 2, 64, sum(ql) + 2, sum(kl) + 5, q_offsets=offsets(*ql), k_offsets=offsets(*kl), causal=True, spoil=True)
        run(c)
        c.check()
